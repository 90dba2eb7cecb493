"""AdamW over a list of tensors, and the norm of its gradients, against the formulas in float64.

Tolerances, with u = 2^-24: m and v take three float32 roundings of their terms (4 u of the magnitudes); a step is
the quotient of m by sqrt(v) and eps, both with their errors, and four roundings (12 u of the step and 4 u of the terms of
m over the denominator), p adds one (u |p|).  A stored code is one of the two codes next to the quotient; which of them is the
random bits' to say, except within 4 u of the quotient (or 16 u where the block's scale is near
the smallest normal) around the border; codes are compared outside of that.
"""
import math

import pytest

torch = pytest.importorskip("torch")
np = pytest.importorskip("numpy")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BLOCK = 256
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.02)
SIZES = [[1], [3, 1, 2], [255, 256, 257], [4096], [4095, 4097, 1, 8192], [100003], [5] * 130, [64, 70000, 1, 300000, 17]]


def step():
    from paper_2408_14267_amd import step as s
    return s


def normal(n, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + n)
    return scale * torch.randn(n, generator=g, device="cuda")


def placed(t, offset):
    """t at an offset of elements inside a buffer of sentinels; and a check of those."""
    raw = torch.full((t.numel() + offset + 9,), 7, device="cuda").to(t.dtype)
    v = raw[offset:offset + t.numel()]
    v.copy_(t)

    def intact():
        assert (raw[:offset].float() == 7).all() and (raw[offset + t.numel():].float() == 7).all()
    return v, intact


def blocks(t):
    """t in rows of BLOCK, zero past its end."""
    return torch.nn.functional.pad(t, (0, -t.numel() % BLOCK)).view(-1, BLOCK)


def coded(t):
    scale = blocks(t).abs().amax(dim=1) / 448
    q = (blocks(t) / scale.clamp_min(1e-30)[:, None]).view(-1)[:t.numel()].to(torch.float8_e4m3fn)
    return q, scale


def worth(q, scale):
    return (blocks(q.double()) * scale.double()[:, None]).view(-1)[:q.numel()]


def make(sizes, states, gt="f32", offset=0, seed=0):
    """Lists of tensors and their checks, as a dict."""
    o = {k: [] for k in ("g", "p", "m", "v", "m_scale", "v_scale")}
    checks = []

    def put(name, t):
        v, ok = placed(t, offset)
        o[name].append(v)
        checks.append(ok)

    for i, n in enumerate(sizes):
        rate = torch.exp(normal(n, 31 * i + seed)) * 1e-3
        put("g", (rate * normal(n, 37 * i + 1 + seed)).to(torch.bfloat16 if gt == "bf16" else torch.float32))
        put("p", normal(n, 41 * i + 2 + seed))
        m, v = rate * normal(n, 43 * i + 3 + seed, 0.3), (rate * (1 + 0.1 * normal(n, 47 * i + 4 + seed))).square()
        if states == "f32":
            put("m", m)
            put("v", v)
        else:
            for name, t in (("m", m), ("v", v.sqrt())):
                q, scale = coded(t)
                put(name, q)
                put(name + "_scale", scale)
    if states == "f32":
        o["m_scale"] = o["v_scale"] = None
    return o, checks


def words(first, n, seed, t):
    from oracle import philox
    return philox.uniform_words(np.arange(first, first + n, dtype=np.uint64), 3, seed, t, 0).astype(np.int64)


def expected(o, i, t, scale, hyper):
    """p, m, v in float64 after the step, and the terms of m."""
    s = 1.0 if scale is None else float(scale)
    g = o["g"][i].double() * s
    if o["m_scale"] is None:
        m0, v0 = o["m"][i].double(), o["v"][i].double()
    else:
        m0, v0 = worth(o["m"][i], o["m_scale"][i]), worth(o["v"][i], o["v_scale"][i]).square()
    b1, b2 = hyper["beta1"], hyper["beta2"]
    m, v = b1 * m0 + (1 - b1) * g, b2 * v0 + (1 - b2) * g * g
    terms = b1 * m0.abs() + (1 - b1) * g.abs()
    den = (v / (1 - b2 ** t)).sqrt() + hyper["eps"]
    rate = hyper["lr"] / (1 - b1 ** t)
    p0 = o["p"][i].double()
    decay = hyper["lr"] * hyper["weight_decay"]
    p = p0 - decay * p0 - rate * m / den
    lim = 2 * U * p0.abs() + (12 * (m.abs()) + 4 * terms) * U * rate / den
    return p, m, v, terms, lim


def unit_at(size):
    """The step of e4m3 at `size` (of float64; a table, since powers on the device are rounded)."""
    powers = torch.tensor([2.0 ** k for k in range(-9, 8)], dtype=torch.float64, device="cuda")
    return powers[(torch.frexp(size)[1] - 1).clamp(-6, 8).long() + 6]


def check_codes(q, scale, want, bits, least, what):
    """Codes of `want` (float64) with the scales and the random bits."""
    top = blocks(want).abs().amax(dim=1)
    assert ((scale.double() - top / 448).abs() <= 8 * U * top / 448 + 1e-45).all(), what
    y = (blocks(want) / torch.where(top > 0, top / 448, 1.0)[:, None]).view(-1)[:want.numel()]
    size = y.abs()
    unit = unit_at(size)
    bits = torch.from_numpy(bits).to("cuda").double() / 65536
    low, high = ((size * (1 + k * 16 * U) / unit + bits).floor() * unit for k in (-1, 1))
    low, high = low.clamp(max=448), high.clamp(max=448)
    if least:
        low, high = (torch.where((want > 0) & (c == 0), 2.0 ** -9, c) for c in (low, high))
    got = q.double()
    assert (got.abs() >= low).all() and (got.abs() <= high).all(), what
    assert ((got == 0) | (torch.sign(got) == torch.sign(want))).all(), what


def run(o, t, states, scale=None, seed=11, first=None, device_step=False, **hyper):
    s = step()
    h = dict(HYPER, **hyper)
    cfg = s.adamw_cfg(seed=seed, states=states, **h)
    params = s.param_list(o["g"], o["p"], o["m"], o["v"], o["m_scale"], o["v_scale"], first=first)
    grad_scale = None if scale is None else torch.tensor([scale], device="cuda")
    number = torch.tensor([t], device="cuda") if device_step else t
    s.fqt_adamw_step(cfg, params, number, grad_scale=grad_scale)
    torch.cuda.synchronize()


def check(sizes, states, t, gt="f32", offset=0, scale=None, seed=11, first=None, device_step=False, **hyper):
    o, intact = make(sizes, states, gt, offset)
    h = dict(HYPER, **hyper)
    want = [expected(o, i, t, None if scale is None else torch.tensor(scale).item(), h) for i in range(len(sizes))]
    run(o, t, states, scale, seed, first, device_step, **hyper)
    at = 0
    for i, n in enumerate(sizes):
        p, m, v, terms, lim = want[i]
        err = (o["p"][i].double() - p).abs()
        assert (err <= lim).all(), f"p[{i}]: off by {(err / lim).max().item():.3g} of the bound"
        if states == "f32":
            assert ((o["m"][i].double() - m).abs() <= 4 * U * terms).all()
            assert ((o["v"][i].double() - v).abs() <= 6 * U * v + 1e-44).all()
        else:
            w = words(at if first is None else first[i], n, seed, t)
            # (m is off by its terms' roundings: those near a border of theirs are left to the bound of a step)
            near = terms <= 4 * m.abs()
            check_codes(torch.where(near, o["m"][i].float(), 0.0), o["m_scale"][i], m, w & 0xFFFF, False, f"m[{i}]") \
                if bool(near.all()) else check_m(o["m"][i], o["m_scale"][i], m, terms, w & 0xFFFF, f"m[{i}]")
            check_codes(o["v"][i], o["v_scale"][i], v.sqrt(), w >> 16, True, f"v[{i}]")
        at += -(-n // BLOCK) * BLOCK
    for ok in intact:
        ok()


def check_m(q, scale, m, terms, bits, what):
    """As check_codes, with the error of m itself (4 u of its terms) around each border."""
    top = blocks(m).abs().amax(dim=1)
    assert ((scale.double() - top / 448).abs() <= 8 * U * (top + blocks(terms).amax(dim=1)) / 448 + 1e-45).all(), what
    unit_of = torch.where(top > 0, top / 448, 1.0)
    y = (blocks(m) / unit_of[:, None]).view(-1)[:m.numel()]
    slack = (blocks(terms) / unit_of[:, None]).view(-1)[:m.numel()] * 4 * U + y.abs() * 16 * U
    bits = torch.from_numpy(bits).to("cuda").double() / 65536

    def code(size):
        size = size.clamp(min=0)
        unit = unit_at(size)
        return ((size / unit + bits).floor() * unit).clamp(max=448)

    got = q.double()
    assert (got.abs() >= code(y.abs() - slack)).all() and (got.abs() <= code(y.abs() + slack)).all(), what
    assert ((got == 0) | (torch.sign(got) == torch.sign(m)) | (y.abs() <= slack)).all(), what


@pytest.mark.parametrize("sizes", SIZES, ids=str)
@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("gt", ["f32", "bf16"])
def test_adamw(sizes, states, gt):
    check(sizes, states, 5, gt)


@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("t", [1, 2, 1000, 1 << 20, (1 << 32) + 7])
def test_adamw_at_steps(states, t):
    check([300, 5000], states, t)
    check([300, 5000], states, t, device_step=True)


@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("offset", [1, 2, 3])
def test_adamw_of_unaligned_tensors(states, offset):
    for gt in ("f32", "bf16"):
        check([1, 1021, 4099], states, 3, gt, offset=offset)


@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_adamw_options(states):
    sizes = [700, 33]
    check(sizes, states, 9, scale=0.125)
    check(sizes, states, 9, weight_decay=0.0)
    check(sizes, states, 9, beta1=0.0)
    check(sizes, states, 9, beta1=0.5, beta2=0.9, eps=1e-3, lr=0.5)
    check(sizes, states, 9, seed=(1 << 63) + 12345, first=[(1 << 34) + 8, 4])


@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_zero_gradients_move_nothing_from_zero_states(states):
    o, _ = make([1000], states)
    for k in ("g", "m", "v"):
        o[k][0].copy_(torch.zeros_like(o[k][0].float()).to(o[k][0].dtype))
    before = o["p"][0].clone()
    run(o, 1, states, weight_decay=0.0)
    assert torch.equal(o["p"][0], before)
    assert (o["m"][0].float() == 0).all() and (o["v"][0].float() == 0).all()
    if states == "e4m3":
        assert (o["m_scale"][0] == 0).all() and (o["v_scale"][0] == 0).all()


def test_a_second_moment_does_not_vanish_beside_a_large_one():
    """An element a million times smaller than its block's largest: its v keeps the smallest code, so a step
    with no gradient stays of the size of its m over it."""
    o, _ = make([256], "e4m3")
    g = torch.full((256,), 1e-6, device="cuda")
    g[0] = 1e6
    for k in ("m", "v"):
        o[k][0].copy_(torch.zeros(256, device="cuda").to(torch.float8_e4m3fn))
    o["g"][0].copy_(g)
    run(o, 1, "e4m3")
    assert (o["v"][0].float() > 0).all()
    o["g"][0].zero_()
    before = o["p"][0].clone()
    run(o, 2, "e4m3", weight_decay=0.0)
    assert ((o["p"][0] - before).abs() <= 10 * HYPER["lr"]).all()


def test_stochastic_rounding_has_no_bias():
    """One value over many elements and seeds: the mean of what is stored is the value, within five standard errors of
    a rounding between neighbours (at most half a step each)."""
    n, value = 200 * 256, 0.3
    o, _ = make([n], "e4m3")
    total = {"m": 0.0, "v": 0.0}
    for seed in range(8):
        for k in ("m", "v"):
            o[k][0].copy_(torch.zeros(n, device="cuda").to(torch.float8_e4m3fn))
        g = torch.full((n,), value, device="cuda")
        g[::256] = 1.0                                       # the block's largest
        o["g"][0].copy_(g)
        run(o, 1, "e4m3", seed=seed, beta1=0.0, beta2=0.0)
        keep = torch.arange(n, device="cuda") % 256 != 0
        for k in ("m", "v"):
            total[k] += worth(o[k][0], o[k + "_scale"][0])[keep].mean().item() / 8
    unit = 16.0 / 448                                        # 0.3 * 448 = 134.4 lies between 128 and 144
    for k, v in total.items():
        assert abs(v - value) <= 5 * unit / 2 / math.sqrt(8 * 255 * 200) + 2.0 ** -16 * unit, k


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_is_not_finite_stays_in_its_block(bad):
    o, _ = make([1024], "e4m3")
    p, _ = make([1024], "e4m3")
    o["g"][0][300] = bad
    run(o, 3, "e4m3")
    run(p, 3, "e4m3")
    assert not torch.isfinite(o["p"][0][300])
    keep = torch.arange(1024, device="cuda") != 300
    assert torch.equal(o["p"][0][keep], p["p"][0][keep])
    assert not torch.isfinite(o["m_scale"][0][1]) and torch.isfinite(o["m_scale"][0][[0, 2, 3]]).all()
    assert torch.equal(o["m"][0].float()[512:], p["m"][0].float()[512:])


def test_tiny_blocks_are_stored_as_zeros():
    o, _ = make([256], "e4m3")
    for k in ("m", "v"):
        o[k][0].copy_(torch.zeros(256, device="cuda").to(torch.float8_e4m3fn))
    o["g"][0].fill_(2.0 ** -104)
    run(o, 1, "e4m3")
    assert (o["m"][0].float() == 0).all() and (o["m_scale"][0] == 0).all() and torch.isfinite(o["p"][0]).all()


def test_many_tensors():
    """More than a launch takes."""
    check([(i * 37) % 600 + 1 for i in range(333)], "e4m3", 2)
    check([(i * 37) % 600 for i in range(333)], "f32", 2)


def test_equal_steps_give_equal_bits():
    a, _ = make([5000, 70], "e4m3")
    b, _ = make([5000, 70], "e4m3")
    run(a, 4, "e4m3")
    run(b, 4, "e4m3")
    for k in ("p", "m", "v", "m_scale", "v_scale"):
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a[k], b[k]))


@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_captured_steps(states):
    """Norm and step in a graph, the step number in device memory: replays go on as eager steps do."""
    s = step()
    a, _ = make([5000, 70, 256], states)
    b, _ = make([5000, 70, 256], states)
    cfg = s.adamw_cfg(seed=3, states=states, **HYPER)

    def state(o):
        params = s.param_list(o["g"], o["p"], o["m"], o["v"], o["m_scale"], o["v_scale"])
        out, ws = torch.empty(2, device="cuda"), s.grad_norm_workspace(params)
        return params, out, ws

    pa, oa, wa = state(a)
    pb, ob, wb = state(b)
    number = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        number += 1
        s.fqt_grad_norm(pa, oa, wa, max_norm=0.01)
        s.fqt_adamw_step(cfg, pa, number, grad_scale=oa[1:])
    for t in range(1, 6):
        for x, y in zip(a["g"], b["g"]):
            g = normal(x.numel(), t, 1e-2)
            x.copy_(g)
            y.copy_(g)
        graph.replay()
        s.fqt_grad_norm(pb, ob, wb, max_norm=0.01)
        s.fqt_adamw_step(cfg, pb, t, grad_scale=ob[1:])
        torch.cuda.synchronize()
        assert torch.equal(oa, ob)
        for k in ("p", "m", "v"):
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a[k], b[k])), (t, k)


# ----------------------------------------------------------------------------- norm

def norm_of(g, max_norm=math.inf):
    s = step()
    params = s.param_list(g)
    out = torch.full((4,), 7.0, device="cuda")
    s.fqt_grad_norm(params, out[1:3], s.grad_norm_workspace(params), max_norm=max_norm)
    assert out[0] == 7 and out[3] == 7
    return out[1].item(), out[2].item()


@pytest.mark.parametrize("sizes", SIZES + [[0], [], [8192], [8191, 8193, 1], [1000003]], ids=str)
@pytest.mark.parametrize("gt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1])
def test_norm(sizes, gt, offset):
    g = [placed(normal(n, i + 5).to(gt), offset)[0] for i, n in enumerate(sizes)]
    want = math.sqrt(sum(t.double().square().sum().item() for t in g))
    for max_norm in (0.5, 1e9, math.inf):
        norm, factor = norm_of(g, max_norm)
        assert abs(norm - want) <= 2 * U * want
        clip = min(1.0, max_norm / (want + 1e-6)) if max_norm < math.inf else 1.0
        assert abs(factor - clip) <= 4 * U * clip


def test_norm_of_large_and_tiny_and_bad():
    n = 10000
    for scale in (1e30, 1e-30):
        g = normal(n, 1) * scale
        norm, _ = norm_of([g])
        want = g.double().norm().item()
        assert abs(norm - want) <= 2 * U * want
    g = normal(n, 1)
    g[77] = math.inf
    assert norm_of([g], 1.0) == (math.inf, 0.0)
    g[78] = math.nan
    norm, factor = norm_of([g], 1.0)
    assert math.isnan(norm) and math.isnan(factor)
