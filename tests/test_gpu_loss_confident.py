"""Gradients of rows whose target is nearly certain: dz at the target, p - 1, relative to itself.

Tolerances, with u = 2^-24 and the formulas of the other tests of the loss.  At the target p - 1 = expm1(log p), and log p
is z - lse with z in float64: its rounding to float32 u, expm1 2 u relative to its result, which for log p > -log 2 is at most 1.4 times as
sensitive, its factor and the product u each: 8 u of dz.  A target below 1/2 and the other classes as anywhere: p by 600 u and z's
error, then 4 u of |lse| p and 4 u of the terms.  Sums over M rows M u of the sum of magnitudes.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = 2.0 ** -8
IGNORE = -100


def step():
    from paper_2408_14267_amd import step as s
    return s


def quantized(x, w, kind):
    """The operands, their scales and their float64 values."""
    if kind == "bf16":
        x, w = x.bfloat16(), w.bfloat16()
        return x, w, None, None, x.double(), w.double()
    top, dt = (127.0, torch.int8) if kind == "int8" else (448.0, torch.float8_e4m3fn)
    sx, sw = (t.abs().amax(dim=1).clamp_min(1e-20) / top for t in (x, w))
    x, w = x / sx[:, None], w / sw[:, None]
    x, w = (t.round() if kind == "int8" else t for t in (x, w))
    x, w = x.to(dt), w.to(dt)
    return x, w, sx, sw, x.float().double() * sx.double()[:, None], w.float().double() * sw.double()[:, None]


def make(M, N, K, kind, seed, low=6.0, high=30.0):
    """Rows that point at their target's weights by different lengths."""
    g = torch.Generator(device="cuda").manual_seed(seed * 104729 + 31 * M + 7 * N + K)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    w = normal(N, K)
    w /= w.norm(dim=1, keepdim=True)
    t = torch.randint(0, N, (M,), generator=g, device="cuda")
    size = low + (high - low) * torch.rand(M, generator=g, device="cuda")
    x = 0.3 * normal(M, K) + size[:, None] * w[t]
    o = dict(zip(("x", "w", "x_scale", "w_scale", "x64", "w64"), quantized(x, w, kind)))
    o["bias"] = 0.3 * normal(N)
    o["target"] = torch.where(torch.rand(M, generator=g, device="cuda") < 0.3, IGNORE, t) if M > 1 else t
    return o


def logits(o):
    z = o["x64"] @ o["w64"].t().contiguous() + o["bias"].double()
    mag = o["x64"].abs() @ o["w64"].abs().t().contiguous() + o["bias"].double().abs()
    return z, ((o["x"].shape[1] + 8) * U * mag).amax(dim=1)


def check(got, o, z, zerr, lse, c, smoothing, own=0.0):
    """dbias, dx and dw (float32) against the formulas with this lse (float64).  own: what dz at a likely target may be
    off by beside 8 u, relative to itself."""
    M, N = z.shape
    t = o["target"].clamp(min=0)[:, None]
    c = torch.where(o["target"] == IGNORE, 0.0, c.double())
    logp = z - lse[:, None]
    p = torch.exp(logp)
    q = torch.full_like(z, smoothing / N).scatter_add_(1, t, torch.full_like(z[:, :1], 1 - smoothing))
    dz = p - q
    at = logp.gather(1, t)
    likely = at > -math.log(2.0)
    dz.scatter_(1, t, torch.where(likely, torch.expm1(at) + (smoothing - smoothing / N), dz.gather(1, t)))
    lim = p * (600 * U + 2 * zerr[:, None] + 4 * U * lse.abs()[:, None]) + 4 * U * (p + q)
    off = (8 * U + own) * torch.expm1(at).abs() + 8 * U * smoothing
    lim.scatter_(1, t, torch.where(likely, off, lim.gather(1, t)))
    dz, lim = dz * c[:, None], lim * c.abs()[:, None] + M * U * (dz * c[:, None]).abs()
    d16 = lim + HALF * (dz.abs() + lim)
    x, w = o["x64"], o["w64"]
    sums = {"dbias": (dz.sum(dim=0), lim.sum(dim=0)),
            "dx": (dz @ w, d16 @ w.abs() + N * U * (dz.abs() @ w.abs())),
            "dw": (dz.t().contiguous() @ x, d16.t().contiguous() @ x.abs() + M * U * (dz.abs().t().contiguous() @ x.abs()))}
    for k, v in got.items():
        want, bound = sums[k]
        bound = bound + 2 * U * want.abs() + 1e-37
        err = (v.double() - want).abs()
        assert torch.isfinite(v).all() and (err <= bound).all(), f"{k}: off by {(err / bound).max().item():.3g} of the bound"


def gradients(o, kind, lse, c, smoothing, **kw):
    s = step()
    (M, K), N = o["x"].shape, o["w"].shape[0]
    desc = s.loss_desc(M, N, K, x_dtype=kind, dx_dtype="f32", dw_dtype="f32", smoothing=smoothing, ignore=IGNORE)
    out = {"dx": torch.empty(M, K, device="cuda"), "dw": torch.empty(N, K, device="cuda"),
           "dbias": torch.empty(N, device="cuda")}
    s.fqt_loss_backward(desc, o["x"], o["w"], o["target"], lse, s.loss_workspace(desc, True), dloss=c, bias=o["bias"],
                        x_scale=o["x_scale"], w_scale=o["w_scale"], **out, **kw)
    return out


# (1 to 64 rows of 2048 and 4096 features: a split contraction; odd features: copied operands; 9000 x 20011: pieces)
SIZES = [(1, 2, 8), (1, 10, 64), (1, 10, 594), (3, 10, 4096), (10, 10, 512), (5, 7, 3), (1, 1000, 4096), (16, 1000, 2048),
         (64, 1000, 4096), (65, 129, 300), (130, 10007, 140), (300, 700, 128), (777, 1000, 513), (2304, 4864, 64),
         (5000, 10, 32), (4608, 12288, 1024), (9000, 20011, 72)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("smoothing", [0.0, 0.1])
def test_gradients_for_an_lse(M, N, K, kind, smoothing):
    """The definition, exp(z - lse), with the float32 lse that is given."""
    if smoothing and M * N > 10 ** 7:
        pytest.skip("sizes of the unsmoothed case")
    o = make(M, N, K, kind, seed=1)
    z, zerr = logits(o)
    lse = torch.logsumexp(z, dim=1).float()
    c = torch.randn(M, generator=torch.Generator(device="cuda").manual_seed(M), device="cuda")
    check(gradients(o, kind, lse, c, smoothing), o, z, zerr, lse.double(), c, smoothing)


# ----------------------------------------------------------------------------- from the forward's own outputs

def peaked(M, N, K, kind, seed):
    """Rows of losses from 1e-1 to 1e-7 under top logits of 10 to 80, a few with another target than the largest; class n
    reads feature n alone, so that z is known to the last bit but for the scales' roundings."""
    assert K >= N
    g = torch.Generator(device="cuda").manual_seed(seed + M + N)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    top = torch.tensor([10.0, 20.0, 40.0, 80.0], device="cuda")[torch.randint(0, 4, (M,), generator=g, device="cuda")]
    loss = 10.0 ** -(1 + 6 * uniform(M))
    t = torch.randint(0, N, (M,), generator=g, device="cuda")
    x = torch.zeros(M, K, device="cuda")
    x[:, :N] = (top + torch.log(loss / max(N - 1, 1)))[:, None] + uniform(M, N) - 0.5
    x.scatter_(1, t[:, None], top[:, None])
    w = torch.zeros(N, K, device="cuda")
    w[torch.arange(N), torch.arange(N)] = 1.0
    o = dict(zip(("x", "w", "x_scale", "w_scale", "x64", "w64"), quantized(x, w, kind)))
    o["bias"] = torch.randint(-2, 3, (N,), generator=g, device="cuda").float() / 8
    if M > 4:
        t = torch.where(uniform(M) < 0.1, (t + 1) % N, t)
        t = torch.where(uniform(M) < 0.1, IGNORE, t)
    o["target"] = t
    return o


PEAKED = [(1, 2, 8), (1, 10, 64), (3, 10, 4096), (4, 5000, 5000), (10, 10, 16), (20, 300, 333), (64, 1000, 4096), (300, 700, 768),
          (513, 300, 320), (1500, 1000, 1024), (2304, 5000, 5120)]


@pytest.mark.parametrize("M,N,K", PEAKED)
@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("smoothing", [0.0, 0.01])
def test_gradients_from_the_forward(M, N, K, kind, smoothing):
    """Forward, then backward: the gradients of the loss itself, relative to themselves where it is small.

    log p = -((top - y) log 2 + log1p(rest)) is off by the exponents of rest: y and top by 2^-25 |y| each (|z| <= 81 here: 80 u of an
    exponential), the scales' products another 3 u of |z| each, 2 u the instruction, 4 u each of at most 80 additions: 420 u and 6 u |z|, within
    600 u and 8 u |z|."""
    s = step()
    o = peaked(M, N, K, kind, seed=1)
    z, _ = logits(o)
    desc = s.loss_desc(M, N, K, x_dtype=kind, smoothing=smoothing, ignore=IGNORE)
    loss, lse, logp = (torch.full((M,), 7.0, device="cuda") for _ in range(3))
    args = dict(bias=o["bias"], x_scale=o["x_scale"], w_scale=o["w_scale"])
    s.fqt_loss_forward(desc, o["x"], o["w"], o["target"], loss, lse, s.loss_workspace(desc), logp=logp, **args)
    again = [torch.empty(M, device="cuda") for _ in range(2)]
    s.fqt_loss_forward(desc, o["x"], o["w"], o["target"], *again, s.loss_workspace(desc), **args)
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
    big = z.abs().amax(dim=1)
    zerr = 8 * U * big
    own = 600 * U + 8 * U * big[:, None]
    # log p itself, without the largest's own 1 in the sum
    counted = o["target"] != IGNORE
    t = o["target"].clamp(min=0)[:, None]
    rest = torch.exp(z - z.amax(dim=1, keepdim=True)).scatter_(1, z.argmax(dim=1, keepdim=True), 0.0).sum(dim=1)
    exact = (z.gather(1, t)[:, 0] - z.amax(dim=1)) - torch.log1p(rest)
    assert (logp[~counted] == 0).all()
    assert ((logp.double() - exact).abs() <= (own[:, 0] * torch.log1p(rest) + 12 * U * big * (exact < -0.5)))[counted].all()
    if not smoothing:
        assert torch.equal(logp[counted], -loss[counted])
    c = torch.randn(M, generator=torch.Generator(device="cuda").manual_seed(M), device="cuda")
    top = z.amax(dim=1, keepdim=True)
    check(gradients(o, kind, lse, c, smoothing, logp=logp), o, z, zerr, (top[:, 0] + torch.log1p(rest)), c, smoothing, own)


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_gradients_of_a_layer(kind, reduction):
    """Linear.loss: the gradient of the bias over rows that are all nearly certain."""
    from paper_2408_14267_amd import blocks
    M, N, K = 40, 30, 64
    o = peaked(M, N, K, "bf16", seed=2)
    mod = blocks.Linear(K, N, operands=kind).cuda()
    mod.weight.data.copy_(o["w"].float())
    mod.bias.data.copy_(o["bias"])
    x = o["x"].float()
    q = dict(zip(("x", "w", "x_scale", "w_scale", "x64", "w64"), quantized(x, o["w"].float(), kind)), bias=o["bias"])
    z, _ = logits(q)
    target = z.argmax(dim=1)
    mod.loss(x, target, reduction=reduction).sum().backward()
    rest = torch.exp(z - z.amax(dim=1, keepdim=True)).scatter_(1, target[:, None], 0.0)
    dz = torch.exp(z - z.amax(dim=1, keepdim=True) - torch.log1p(rest.sum(dim=1, keepdim=True)))
    dz.scatter_(1, target[:, None], torch.expm1(-torch.log1p(rest.sum(dim=1, keepdim=True))))
    if reduction == "mean":
        dz = dz / M
    # (every term by 1300 u and 16 u of |z| <= 81, and the sums)
    bound = (2600 + M) * U * dz.abs().sum(dim=0)
    assert ((mod.bias.grad.double() - dz.sum(dim=0)).abs() <= bound).all()


# ----------------------------------------------------------------------------- rows and calls

@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
def test_more_rows_than_a_launch_has_waves(kind):
    M, N, K = 70001, 10, 40
    o = make(M, N, K, kind, seed=3)
    z, zerr = logits(o)
    lse = torch.logsumexp(z, dim=1).float()
    c = torch.randn(M, generator=torch.Generator(device="cuda").manual_seed(M), device="cuda") / 100
    check(gradients(o, kind, lse, c, 0.0), o, z, zerr, lse.double(), c, 0.0)


@pytest.mark.parametrize("M,N,K", [(6, 30, 100), (64, 1000, 2048), (300, 700, 96)])
@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
def test_strided_rows(M, N, K, kind):
    s = step()
    o = make(M, N, K, kind, seed=4)
    z, zerr = logits(o)
    lse = torch.logsumexp(z, dim=1).float()
    c = torch.randn(M, generator=torch.Generator(device="cuda").manual_seed(M), device="cuda")
    want = gradients(o, kind, lse, c, 0.0)
    for more in (3, 32):
        wide = [torch.full((t.shape[0], K + more), 3.0, device="cuda").to(t.dtype) for t in (o["x"], o["w"])]
        for t, v in zip(wide, (o["x"], o["w"])):
            t[:, :K] = v
        desc = s.loss_desc(M, N, K, x_dtype=kind, dx_dtype="f32", dw_dtype="f32", ignore=IGNORE, ldx=K + more, ldw=K + more)
        out = {k: torch.empty_like(v) for k, v in want.items()}
        s.fqt_loss_backward(desc, wide[0][:, :K], wide[1][:, :K], o["target"], lse, s.loss_workspace(desc, True), dloss=c,
                            bias=o["bias"], x_scale=o["x_scale"], w_scale=o["w_scale"], **out)
        check(out, o, z, zerr, lse.double(), c, 0.0)


@pytest.mark.parametrize("M,N,K", [(2, 10, 64), (64, 1000, 2048), (700, 1500, 128)])
def test_captured(M, N, K):
    """Both ways to log p in one graph, replayed on other inputs between eager calls."""
    s = step()
    desc = s.loss_desc(M, N, K, dx_dtype="f32", dw_dtype="f32", ignore=IGNORE)
    held = make(M, N, K, "bf16", seed=5)
    loss, lse, logp, c = (torch.ones(M, device="cuda") for _ in range(4))
    outs = [{"dx": torch.empty(M, K, device="cuda"), "dw": torch.empty(N, K, device="cuda"),
             "dbias": torch.empty(N, device="cuda")} for _ in range(2)]
    wf, wb = s.loss_workspace(desc), s.loss_workspace(desc, True)

    def call():
        s.fqt_loss_forward(desc, held["x"], held["w"], held["target"], loss, lse, wf, bias=held["bias"], logp=logp)
        for out, given in zip(outs, (logp, None)):
            s.fqt_loss_backward(desc, held["x"], held["w"], held["target"], lse, wb, dloss=c, bias=held["bias"], logp=given,
                                **out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    every = [logp] + [t for out in outs for t in out.values()]
    for seed in (6, 7, 8):
        o = make(M, N, K, "bf16", seed=seed)
        for k in ("x", "w", "target", "bias"):
            held[k].copy_(o[k])
        call()
        want = [t.clone() for t in every]
        for t in every:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, every))
