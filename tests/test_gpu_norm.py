"""RMS norm of a residual sum (forward, codes, backward) against the formulas in float64.

Tolerances, with u = 2^-24: a float32 sum of n terms in threads of at most 32 and trees of at most 11
levels is off by at most 43 u of the sum of magnitudes; rstd adds a division, a square root and its
operands (6 u), y two products.  60 u (3.6e-6) relative covers y, rstd and the scales; stored bf16 adds
half a unit in the last place of 8 bits, 2^-8.  dx is a difference, so its bound is 64 u of the magnitudes of its
terms; dg sums rows one after the other in `rows / parts` and `parts / 8` steps.  A code may be off its
real-valued quotient by half a step and 2e-5 of the quotient.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ROUND = {"f32": 0.0, "bf16": 2.0 ** -8}
TOP = {"int8": 127.0, "e4m3": 448.0}
EPS = 1e-5


def dense():
    from paper_2408_14267_amd import dense as d
    return d


def gen(*shape, seed=0, dt=torch.float32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + sum(shape))
    return (scale * torch.randn(shape, generator=g, device="cuda")).to(dt)


def guarded(rows, cols, dt, ld=None, offset=0):
    """A [rows][cols] view, stride ld, inside a buffer of sentinels; and a check that only the view was
    written."""
    ld = ld or cols
    n = offset + rows * ld + 64
    raw = torch.full((n,), 7, device="cuda").to(dt)
    view = raw[offset:offset + rows * ld].view(rows, ld)[:, :cols] if rows and cols else raw[:0].view(rows, cols)

    def intact():
        keep = torch.ones(n, dtype=torch.bool, device="cuda")
        if rows and cols:
            keep[offset:offset + rows * ld].view(rows, ld)[:, :cols] = False
        assert (raw[keep].float() == 7).all()
    return view, intact


def close(got, want, rel, absolute=0.0, what=""):
    err = (got.double() - want).abs()
    lim = rel * want.abs() + absolute
    assert torch.isfinite(got.double()).all(), what
    assert (err <= lim).all(), f"{what}: off by {(err / lim.clamp_min(1e-300)).max().item():.3g} of the bound"


SHAPES = [(1, 1), (1, 4096), (3, 8), (5, 513), (2, 512), (7, 1000), (257, 1024), (33, 1153),
          (4, 2048), (9, 2049), (130, 4096), (3, 4097), (2, 8192), (3, 8193), (2, 16384), (2, 16392),
          (2, 25088), (300, 25088), (2100, 64), (3, 32768), (3, 32775), (70, 40000)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("xt,yt,qt", [("bf16", "bf16", "e4m3"), ("f32", "f32", "int8"),
                                      ("bf16", "f32", "int8"), ("f32", "bf16", "e4m3")])
def test_forward(rows, cols, xt, yt, qt):
    d = dense()
    x, r = gen(rows, cols, seed=1, dt=DT[xt]), gen(rows, cols, seed=2, dt=DT[xt], scale=3.0)
    g = 1.0 + 0.3 * gen(cols, seed=3)
    h, h_ok = guarded(rows, cols, DT[xt])
    y, y_ok = guarded(rows, cols, DT[yt])
    q = torch.zeros(rows, cols, device="cuda").to(d._TORCH_OF[d.dtype_code(qt)])
    scale, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    desc = d.norm_desc(rows, cols, x_dtype=xt, y_dtype=yt, q_dtype=qt, eps=EPS)
    d.fqt_rmsnorm_forward(desc, x, g, residual=r, h=h, y=y, q=q, scale=scale, rstd=rstd)
    h_ok(), y_ok()
    assert torch.equal(h, (x.float() + r.float()).to(DT[xt]))
    h64 = (x.float() + r.float()).double()              # (the float32 sum is the definition)
    r64 = (h64.square().mean(dim=1) + EPS).rsqrt()
    y64 = h64 * r64[:, None] * g.double()
    close(rstd, r64, 60 * U, what="rstd")
    close(y, y64, 60 * U + ROUND[yt], what="y")
    s64 = y64.abs().amax(dim=1) / TOP[qt]
    close(scale, s64, 60 * U, what="scale")
    v = y64 / s64[:, None]
    got = q.to(torch.float32).double()
    if qt == "int8":
        step = torch.ones_like(v)
    else:                                               # 3 mantissa bits, subnormals from 2^-6 down
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    close(got, v, 2e-5, 0.5 * step, what="codes")
    assert got.abs().amax() <= TOP[qt]
    # the same call again gives the same bits
    y2, q2 = torch.empty_like(y), torch.empty_like(q)
    d.fqt_rmsnorm_forward(desc, x, g, residual=r, h=h, y=y2, q=q2, scale=scale, rstd=rstd)
    assert torch.equal(y2, y) and torch.equal(q2.view(torch.uint8), q.view(torch.uint8))


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("xt,yt,residual", [("bf16", "bf16", True), ("f32", "f32", False),
                                            ("f32", "bf16", True), ("bf16", "f32", False)])
def test_backward(rows, cols, xt, yt, residual):
    d = dense()
    h, dy = gen(rows, cols, seed=4, dt=DT[xt]), gen(rows, cols, seed=5, dt=DT[yt])
    dres = gen(rows, cols, seed=6, dt=DT[xt]) if residual else None
    g = 1.0 + 0.3 * gen(cols, seed=3)
    rstd = (h.float().square().mean(dim=1) + EPS).rsqrt()
    dx, dx_ok = guarded(rows, cols, DT[xt])
    dg = torch.empty(cols, device="cuda")
    desc = d.norm_desc(rows, cols, x_dtype=xt, y_dtype=yt, eps=EPS)
    ws = d.norm_workspace(desc).fill_(0xFF)
    d.fqt_rmsnorm_backward(desc, h, g, rstd, dy, dx, dg, ws, dres=dres)
    dx_ok()
    r64 = rstd.double()[:, None]
    t, u = h.double() * r64, dy.double() * g.double()
    m = (u * t).mean(dim=1, keepdim=True)
    want = r64 * (u - t * m)
    size = r64 * (u.abs() + t.abs() * (u * t).abs().mean(dim=1, keepdim=True))
    if residual:
        want, size = want + dres.double(), size + dres.double().abs()
    close(dx, want, ROUND[xt], 64 * U * size, what="dx")
    depth = rows / 64 + 64 + 16
    close(dg, (dy.double() * t).sum(dim=0), 0.0, depth * U * (dy.double() * t).abs().sum(dim=0) + 1e-30,
          what="dg")
    again = torch.empty_like(dg)
    d.fqt_rmsnorm_backward(desc, h, g, rstd, dy, dx, again, ws, dres=dres)
    assert torch.equal(again, dg)


def test_backward_against_differences():
    """<dx, v> and <dg, v> against central differences of sum(y dy) in float64."""
    d = dense()
    rows, cols = 6, 40
    x, dy, g = gen(rows, cols, seed=1), gen(rows, cols, seed=2), 1.0 + 0.3 * gen(cols, seed=3)
    desc = d.norm_desc(rows, cols, x_dtype="f32", eps=EPS)
    rstd, dx, dg = torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty_like(g)
    y = torch.empty_like(x)
    d.fqt_rmsnorm_forward(desc, x, g, y=y, rstd=rstd)
    d.fqt_rmsnorm_backward(desc, x, g, rstd, dy, dx, dg, d.norm_workspace(desc))

    def f(a, b):
        return (a * (a.square().mean(dim=1, keepdim=True) + EPS).rsqrt() * b * dy.double()).sum()

    e = 1e-5
    for seed in range(3):
        v, w = gen(rows, cols, seed=10 + seed).double(), gen(cols, seed=20 + seed).double()
        num = (f(x.double() + e * v, g.double()) - f(x.double() - e * v, g.double())) / (2 * e)
        assert abs((dx.double() * v).sum() - num) <= 1e-5 * (dx.double() * v).abs().sum()
        num = (f(x.double(), g.double() + e * w) - f(x.double(), g.double() - e * w)) / (2 * e)
        assert abs((dg.double() * w).sum() - num) <= 1e-5 * (dg.double() * w).abs().sum()


@pytest.mark.parametrize("xt", ["bf16", "f32"])
@pytest.mark.parametrize("cols,ld,offset", [(100, 104, 0), (100, 131, 3), (1024, 1032, 8), (4096, 4099, 1),
                                            (17000, 17001, 1)])
def test_strides_and_offsets(xt, cols, ld, offset):
    """Rows apart by more than their length, at any element offset, equal the dense call bit for bit where
    both take the same path and to rounding where they do not."""
    d = dense()
    rows = 5
    base = gen(rows, cols, seed=1, dt=DT[xt])
    g = 1.0 + 0.3 * gen(cols, seed=3)
    views, checks = zip(*(guarded(rows, cols, DT[xt], ld, offset) for _ in range(4)))
    x, r, h, y = views
    x.copy_(base), r.copy_(base)
    q, q_ok = guarded(rows, cols, torch.int8, ld, offset)
    scale, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    desc = d.norm_desc(rows, cols, x_dtype=xt, q_dtype="int8", ldx=ld, ldr=ld, ldh=ld, ldy=ld, ldq=ld)
    d.fqt_rmsnorm_forward(desc, x, g, residual=r, h=h, y=y, q=q, scale=scale, rstd=rstd)
    q_ok(), checks[2](), checks[3]()
    D = d.norm_desc(rows, cols, x_dtype=xt, q_dtype="int8")
    y0, q0, s0, r0 = torch.empty_like(base), torch.empty(rows, cols, dtype=torch.int8, device="cuda"), \
        torch.empty_like(scale), torch.empty_like(rstd)
    d.fqt_rmsnorm_forward(D, base, g, residual=base, y=y0, q=q0, scale=s0, rstd=r0)
    close(y, y0.double(), 120 * U + 2 * ROUND[xt], what="y")
    close(rstd, r0.double(), 120 * U, what="rstd")
    assert (q.int() - q0.int()).abs().max() <= 1
    dx, dx_ok = guarded(rows, cols, DT[xt], ld, offset)
    dg, dg0, dx0 = torch.empty_like(g), torch.empty_like(g), torch.empty_like(base)
    d.fqt_rmsnorm_backward(desc, x, g, r0, r, dx, dg, d.norm_workspace(desc), dres=h)
    dx_ok()
    d.fqt_rmsnorm_backward(D, base, g, r0, base, dx0, dg0, d.norm_workspace(D), dres=h.contiguous())
    close(dg, dg0.double(), 0.0, 60 * U * (base.double().square() * r0.double()[:, None]).sum(dim=0) * 2, what="dg")
    close(dx, dx0.double(), 2 * ROUND[xt], 200 * U * (dx0.double().abs().amax() + 1), what="dx")


@pytest.mark.parametrize("cols", [1000, 4096, 20000])
def test_in_place_residual_stream(cols):
    """h may be x or the residual, dx may be dres."""
    d = dense()
    rows, g = 70, 1.0 + 0.3 * gen(cols, seed=3)
    x, r = gen(rows, cols, seed=1, dt=torch.bfloat16), gen(rows, cols, seed=2, dt=torch.bfloat16)
    desc = d.norm_desc(rows, cols)
    want_h, want_y = torch.empty_like(x), torch.empty_like(x)
    d.fqt_rmsnorm_forward(desc, x, g, residual=r, h=want_h, y=want_y)
    for which in (0, 1):
        a, b, y = x.clone(), r.clone(), torch.empty_like(x)
        d.fqt_rmsnorm_forward(desc, a, g, residual=b, h=(a, b)[which], y=y)
        assert torch.equal((a, b)[which], want_h) and torch.equal(y, want_y)
    rstd, dg, dg2, dx = torch.ones(rows, device="cuda"), torch.empty_like(g), torch.empty_like(g), torch.empty_like(x)
    ws = d.norm_workspace(desc)
    d.fqt_rmsnorm_backward(desc, x, g, rstd, r, dx, dg, ws, dres=want_h)
    again = want_h.clone()
    d.fqt_rmsnorm_backward(desc, x, g, rstd, r, again, dg2, ws, dres=again)
    assert torch.equal(again, dx) and torch.equal(dg, dg2)


@pytest.mark.parametrize("qt", ["int8", "e4m3"])
def test_rows_of_zeros_extremes_and_non_finite_values(qt):
    """A row of zeros has scale 0 and codes 0; tiny and large rows keep their codes; a row with an infinity
    or a NaN has a scale that is not finite, and the rows beside it are untouched."""
    d = dense()
    cols = 300
    x = gen(8, cols, seed=1)
    x[1] = 0
    x[2] *= 1e-18
    x[3] *= 1e18
    x[5, 7], x[6, 9] = float("inf"), float("nan")
    q = torch.empty(8, cols, device="cuda").to(d._TORCH_OF[d.dtype_code(qt)])
    scale, rstd, y = torch.empty(8, device="cuda"), torch.empty(8, device="cuda"), torch.empty_like(x)
    desc = d.norm_desc(8, cols, x_dtype="f32", q_dtype=qt, eps=1e-30)
    d.fqt_rmsnorm_forward(desc, x, torch.ones(cols, device="cuda"), y=y, q=q, scale=scale, rstd=rstd)
    assert scale[1] == 0 and (q[1].float() == 0).all() and (y[1] == 0).all()
    ok = [0, 2, 3, 4, 7]
    want = x[ok].double() * (x[ok].double().square().mean(dim=1, keepdim=True) + 1e-30).rsqrt()
    close(y[ok], want, 60 * U, what="y")
    assert (q[ok].float().abs().amax(dim=1) == TOP[qt]).all()
    assert not torch.isfinite(scale[[5, 6]]).any()
    # the row quantiser on the same rows, and on rows near the smallest and the largest float32
    x[2] *= 1e-20
    x[3] *= 1e19
    d.fqt_quantize_rows(desc, x, q, scale)
    assert scale[1] == 0 and (q[1].float() == 0).all()
    back = q[ok].float().double() * scale[ok].double()[:, None]
    top = x[ok].double().abs().amax(dim=1, keepdim=True)
    assert ((back - x[ok].double()).abs() <= top * (0.5 / 127 if qt == "int8" else 2.0 ** -4) * 1.001).all()
    assert not torch.isfinite(scale[[5, 6]]).any()


@pytest.mark.parametrize("rows,cols", [(0, 16), (16, 0), (0, 0)])
def test_empty(rows, cols):
    d = dense()
    desc = d.norm_desc(rows, cols, q_dtype="int8")
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    g, dg, v = torch.ones(cols, device="cuda"), torch.full((cols,), 3.0, device="cuda"), torch.empty(rows, device="cuda")
    d.fqt_rmsnorm_forward(desc, x, g, y=x.clone(), rstd=v)
    d.fqt_quantize_rows(desc, x, torch.empty(rows, cols, dtype=torch.int8, device="cuda"), v)
    d.fqt_rmsnorm_backward(desc, x, g, v, x, x.clone(), dg, d.norm_workspace(desc))
    assert (dg == 0).all()                              # a sum over no rows


def test_offsets_beyond_31_bits():
    """Rows whose element offsets pass 2^31: 520 rows 2^22 elements apart."""
    d = dense()
    rows, cols, ld = 520, 96, 1 << 22
    buf = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    x = buf.view(rows, ld)[:, :cols]
    x.copy_(gen(rows, cols, seed=1))
    y = buf.view(rows, ld)[:, 128:128 + cols]
    g = torch.ones(cols, device="cuda")
    d.fqt_rmsnorm_forward(d.norm_desc(rows, cols, ldx=ld, ldy=ld), x, g, y=y)
    want = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    d.fqt_rmsnorm_forward(d.norm_desc(rows, cols), x.contiguous(), g, y=want)
    assert torch.equal(y, want)


def test_own_stream_and_captured_replays():
    d = dense()
    rows, cols = 300, 1024
    x, g = gen(rows, cols, seed=1, dt=torch.bfloat16), 1.0 + 0.3 * gen(cols, seed=3)
    desc = d.norm_desc(rows, cols, q_dtype="e4m3")
    ws = d.norm_workspace(desc)
    h, y, dx = (torch.empty_like(x) for _ in range(3))
    q = torch.empty(rows, cols, device="cuda").to(torch.float8_e4m3fn)
    scale, rstd, dg = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")

    def step():
        d.fqt_rmsnorm_forward(desc, x, g, residual=x, h=h, y=y, q=q, scale=scale, rstd=rstd)
        d.fqt_rmsnorm_backward(desc, h, g, rstd, y, dx, dg, ws, dres=x)

    def outputs():
        return [t.clone() for t in (h, y, q.view(torch.uint8), scale, rstd, dx, dg)]

    step()
    torch.cuda.synchronize()
    want = outputs()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(outputs(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for t in (h, y, scale, rstd, dx, dg):
            t.fill_(float(i))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), want)), i
        step()                                           # the program's own eager work between replays
    x.copy_(gen(rows, cols, seed=9, dt=torch.bfloat16))  # new inputs reach a replay
    graph.replay()
    got = outputs()
    step()
    assert all(torch.equal(a, b) for a, b in zip(got, outputs()))
    assert math.isfinite(dg.sum().item())
