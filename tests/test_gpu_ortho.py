"""Newton-Schulz orthogonalisation and the optimizer step on it against the iteration in float64.

Tolerances: an operand's two float16 parts and the float32 sums leave each product a relative error of a
few 2^-23 of its norm, and a step multiplies what the steps before it left by at most a = 3.4445, the
slope of the quintic at 0.  Over five steps that is at most 485 times a few 2^-23; the bound is 1.2e-4 of
the result's norm (errors of one direction only; whole results are off by 1e-6 to 3e-6).  Stored bf16
adds 2^-8 of an entry.  m is one float32 multiply-add; w two.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
BOUND = {"f32": 1.2e-4, "bf16": 1.2e-4 + 2.0 ** -8}


def dense():
    from paper_2408_14267_amd import dense as d
    return d


def gen(*shape, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + sum(shape))
    return scale * torch.randn(shape, generator=g, device="cuda")


def ns64(u, steps=5, eps=1e-7):
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = (x.t() if tall else x).contiguous()
    x = x / (torch.linalg.vector_norm(x) + eps)
    for _ in range(steps):
        p = torch.mm(x, x.t().contiguous())
        x = A * x + torch.mm(B * p + C * torch.mm(p, p), x)
    return x.t().contiguous() if tall else x


def off(got, want):
    assert torch.isfinite(got.double()).all()
    n = torch.linalg.vector_norm(want).item()
    return torch.linalg.vector_norm(got.double() - want).item() / (n or 1.0)


SHAPES = [(1, 1), (1, 300), (300, 1), (10, 27), (64, 64), (64, 576), (576, 64), (33, 4097), (64, 25088),
          (65, 65), (65, 100), (128, 1152), (1000, 513), (512, 4608), (4608, 512), (700, 1999), (2304, 2304)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_orthogonalize(rows, cols, dt):
    d = dense()
    r = min(8, rows, cols)
    g = (gen(rows, r, seed=1) @ gen(r, cols, seed=2) + 0.3 * gen(rows, cols, seed=3)).to(DT[dt])
    raw = torch.full((rows * cols + 64,), 7.0, device="cuda").to(DT[dt])
    o = raw[:rows * cols].view(rows, cols)
    desc = d.ortho_desc(rows, cols, g_dtype=dt, o_dtype=dt)
    ws = d.ortho_workspace(desc).fill_(0xFF)
    d.fqt_orthogonalize(desc, g, o, ws)
    assert (raw[rows * cols:].float() == 7).all()
    assert off(o, ns64(g)) <= BOUND[dt]
    again = torch.empty_like(o)
    d.fqt_orthogonalize(desc, g, again, ws)
    assert torch.equal(again, o)
    d.fqt_orthogonalize(desc, g, g, ws)                  # in place
    assert torch.equal(g, o)


@pytest.mark.parametrize("rows,cols,mixed", [(64, 576, ("f32", "bf16")), (300, 200, ("bf16", "f32")), (40, 30, ("bf16", "f32"))])
def test_types_differ(rows, cols, mixed):
    d = dense()
    g = gen(rows, cols, seed=1).to(DT[mixed[0]])
    o = torch.empty(rows, cols, dtype=DT[mixed[1]], device="cuda")
    desc = d.ortho_desc(rows, cols, g_dtype=mixed[0], o_dtype=mixed[1])
    d.fqt_orthogonalize(desc, g, o, d.ortho_workspace(desc))
    assert off(o, ns64(g)) <= BOUND[mixed[1]]


@pytest.mark.parametrize("rows,cols", [(48, 200), (300, 420)])
@pytest.mark.parametrize("steps", [1, 2, 9])
def test_steps(rows, cols, steps):
    d = dense()
    g, o = gen(rows, cols, seed=1), torch.empty(rows, cols, device="cuda")
    desc = d.ortho_desc(rows, cols, steps=steps)
    d.fqt_orthogonalize(desc, g, o, d.ortho_workspace(desc))
    # (the quintic does not settle: directions near its fixed point move apart by up to 2 a step)
    assert off(o, ns64(g, steps)) <= BOUND["f32"] * max(1, 2 ** (steps - 5))


@pytest.mark.parametrize("rows,cols", [(64, 576), (50, 50), (200, 333), (700, 130)])
def test_singular_values_come_near_one(rows, cols):
    d = dense()
    g, o = gen(rows, cols, seed=4), torch.empty(rows, cols, device="cuda")
    desc = d.ortho_desc(rows, cols)
    d.fqt_orthogonalize(desc, g, o, d.ortho_workspace(desc))
    s = torch.linalg.svdvals(o.cpu().double())
    s0 = torch.linalg.svdvals((g / torch.linalg.vector_norm(g)).cpu().double())
    assert s.max() < 1.21 and s[s0 > 0.01].min() > 0.6


@pytest.mark.parametrize("rows,cols", [(40, 100), (130, 100)])
@pytest.mark.parametrize("scale", [1e-30, 1e-16, 3e-12, 1.2e-11, 2.5e-11, 1e-10, 1e-9, 1e-3, 1e25])
def test_scale_of_the_gradient(rows, cols, scale):
    """|u| is summed in float64: entries whose squares leave float32 give the same result.  eps is
    1e-7, so the smallest ones are damped by it, as the formula says."""
    d = dense()
    g, o = gen(rows, cols, seed=1) * scale, torch.empty(rows, cols, device="cuda")
    desc = d.ortho_desc(rows, cols)
    d.fqt_orthogonalize(desc, g, o, d.ortho_workspace(desc))
    assert off(o, ns64(g)) <= BOUND["f32"]


@pytest.mark.parametrize("rows,cols", [(40, 100), (100, 40), (130, 300)])
def test_zero_and_low_rank(rows, cols):
    d = dense()
    desc = d.ortho_desc(rows, cols)
    ws, o = d.ortho_workspace(desc), torch.empty(rows, cols, device="cuda")
    d.fqt_orthogonalize(desc, torch.zeros(rows, cols, device="cuda"), o, ws)
    assert (o == 0).all()
    g = gen(rows, 1, seed=1) @ gen(1, cols, seed=2)      # rank one, rows and columns of zeros in it
    g[3], g[:, 5] = 0, 0
    d.fqt_orthogonalize(desc, g, o, ws)
    assert off(o, ns64(g)) <= BOUND["f32"]
    g[0, 0] = float("nan")
    d.fqt_orthogonalize(desc, g, o, ws)
    assert not torch.isfinite(o).all()                   # not hidden
    d.fqt_orthogonalize(desc, torch.zeros(rows, cols, device="cuda"), o, ws)
    assert (o == 0).all()                                # and not kept


@pytest.mark.parametrize("rows,cols", [(1, 5), (64, 576), (60, 33), (512, 4608), (300, 200)])
@pytest.mark.parametrize("gt,nesterov", [("f32", True), ("bf16", False)])
def test_muon_step(rows, cols, gt, nesterov):
    d = dense()
    lr, mu, wd, scale = 0.3, 0.9, 0.05, 1.7
    w, m = gen(rows, cols, seed=1), gen(rows, cols, seed=2, scale=1e-2)
    w64, m64 = w.double(), m.double()
    desc = d.ortho_desc(rows, cols, g_dtype=gt)
    ws = d.ortho_workspace(desc).fill_(0xFF)
    for step in range(3):
        g = gen(rows, cols, seed=3 + step, scale=1e-2).to(DT[gt])
        d.fqt_muon_step(desc, w, g, m, ws, lr=lr, momentum=mu, weight_decay=wd, scale=scale, nesterov=nesterov)
        m64 = mu * m64 + g.double()
        u = g.double() + mu * m64 if nesterov else m64
        w64 = (1 - lr * wd) * w64 - lr * scale * ns64(u)
        assert ((m.double() - m64).abs() <= 3e-7 * (step + 1) * (m64.abs() + g.double().abs() + 1e-2)).all()
        assert off(w, w64) <= BOUND["f32"] * (step + 1)


@pytest.mark.parametrize("rows,cols,ld,offset", [(40, 100, 104, 0), (40, 100, 107, 3), (200, 130, 133, 1)])
def test_strides(rows, cols, ld, offset):
    d = dense()

    def view(v):
        raw = torch.full((offset + rows * ld + 64,), 7.0, device="cuda")
        t = raw[offset:offset + rows * ld].view(rows, ld)[:, :cols]
        t.copy_(v)
        return raw, t

    g, m, w = gen(rows, cols, seed=1), gen(rows, cols, seed=2), gen(rows, cols, seed=3)
    (_, gv), (mr, mv), (wr, wv) = view(g), view(m), view(w)
    desc = d.ortho_desc(rows, cols, ldg=ld, ldm=ld, ldo=ld)
    d.fqt_muon_step(desc, wv, gv, mv, d.ortho_workspace(desc), lr=0.1)
    D = d.ortho_desc(rows, cols)
    d.fqt_muon_step(D, w, g, m, d.ortho_workspace(D), lr=0.1)
    assert torch.equal(mv, m)
    assert off(wv, w.double()) <= 1e-6                   # (the norm's partial sums differ)
    for raw in (mr, wr):
        keep = torch.ones_like(raw, dtype=torch.bool)
        keep[offset:offset + rows * ld].view(rows, ld)[:, :cols] = False
        assert (raw[keep] == 7).all()


@pytest.mark.parametrize("rows,cols", [(0, 5), (5, 0), (0, 0)])
def test_empty(rows, cols):
    d = dense()
    desc = d.ortho_desc(rows, cols)
    t = torch.empty(rows, cols, device="cuda")
    d.fqt_orthogonalize(desc, t, t, d.ortho_workspace(desc))
    d.fqt_muon_step(desc, t, t, t, d.ortho_workspace(desc), lr=0.1)


@pytest.mark.parametrize("rows,cols", [(64, 576), (256, 300)])
def test_own_stream_and_captured_replays(rows, cols):
    d = dense()
    g, o = gen(rows, cols, seed=1), torch.empty(rows, cols, device="cuda")
    desc = d.ortho_desc(rows, cols)
    ws = d.ortho_workspace(desc)

    def step():
        d.fqt_orthogonalize(desc, g, o, ws)

    step()
    want = o.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(o, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        o.fill_(float(i))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want), i
        step()
