"""Orthogonalisation over many steps of gradients that are small beside eps, against the iteration in
float64.

While |X_i| is below 1/4 the iteration is X <- a X up to terms of |X|^3, every direction keeps its share, and
a step leaves what its roundings leave: an entry's two float16 parts 2^-22, the float32 sums and the
multiply-add 2^-23, together at most 5e-7 of the norm.  `end` steps of a before 1, that is 5e-7 steps; where
the last two steps go past it (a Frobenius norm of a^2 at most, singular values about 1), what was there
before may grow by a^2 = 12 beside the strongest directions.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315
EPS = 2.0 ** -23                       # (exact in float32)


def dense():
    from paper_2408_14267_amd import dense as d
    return d


def gen(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + sum(shape))
    return torch.randn(shape, generator=g, device="cuda")


def ns64(u, steps):
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = (x.t() if tall else x).contiguous()
    x = x / (torch.linalg.vector_norm(x) + EPS)
    for _ in range(steps):
        p = torch.mm(x, x.t().contiguous())
        x = A * x + torch.mm(B * p + C * torch.mm(p, p), x)
    return x.t().contiguous() if tall else x


def off(got, want):
    assert torch.isfinite(got.double()).all()
    return (torch.linalg.vector_norm(got.double() - want) / torch.linalg.vector_norm(want)).item()


@pytest.mark.parametrize("rows,cols", [(48, 200), (333, 40), (300, 420), (420, 130)])
@pytest.mark.parametrize("steps", [5, 10, 16, 32])
@pytest.mark.parametrize("end", [2, -2])
def test_small_gradients(rows, cols, steps, end):
    """|u| = eps a^-(steps + end): |X| ends at a^-end, or would."""
    d = dense()
    g = gen(rows, cols, seed=1)
    g *= EPS * A ** -(steps + end) / torch.linalg.vector_norm(g)
    o = torch.empty(rows, cols, device="cuda")
    desc = d.ortho_desc(rows, cols, steps=steps, eps=EPS)
    d.fqt_orthogonalize(desc, g, o, d.ortho_workspace(desc).fill_(0xFF))
    assert off(o, ns64(g, steps)) <= 5e-7 * steps * (A ** 2 if end < 0 else 1.0)


@pytest.mark.parametrize("rows,cols", [(48, 200), (300, 420)])
def test_momentum_that_starts_small(rows, cols):
    """The optimizer step over many iterations takes the same path; the first gradients of a run are tiny."""
    d = dense()
    steps, lr = 16, 0.5
    g = gen(rows, cols, seed=2) * (EPS * A ** -(steps + 2) / (rows * cols) ** 0.5)
    w, m = torch.zeros(rows, cols, device="cuda"), torch.zeros(rows, cols, device="cuda")
    desc = d.ortho_desc(rows, cols, steps=steps, eps=EPS)
    d.fqt_muon_step(desc, w, g, m, d.ortho_workspace(desc), lr=lr, momentum=0.0, nesterov=False)
    assert off(w, -lr * ns64(g, steps)) <= 5e-7 * (steps + 1)


@pytest.mark.parametrize("rows,cols,ld,offset", [(40, 100, 107, 3), (200, 130, 133, 1), (100, 40, 41, 2)])
def test_strides_do_not_change_a_bit(rows, cols, ld, offset):
    """The order of every sum depends on the sizes alone."""
    d = dense()

    def view(v):
        t = torch.zeros(offset + rows * ld, device="cuda")[offset:].view(rows, ld)[:, :cols]
        return t.copy_(v)

    g, m, w = gen(rows, cols, seed=1), gen(rows, cols, seed=2), gen(rows, cols, seed=3)
    gv, mv, wv = view(g), view(m), view(w)
    desc, D = d.ortho_desc(rows, cols, ldg=ld, ldm=ld, ldo=ld), d.ortho_desc(rows, cols)
    d.fqt_muon_step(desc, wv, gv, mv, d.ortho_workspace(desc), lr=0.1)
    d.fqt_muon_step(D, w, g, m, d.ortho_workspace(D), lr=0.1)
    assert torch.equal(mv, m) and torch.equal(wv, w)
