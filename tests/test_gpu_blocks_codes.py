"""8-bit modules on inputs and weights that their codes hold exactly: nothing is left to the codes' own rounding, so a
wrong scale, row or column shows at once.

Every row is integers that the type holds, the largest code among them, times a power of two of its own; dy is
small integers.  All products are exact in float32 then, but for their sums' rounding: 1e-6 of the norm.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

CODES = {"int8": torch.arange(-127, 128).float(), "e4m3": torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()}


def exact(rows, cols, kind, seed):
    g = torch.Generator().manual_seed(seed)
    values = CODES[kind][torch.isfinite(CODES[kind])]
    t = values[torch.randint(len(values), (rows, cols), generator=g)]
    t[:, seed % cols] = values.max()
    return (t * torch.exp2(torch.randint(-6, 7, (rows, 1), generator=g).float())).cuda()


def rel(a, b):
    return (torch.linalg.vector_norm(a.detach().double() - b) / torch.linalg.vector_norm(b)).item()


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("M", [1, 3, 33, 130])
@pytest.mark.parametrize("fin,fout", [(48, 40), (515, 77)])
def test_linear(kind, M, fin, fout):
    from paper_2408_14267_amd import blocks as b
    mod = b.Linear(fin, fout, operands=kind).cuda()
    mod.weight.data.copy_(exact(fout, fin, kind, 1))
    mod.bias.data.copy_(exact(1, fout, kind, 2)[0])
    x = exact(M, fin, kind, 3).requires_grad_()
    dy = torch.randint(-8, 9, (M, fout), generator=torch.Generator().manual_seed(4)).float().cuda()
    y = mod(x)
    y.backward(dy)
    X, W, D = x.detach().double(), mod.weight.detach().double(), dy.double()
    assert rel(y, X @ W.t() + mod.bias.detach().double()) <= 1e-6
    assert rel(x.grad, D @ W) <= 1e-6
    assert rel(mod.weight.grad, D.t().contiguous() @ X) <= 1e-6
    assert rel(mod.bias.grad, D.sum(dim=0)) <= 1e-6


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_norm_linear(kind):
    """The norm's codes are its own; they are read back by a product with the unit matrix, whose codes and scales are
    exact, and must be within half a step of the norm in float64."""
    from paper_2408_14267_amd import blocks as b
    cols, top = 200, {"int8": 127.0, "e4m3": 448.0}[kind]
    mod = b.NormLinear(cols, cols, bias=False, operands=kind).cuda()
    mod.weight.data.copy_(torch.diag(torch.exp2(torch.arange(cols) % 7 - 3.0)))
    mod.norm_weight.data.copy_(1 + 0.3 * torch.randn(cols, generator=torch.Generator().manual_seed(1)).cuda())
    x = torch.randn(70, cols, generator=torch.Generator().manual_seed(2)).cuda() * torch.exp2(torch.arange(70) % 9 - 4.0).cuda()[:, None]
    got = mod(x).detach().double() / torch.diagonal(mod.weight.detach().double())
    X = x.double()
    want = X * (X.square().mean(dim=1, keepdim=True) + mod.eps).rsqrt() * mod.norm_weight.detach().double()
    scale = want.abs().amax(dim=1, keepdim=True) / top
    v = want / scale
    step = torch.ones_like(v) if kind == "int8" else torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    assert ((got - want).abs() <= (0.5 * step + 2e-5 * v.abs()) * scale).all()
