"""Modules at the ends of their ranges: no rows, one row, single vectors, more dimensions, no blocks, weights that are
views."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def gen(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + sum(shape))
    return torch.randn(shape, generator=g, device="cuda")


def modules():
    from paper_2408_14267_amd import blocks as b
    torch.manual_seed(0)
    return [b.RMSNorm(40).cuda(), b.Linear(40, 24, act="gelu").cuda(), b.Linear(40, 24, operands="int8").cuda(),
            b.NormLinear(40, 24, operands="e4m3").cuda(), b.NormLinear(40, 24, operands="bf16").cuda()]


@pytest.mark.parametrize("which", range(5))
@pytest.mark.parametrize("shape", [(0, 40), (3, 0, 40), (1, 40), (40,), (2, 3, 5, 40)])
def test_shapes(which, shape):
    """The rows of any shape are those of the flat call; gradients over no rows are zero."""
    mod = modules()[which]
    x = gen(*shape, seed=1).requires_grad_()
    flat = x.detach().reshape(-1, 40).clone().requires_grad_()
    y, z = mod(x), mod(flat)
    assert y.shape[:-1] == x.shape[:-1] and torch.equal(y.reshape(z.shape), z)
    got = torch.autograd.grad(y.sum(), [x, *mod.parameters()])
    want = torch.autograd.grad(z.sum(), [flat, *mod.parameters()])
    assert torch.equal(got[0].reshape(want[0].shape), want[0])
    assert all(torch.equal(a, b) for a, b in zip(got[1:], want[1:]))
    if x.numel() == 0:
        assert all((g == 0).all() for g in got)


@pytest.mark.parametrize("operands", ["bf16", "int8"])
def test_weight_that_is_a_view(operands):
    from paper_2408_14267_amd import blocks as b
    mod, twin = b.Linear(40, 24, operands=operands).cuda(), b.Linear(40, 24, operands=operands).cuda()
    table = gen(40, 30, seed=1)
    mod.weight = torch.nn.Parameter(table.t()[:24])
    twin.weight.data.copy_(mod.weight)
    x, dy = gen(9, 40, seed=2), gen(9, 24, seed=3)
    for m in (mod, twin):
        m(x).backward(dy)
    assert torch.equal(mod(x), twin(x)) and torch.equal(mod.weight.grad, twin.weight.grad)


@pytest.mark.parametrize("depth", [0, 1, 2])
def test_residual_network_of_any_depth(depth):
    from paper_2408_14267_amd import blocks as b
    net = b.ResidualMLP(20, 5, width=32, hidden=64, depth=depth).cuda()
    x = gen(16, 20, seed=1)
    y = net(x)
    y.square().mean().backward()
    assert y.shape == (16, 5) and all(torch.isfinite(p.grad).all() for p in net.parameters())
    if depth == 0:
        assert torch.equal(y, net.head(net.norm(net.stem(x))))
