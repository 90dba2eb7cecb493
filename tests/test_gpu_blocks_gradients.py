"""Input gradients of the modules in the type of their input: a float32 stream's keep float32's bits.

Operands and dy are small integers, so the products below are exact, in more bits than bf16 has: nothing but a
rounding of the output can show.  The norm's backward is float32: 1e-6 of the norm.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def ints(*shape, seed, top):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-top, top + 1, shape, generator=g, device="cuda").float()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [2, 70])
def test_linear(dtype, M):
    from paper_2408_14267_amd import blocks as b
    mod = b.Linear(48, 200).cuda()
    mod.weight.data.copy_(ints(200, 48, seed=1, top=100))
    x = ints(M, 48, seed=2, top=3).to(dtype).requires_grad_()
    dy = ints(M, 200, seed=3, top=100).to(dtype)
    y = mod(x)
    assert y.dtype is dtype
    y.backward(dy)
    want = dy.double() @ mod.weight.double()
    assert x.grad.dtype is dtype and torch.equal(x.grad.double(), want.to(dtype).double())


@pytest.mark.parametrize("operands", ["bf16", "int8"])
@pytest.mark.parametrize("residual", [True, False])
def test_norm_linear(operands, residual):
    from paper_2408_14267_amd import blocks as b
    mod = b.NormLinear(48, 200, operands=operands).cuda()
    mod.weight.data.copy_(ints(200, 48, seed=1, top=100))
    mod.weight.data[:, 0] = 127                            # (the rows' scales are 1)
    x = ints(70, 48, seed=2, top=9).requires_grad_()
    dy = ints(70, 200, seed=3, top=100)
    if residual:
        y, h = mod(x, torch.zeros_like(x))
    else:
        y, h = mod(x), x
    y.backward(dy)
    H = h.detach().double()
    r = (H.square().mean(dim=1, keepdim=True) + mod.eps).rsqrt()
    u, t = (dy.double() @ mod.weight.double()) * mod.norm_weight.double(), H * r
    want = r * (u - t * (u * t).mean(dim=1, keepdim=True))
    assert torch.linalg.vector_norm(x.grad.double() - want) <= 1e-6 * torch.linalg.vector_norm(want)
