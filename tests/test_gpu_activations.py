"""gelu and silu of the linear epilogue over their whole range: a product over no columns is its bias, so the
bias is z exactly.

With u = 2^-24 and reciprocal and 2^x good to 2 u: gelu is max(z, 0) - a Phi(-a), a = |z|, whose second
term takes 14 u of itself from the quotient, the polynomial in it and the products, 2.1 a^2 u from the exponent of
exp(-a^2 / 2), and 1e-8 from the polynomial's fit; the last multiply-add adds u of the result.  In the tail the
fit's relative error stays below 2e-4 (bf16 outputs are rounded to 2^-8).  silu = z / (1 + exp(-z)) takes
8 u of itself where exp(-z) and its reciprocal are normal numbers.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def phi(z):
    """The normal distribution function to float64 in its tail too (1 + erf would lose it there)."""
    return 0.5 * torch.special.erfc(-z * 0.5 ** 0.5)


def dense():
    from paper_2408_14267_amd import dense as d
    return d


def activated(z, act, M, dtype):
    d = dense()
    bf = torch.bfloat16
    desc = d.linear_desc(M, z.numel(), 0, act=act, y_dtype=dtype)
    y = torch.empty(M, z.numel(), dtype=dtype, device="cuda")
    d.fqt_linear_forward(desc, torch.empty(M, 0, dtype=bf, device="cuda"),
                         torch.empty(z.numel(), 0, dtype=bf, device="cuda"), y, d.linear_workspace(desc), bias=z)
    assert torch.equal(y.nan_to_num(), y[:1].expand_as(y).nan_to_num())
    return y[0].double()


@pytest.mark.parametrize("M", [1, 8])
def test_gelu(M):
    z = torch.cat([torch.linspace(-12, 12, 240001), torch.linspace(-0.01, 0.01, 2001),
                   torch.tensor([-1e30, -40.0, 40.0, 1e30])]).cuda()
    y, a = activated(z, "gelu", M, torch.float32), z.double().abs()
    want, tail = z.double() * phi(z.double()), a * phi(-a)
    assert ((y - want).abs() <= (14 + 2.1 * a.clamp(max=20) ** 2) * U * tail + U * want.abs() + 1e-8).all()


@pytest.mark.parametrize("M", [1, 8])
def test_gelu_tail_in_bf16(M):
    z = torch.linspace(-8, -2, 60001).cuda()
    y = activated(z, "gelu", M, torch.bfloat16)
    want = z.double() * phi(z.double())
    assert ((y - want).abs() <= (2.0 ** -8 + 2e-4) * want.abs()).all()


@pytest.mark.parametrize("M", [1, 8])
def test_silu(M):
    z = torch.linspace(-85, 85, 170001).cuda()
    y = activated(z, "silu", M, torch.float32)
    want = z.double() * torch.sigmoid(z.double())
    assert ((y - want).abs() <= 8 * U * want.abs()).all()
    z = torch.tensor([-1e30, -200.0, 200.0, 1e30, float("inf"), float("nan")], device="cuda")
    y = activated(z, "silu", M, torch.float32)
    assert (y[:2] == 0).all() and torch.equal(y[2:5], z[2:5].double()) and torch.isnan(y[5])
