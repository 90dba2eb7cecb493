"""Products of codes whose two scales multiply to nothing or to infinity, though the result is ordinary."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def dense():
    from paper_2408_14267_amd import dense as d
    return d


@pytest.mark.parametrize("M,N,K", [(1, 33, 16384), (4, 2600, 16384), (40, 33, 16384), (70, 300, 16384)])
@pytest.mark.parametrize("xt", ["int8", "e4m3"])
def test_scales_far_from_one(M, N, K, xt):
    """Codes of 32 and 64: the sums are 2^10 times integers of 17 bits, from 2^24 on, and every product below is
    exact.  2^-80 times 2^-70 would be 0, 2^-75 times 1.5 2^-74 rounded, 2^70 times 2^70 infinite (and
    that times a sum of 0 NaN)."""
    d = dense()
    g = torch.Generator(device="cuda").manual_seed(M)
    code = torch.int8 if xt == "int8" else torch.float8_e4m3fn
    x = 32.0 * torch.randint(1, 3, (M, K), generator=g, device="cuda")
    w = 32.0 * torch.randint(1, 3, (N, K), generator=g, device="cuda")
    w[0] = 0
    desc = d.linear_desc(M, N, K, x_dtype=xt, y_dtype="f32")
    y, ws = torch.empty(M, N, device="cuda"), d.linear_workspace(desc)
    a, b, base = x.to(code), w.to(code), (x.double() @ w.double().t()).float()

    def product(sx, sw):
        d.fqt_linear_forward(desc, a, b, y, ws, x_scale=torch.full((M,), sx, device="cuda"),
                             w_scale=torch.full((N,), sw, device="cuda"))
        return y.double()

    assert torch.equal(product(1.0, 1.0), base.double())
    assert torch.equal(product(2.0 ** -80, 2.0 ** -70), base.double() * 2.0 ** -150)
    assert torch.equal(product(2.0 ** -75, 1.5 * 2.0 ** -74), base.double() * 1.5 * 2.0 ** -149)
    far = product(2.0 ** 70, 2.0 ** 70)
    assert (far[:, 0] == 0).all() and torch.isinf(far[:, 1:]).all()
