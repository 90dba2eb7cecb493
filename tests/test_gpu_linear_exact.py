"""int8 products whose contraction is split over workgroups: the sums are exact in int32 and rounded once."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def dense():
    from paper_2408_14267_amd import dense as d
    return d


@pytest.mark.parametrize("M,N,K", [(1, 40, 25088), (5, 10, 25088), (64, 1000, 25088), (100, 70, 25090),
                                   (512, 512, 25088), (16, 16, 133144)])
def test_int8_sums_are_exact(M, N, K):
    """Large codes whose products cancel: partial sums beyond 2^24, where float32 has no odd numbers, and sums
    that need every bit of them."""
    d = dense()
    gen = torch.Generator(device="cuda").manual_seed(K)
    x = torch.randint(100, 128, (M, K), generator=gen, device="cuda")
    w = torch.randint(100, 128, (N, K), generator=gen, device="cuda")
    w[:, K // 2:] *= -1
    w[::3] = -w[::3].flip(1)
    w[1::5] = w[1::5].abs()                                # these add up to 13000 K
    want = (x.double() @ w.double().t()).float()           # exact before its one rounding
    desc = d.linear_desc(M, N, K, x_dtype="int8", y_dtype="f32")
    y, ws = torch.empty(M, N, device="cuda"), d.linear_workspace(desc).fill_(0xFF)
    d.fqt_linear_forward(desc, x.to(torch.int8), w.to(torch.int8), y, ws, x_scale=torch.ones(M, device="cuda"),
                         w_scale=torch.ones(N, device="cuda"))
    assert torch.equal(y, want)
