"""A step that cannot be taken whole is not taken in part."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("spoil", ["lr", "momentum", "steps", "sparse", "host"])
def test_nothing_is_updated(spoil):
    from paper_2408_14267_amd import blocks as b
    ps = [torch.nn.Parameter(torch.randn(8, 16, device="cuda" if i == 0 or spoil != "host" else "cpu")) for i in range(2)]
    opt = b.Muon([dict(params=ps[:1]), dict(params=ps[1:])])
    for p in ps:
        p.grad = torch.ones_like(p)
    if spoil == "sparse":
        ps[1].grad = torch.zeros_like(ps[1]).to_sparse()
    elif spoil != "host":
        opt.param_groups[1][spoil] = {"lr": float("nan"), "momentum": 1.5, "steps": 40}[spoil]
    before = [p.detach().clone() for p in ps]
    with pytest.raises((ValueError, RuntimeError)):
        opt.step()
    assert all(torch.equal(p, q) for p, q in zip(ps, before)) and not opt.state
