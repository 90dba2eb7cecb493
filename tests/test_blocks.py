"""What the modules and the optimizer refuse before anything runs (no GPU needed)."""
import copy

import pytest

torch = pytest.importorskip("torch")
fqt = pytest.importorskip("paper_2408_14267_amd.fqt", reason="libfqt.so not built")
from paper_2408_14267_amd import blocks  # noqa: E402


def weight(*shape, device="cpu", dtype=torch.float32):
    return torch.nn.Parameter(torch.zeros(*shape, device=device, dtype=dtype))


@pytest.mark.parametrize("kw", [dict(steps=0), dict(steps=33), dict(eps=0.0), dict(eps=float("nan"))])
def test_muon_refuses_settings_when_made(kw):
    with pytest.raises(fqt.FqtError):
        blocks.Muon([weight(4, 8)], **kw)
    opt = blocks.Muon([weight(4, 8)])
    with pytest.raises(fqt.FqtError):
        opt.add_param_group(dict(params=[weight(3, 5)], **kw))
    assert len(opt.param_groups) == 1


@pytest.mark.parametrize("kw", [dict(lr=-1.0), dict(momentum=1.0), dict(momentum=-0.1), dict(weight_decay=-1.0)])
def test_muon_refuses_rates(kw):
    with pytest.raises(ValueError, match="out of range"):
        blocks.Muon([weight(4, 8)], **kw)
    with pytest.raises(ValueError, match="out of range"):
        blocks.Muon([dict(params=[weight(4, 8)], **kw)])


def test_muon_refuses_weights_when_added():
    for bad in (weight(7), weight(4, 4, dtype=torch.bfloat16)):
        with pytest.raises(ValueError, match="float32 matrices"):
            blocks.Muon([weight(4, 8), bad])
    with pytest.raises(fqt.FqtError) as e:
        blocks.Muon([weight(65537, 65537, device="meta")])
    assert e.value.status == fqt.FQT_E_SHAPE
    opt = blocks.Muon([weight(4, 8), weight(2, 0),
                       torch.nn.Parameter(torch.zeros(6, 4, 3, 3).contiguous(memory_format=torch.channels_last))])
    with pytest.raises(ValueError, match="float32 matrices"):
        opt.add_param_group(dict(params=[weight(7)]))
    assert len(opt.param_groups) == 1


def test_optimizers_checkpoint_and_schedule():
    def make():
        torch.manual_seed(0)
        m = torch.nn.Sequential(torch.nn.Linear(4, 8), torch.nn.LayerNorm(8), torch.nn.Linear(8, 2))
        o = blocks.Optimizers(torch.optim.SGD([m[0].weight, m[2].weight], lr=0.1, momentum=0.9),
                              torch.optim.Adam([*m[0].parameters()][1:] + [*m[1].parameters()] + [m[2].bias]))
        return m, o

    def train(m, o, seeds):
        for s in seeds:
            o.zero_grad()
            m(torch.randn(6, 4, generator=torch.Generator().manual_seed(s))).square().sum().backward()
            o.step()

    m, o = make()
    assert [g["lr"] for g in o.param_groups] == [0.1, 1e-3]
    o.param_groups[0]["lr"] = 0.05
    torch.optim.lr_scheduler.StepLR(o.optimizers[1], 1)
    train(m, o, range(3))
    again, p = make()
    again.load_state_dict(m.state_dict())
    p.load_state_dict(copy.deepcopy(o.state_dict()))       # (torch keeps the tensors it is given)
    assert p.param_groups[0]["lr"] == 0.05
    train(m, o, range(3, 6))
    train(again, p, range(3, 6))
    assert all(torch.equal(a, b) for a, b in zip(m.parameters(), again.parameters()))
    with pytest.raises(ValueError, match="a state of 1"):
        p.load_state_dict({"optimizers": o.state_dict()["optimizers"][:1]})


def test_models_without_matrices_or_without_vectors():
    only = blocks.muon_and_adam(torch.nn.Linear(4, 8, bias=False))
    assert [type(o) for o in only.optimizers] == [blocks.Muon]
    vectors = blocks.muon_and_adam(torch.nn.LayerNorm(8))
    assert [type(o) for o in vectors.optimizers] == [torch.optim.Adam]
