"""What the modules and the optimizer refuse before anything runs (no GPU needed)."""
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
