"""A run of muon_and_adam goes on from its checkpoint as if it had not stopped."""
import copy

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_checkpoint():
    from paper_2408_14267_amd import blocks as b

    def make():
        torch.manual_seed(0)
        m = torch.nn.Sequential(b.Linear(40, 64, act="gelu"), b.RMSNorm(64), b.NormLinear(64, 10)).cuda()
        return m, b.muon_and_adam(m, lr=0.05)

    def train(m, o, seeds):
        for s in seeds:
            g = torch.Generator(device="cuda").manual_seed(s)
            o.zero_grad()
            m(torch.randn(32, 40, generator=g, device="cuda")).square().mean().backward()
            o.step()

    m, o = make()
    train(m, o, range(3))
    again, p = make()
    again.load_state_dict(m.state_dict())
    p.load_state_dict(copy.deepcopy(o.state_dict()))
    train(m, o, range(3, 6))
    train(again, p, range(3, 6))
    assert all(torch.equal(a, c) for a, c in zip(m.parameters(), again.parameters()))
