"""The optimizer on weights, gradients and momentum of any memory order: the update of their contiguous twins, bit for bit."""
import copy

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def gen(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + sum(shape))
    return torch.randn(shape, generator=g, device="cuda")


def layouts():
    last = dict(memory_format=torch.channels_last)
    padded = torch.zeros(30, 70, device="cuda")[:, :50]
    return [gen(16, 8, 3, 3, seed=1).contiguous(**last), gen(70, 33, 1, 2, seed=2).contiguous(**last),
            gen(50, 20, seed=3).t(), padded.copy_(gen(30, 50, seed=4)), gen(40, 90, seed=5)]


def test_any_order():
    from paper_2408_14267_amd import blocks as b
    ps = [torch.nn.Parameter(t) for t in layouts()]
    assert sum(not p.is_contiguous() for p in ps) == 4
    twins = [torch.nn.Parameter(p.detach().clone(memory_format=torch.contiguous_format)) for p in ps]
    one, two = b.Muon(ps, lr=0.1, weight_decay=0.1), b.Muon(twins, lr=0.1, weight_decay=0.1)
    where = [(p.data_ptr(), p.stride()) for p in ps]
    for step in range(3):
        for p, q in zip(ps, twins):
            g = gen(*p.shape, seed=10 + step)
            p.grad, q.grad = torch.empty_like(p).copy_(g), g
        one.step()
        two.step()
        if step == 1:
            one.load_state_dict(copy.deepcopy(one.state_dict()))
        for p, q in zip(ps, twins):
            assert torch.equal(p, q) and torch.equal(one.state[p]["momentum"], two.state[q]["momentum"])
    assert where == [(p.data_ptr(), p.stride()) for p in ps]


def test_empty_weights_are_left_alone():
    from paper_2408_14267_amd import blocks as b
    ps = [torch.nn.Parameter(torch.zeros(s, device="cuda")) for s in ((0, 4), (4, 0), (3, 5))]
    opt = b.Muon(ps)
    for p in ps:
        p.grad = torch.ones_like(p)
    opt.step()
    assert (ps[2] != 0).all()
