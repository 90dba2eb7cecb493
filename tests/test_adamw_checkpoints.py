"""Checkpoints of blocks.AdamW: step numbers that are kept in the states or on the device, states of other optimizers, what a step
refuses before it updates anything."""
import copy
import io

import pytest

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2408_14267_amd.fqt", reason="libfqt.so not built")
from paper_2408_14267_amd import blocks  # noqa: E402

SHAPES = [[(30, 7), (5,)], [(300,)]]


def gen(*shape, seed=0, device="cpu"):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed * 7919 + sum(shape))).to(device)


def groups(device="cpu"):
    return [dict(params=[torch.nn.Parameter(gen(*s, seed=i, device=device)) for i, s in enumerate(g)]) for g in SHAPES]


def with_states(opt, numbers, clocks=None):
    """Float32 states as after this many steps."""
    for g, group in enumerate(opt.param_groups):
        for p, n in zip(group["params"], numbers[g]):
            if n is not None:
                opt.state[p] = {"step": n, "m": torch.ones_like(p), "v": torch.ones_like(p)}
        if clocks and clocks[g] is not None:
            group["clock"] = torch.tensor([clocks[g]])
    return opt


def numbers(opt):
    return [[opt.state[p]["step"] if opt.state.get(p) else None for p in g["params"]] for g in opt.param_groups]


def clocks(opt):
    return [None if g.get("clock") is None else g["clock"].item() for g in opt.param_groups]


def test_plain_to_capturable():
    old = with_states(blocks.AdamW(groups()), [[1000, 1000], [7]])
    new = blocks.AdamW(groups(), capturable=True)
    new.load_state_dict(copy.deepcopy(old.state_dict()))
    assert clocks(new) == [1000, 7] and new.param_groups[0]["clock"].dtype == torch.int64
    # a weight that has had no gradient counts with its group; a group without states has no number yet
    old = with_states(blocks.AdamW(groups()), [[1000, None], [None]])
    new = blocks.AdamW(groups(), capturable=True)
    new.load_state_dict(copy.deepcopy(old.state_dict()))
    assert clocks(new) == [1000, None]


def test_plain_to_capturable_of_different_numbers():
    old = with_states(blocks.AdamW(groups()), [[1000, 999], [7]])
    new = with_states(blocks.AdamW(groups(), capturable=True), [[0, 0], [0]], [3, 3])
    with pytest.raises(ValueError, match="different numbers of steps"):
        new.load_state_dict(copy.deepcopy(old.state_dict()))
    assert clocks(new) == [3, 3] and numbers(new) == [[0, 0], [0]]         # nothing was loaded


def test_capturable_to_plain():
    old = with_states(blocks.AdamW(groups(), capturable=True), [[0, None], [0]], [1000, 7])
    new = blocks.AdamW(groups())
    new.load_state_dict(copy.deepcopy(old.state_dict()))
    assert numbers(new) == [[1000, None], [7]] and clocks(new) == [None, None]
    # and back
    again = blocks.AdamW(groups(), capturable=True)
    again.load_state_dict(copy.deepcopy(new.state_dict()))
    assert clocks(again) == [1000, 7]
    assert all(torch.equal(again.state[p]["m"], torch.ones_like(p)) for p in again.state)


def test_capturable_to_capturable():
    old = with_states(blocks.AdamW(groups(), capturable=True), [[0, 0], [0]], [1000, 7])
    new = blocks.AdamW(groups(), capturable=True)
    new.load_state_dict(old.state_dict())
    assert clocks(new) == [1000, 7]
    old.param_groups[0]["clock"].add_(1)                               # a counter of its own
    assert clocks(new) == [1000, 7]


def saved(opt):
    f = io.BytesIO()
    torch.save(opt.state_dict(), f)
    f.seek(0)
    return torch.load(f, map_location="cpu", weights_only=True)


@pytest.mark.gpu
@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_steps_go_on_in_either_mode(states):
    """Plain, capturable and plain again, each from a checkpoint on the host: the same bits as one optimizer's steps."""
    def steps(opt, seeds):
        for s in seeds:
            for group in opt.param_groups:
                for i, p in enumerate(group["params"]):
                    p.grad = gen(*p.shape, seed=10 * s + i, device="cuda")
            opt.step()
    kw = dict(lr=0.01, states=states, seed=5, max_norm=1.0)
    one = blocks.AdamW(groups("cuda"), **kw)
    steps(one, range(9))
    now = blocks.AdamW(groups("cuda"), **kw)
    steps(now, range(2))
    for i, capturable in enumerate((True, True, False)):
        then = blocks.AdamW(groups("cuda"), capturable=capturable, **kw)
        for g, h in zip(then.param_groups, now.param_groups):
            for p, q in zip(g["params"], h["params"]):
                p.data.copy_(q.data)
        then.load_state_dict(saved(now))
        steps(then, range(2 + 2 * i, 4 + 2 * i))
        now = then
    steps(now, range(8, 9))
    for g, h in zip(one.param_groups, now.param_groups):
        assert all(torch.equal(p, q) for p, q in zip(g["params"], h["params"]))
    assert numbers(now) == [[9, 9], [9]]


@pytest.mark.gpu
def test_a_counter_elsewhere_is_refused():
    opt = blocks.AdamW(groups("cuda"), capturable=True)

    def step():
        for group in opt.param_groups:
            for p in group["params"]:
                p.grad = torch.ones_like(p)
        opt.step()
    step()
    before = [p.detach().clone() for g in opt.param_groups for p in g["params"]]
    opt.param_groups[1]["clock"] = torch.tensor([1])
    with pytest.raises(ValueError, match="counter"):
        step()
    assert clocks(opt) == [1, 1]
    assert all(torch.equal(p, q) for p, q in zip(before, [p for g in opt.param_groups for p in g["params"]]))


# ----------------------------------------------------------------------------- what is refused

@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_states_of_another_optimizer(states):
    p = torch.nn.Parameter(gen(30, 7))
    p.grad = torch.ones_like(p)
    other = torch.optim.AdamW([p])
    other.step()
    opt = blocks.AdamW([p], states=states)
    with pytest.raises(ValueError, match="state"):
        opt.load_state_dict(other.state_dict())
    assert not opt.state.get(p)
    # and a part of one of its own
    whole = with_states(blocks.AdamW([p]), [[3]]).state_dict()
    for missing in ("step", "m", "v"):
        part = copy.deepcopy(whole)
        del part["state"][0][missing]
        opt = blocks.AdamW([p])
        with pytest.raises(ValueError, match=missing):
            opt.load_state_dict(part)
        assert not opt.state.get(p)
    blocks.AdamW([p]).load_state_dict(whole)


@pytest.mark.parametrize("kw", [dict(lr=2e30), dict(eps=2e30), dict(weight_decay=2e30), dict(lr=1e20, weight_decay=1e20)])
def test_settings_that_a_step_refuses(kw):
    """What fqt_adamw_step takes no value of is refused with its group, not in a step whose other groups are updated."""
    a, b = (torch.nn.Parameter(gen(5)) for _ in range(2))
    opt = blocks.AdamW([a])
    with pytest.raises(ValueError, match="out of range"):
        opt.add_param_group(dict(params=[b], **kw))
    assert len(opt.param_groups) == 1
    opt.add_param_group(dict(params=[b], lr=1e30))


@pytest.mark.gpu
def test_settings_changed_between_steps():
    opt = blocks.AdamW(groups("cuda"))

    def step():
        for group in opt.param_groups:
            for p in group["params"]:
                p.grad = torch.ones_like(p)
        opt.step()
    step()
    opt.param_groups[1]["lr"] = 1e31
    before = [p.detach().clone() for g in opt.param_groups for p in g["params"]]
    with pytest.raises(ValueError, match="out of range"):
        step()
    assert numbers(opt) == [[1, 1], [1]]
    assert all(torch.equal(p, q) for p, q in zip(before, [p for g in opt.param_groups for p in g["params"]]))


@pytest.mark.parametrize("shape", [(0,), (5, 0), (0, 5), (3, 0, 2)])
def test_empty_weights(shape):
    """A weight of no elements has no gaps, whatever its strides."""
    opt = blocks.AdamW([torch.nn.Parameter(torch.zeros(shape))])
    assert len(opt.param_groups[0]["params"]) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("states", ["f32", "e4m3"])
@pytest.mark.parametrize("change", ["gaps", "bf16"])
@pytest.mark.parametrize("first", [True, False])
def test_weights_that_changed(states, change, first):
    """A weight that can no longer be updated is refused before a state is made or another weight is updated."""
    q, p = (torch.nn.Parameter(gen(*s, device="cuda")) for s in ((7,), (40, 6)))
    opt = blocks.AdamW([dict(params=[q]), dict(params=[p])], states=states)

    def step():
        for t in (p, q):
            t.grad = torch.ones_like(t)
        opt.step()
    if not first:
        step()
    good = p.data
    p.data = torch.zeros(40, 12, device="cuda")[:, :6] if change == "gaps" else good.bfloat16()
    before = q.detach().clone()
    with pytest.raises(ValueError, match="AdamW"):
        step()
    assert torch.equal(q, before)
    assert [opt.state[t]["step"] for t in (p, q) if opt.state.get(t)] == ([] if first else [1, 1])
    p.grad, p.data = None, good
    step()
    assert torch.isfinite(p).all() and not torch.equal(q, before)
