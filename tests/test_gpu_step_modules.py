"""Linear.loss, AdamW and grad_norm as modules: against torch in float64, on another stream, captured, checkpointed,
and all of them together in training steps.

Tolerances: with bf16 operands a product's terms carry 2^-8 each (operand roundings of 2^-9 twice, gradients 2^-8):
relative norms of 0.01 hold them with their sums.  AdamW in float32 repeats torch's formula with other roundings:
a step is off by 2^-20 of itself.
"""
import copy
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def blocks():
    from paper_2408_14267_amd import blocks as b
    return b


def gen(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + sum(shape))
    return torch.randn(shape, generator=g, device="cuda")


def rel(a, b):
    return (torch.linalg.vector_norm(a.double() - b.double()) / torch.linalg.vector_norm(b.double())).item()


def targets(shape, classes, seed=0, ignored=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(classes, shape, generator=g, device="cuda")
    return torch.where(torch.rand(shape, generator=g, device="cuda") < ignored, -100, t)


# ----------------------------------------------------------------------------- loss

@pytest.mark.parametrize("operands", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("shape,classes,fin", [((3,), 7, 40), ((4, 33), 100, 96), ((300,), 1000, 64)])
@pytest.mark.parametrize("reduction", ["mean", "none"])
@pytest.mark.parametrize("smoothing", [0.0, 0.1])
def test_loss_of_a_layer(operands, shape, classes, fin, reduction, smoothing):
    b = blocks()
    mod = b.Linear(fin, classes, operands=operands).cuda()
    mod.weight.data.mul_(3)
    mod.bias.data += 0.3 * gen(classes, seed=9)
    x = gen(*shape, fin, seed=1).requires_grad_()
    t = targets(shape, classes, ignored=0.2 if len(shape) > 1 else 0.0)
    # the reference takes the operands as they are quantized (straight through)
    xq, xs = b._quantized(x.detach().reshape(-1, fin), operands)
    wq, ws = b._quantized(mod.weight.detach(), operands)
    X, W = ((q.float().double() * (1 if s is None else s.double()[:, None])).requires_grad_() for q, s in ((xq, xs), (wq, ws)))
    B = mod.bias.detach().double().requires_grad_()
    want = torch.nn.functional.cross_entropy(X @ W.t() + B, t.reshape(-1), label_smoothing=smoothing, reduction=reduction)
    got = mod.loss(x, t, smoothing=smoothing, reduction=reduction)
    assert got.dtype == torch.float32 and got.shape == (t.shape if reduction == "none" else ())
    assert rel(got.reshape(-1), want.reshape(-1)) < 1e-5
    if reduction == "none":
        a = gen(t.numel(), seed=3)
        (got.reshape(-1) * a).sum().backward()
        (want * a.double()).sum().backward()
    else:
        (2.5 * got).backward()
        (2.5 * want).backward()
    assert x.grad.shape == x.shape and rel(x.grad.reshape(-1, fin), X.grad) < 0.01
    assert rel(mod.weight.grad, W.grad) < 0.01 and rel(mod.bias.grad, B.grad) < 1e-4


def test_loss_equals_that_of_the_outputs():
    b = blocks()
    mod = b.Linear(64, 50).cuda()
    x, t = gen(40, 64), targets((40,), 50)
    want = torch.nn.functional.cross_entropy(mod(x).double(), t)
    assert abs(mod.loss(x, t).item() - want.item()) < 1e-5
    assert mod.loss(x[:0], t[:0]).item() == 0
    assert mod.loss(x.bfloat16(), t).dtype == torch.float32


def test_loss_refusals():
    b = blocks()
    mod = b.Linear(16, 5).cuda()
    x, t = gen(4, 16), torch.zeros(4, dtype=torch.int64, device="cuda")
    for bad in (t.int(), t[:3], t.cpu(), t[:, None]):
        with pytest.raises(ValueError, match="target"):
            mod.loss(x, bad)
    with pytest.raises(ValueError, match="reduction"):
        mod.loss(x, t, reduction="sum")
    with pytest.raises(ValueError, match="no logits"):
        b.Linear(16, 5, act="relu").cuda().loss(x, t)
    with pytest.raises(RuntimeError):
        mod.loss(x, t, smoothing=1.5)
    with pytest.raises(RuntimeError):
        x.requires_grad_()
        g, = torch.autograd.grad(mod.loss(x, t), x, create_graph=True)
        g.sum().backward()                               # not differentiable twice: refused, not wrong


def test_loss_of_frozen_parts():
    b = blocks()
    mod = b.Linear(32, 20).cuda()
    x, t = gen(30, 32), targets((30,), 20)
    mod.loss(x, t).backward()
    whole = mod.weight.grad.clone(), mod.bias.grad.clone()
    mod.weight.requires_grad_(False)
    mod.weight.grad = mod.bias.grad = None
    mod.loss(x, t).backward()
    assert mod.weight.grad is None and torch.equal(mod.bias.grad, whole[1])
    mod.bias.requires_grad_(False)
    x.requires_grad_()
    mod.loss(x, t).backward()
    assert torch.isfinite(x.grad).all() and mod.weight.grad is None
    # the scalar may be changed in place
    loss = mod.loss(x, t)
    loss /= 2
    loss.backward()


# ----------------------------------------------------------------------------- AdamW

def weights(seed=0):
    conv = torch.nn.Parameter(gen(16, 8, 3, 3, seed=seed).to(memory_format=torch.channels_last))
    return [torch.nn.Parameter(gen(300, 70, seed=seed + 1)), conv, torch.nn.Parameter(gen(5, seed=seed + 2)),
            torch.nn.Parameter(gen(40, 30, seed=seed + 3).t()), torch.nn.Parameter(gen(1, seed=seed + 4)[0])]


@pytest.mark.parametrize("max_norm", [None, 0.5])
def test_adamw_against_torch(max_norm):
    b = blocks()
    mine, theirs = weights(), [p.detach().double().clone().requires_grad_() for p in weights()]
    kw = dict(lr=0.01, betas=(0.8, 0.95), eps=1e-6)
    opt = b.AdamW([dict(params=mine[:2], weight_decay=0.1), dict(params=mine[2:])], max_norm=max_norm, **kw)
    ref = torch.optim.AdamW([dict(params=theirs[:2], weight_decay=0.1), dict(params=theirs[2:], weight_decay=0.0)], **kw)
    for s in range(5):
        for i, (p, q) in enumerate(zip(mine, theirs)):
            if i == 2 and s == 1:                          # a weight without a gradient counts no step
                p.grad = q.grad = None
                continue
            g = gen(*p.shape, seed=10 * s + i)
            p.grad, q.grad = g, g.double()
        if max_norm is not None:
            norm = torch.nn.utils.clip_grad_norm_([q for q in theirs if q.grad is not None], max_norm)
        opt.step()
        ref.step()
        if max_norm is not None:
            assert abs(opt.grad_norm[0].item() - norm.item()) < 1e-6 * norm.item()
        for p, q in zip(mine, theirs):
            assert ((p.detach().double() - q.detach()).abs() <= 2.0 ** -22 * q.detach().abs() * (s + 1) + 1e-7 * (s + 1)).all()


def test_adamw_takes_a_scheduler_and_moved_weights():
    b = blocks()
    p = torch.nn.Parameter(gen(1000))
    opt = b.AdamW([p], lr=0.1, eps=0.0)
    sched = torch.optim.lr_scheduler.StepLR(opt, 1, 0.5)
    for lr in (0.1, 0.05, 0.025):
        before = p.detach().clone()
        p.grad = torch.ones_like(p)
        opt.step()
        assert torch.allclose(before - p.detach(), torch.full_like(before, lr), rtol=1e-4)
        sched.step()
        p.data = p.detach().clone()                      # elsewhere now
    assert torch.isfinite(p).all()


@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_adamw_checkpoint(states):
    b = blocks()

    def run(params, opt, seeds):
        for s in seeds:
            for i, p in enumerate(params):
                p.grad = gen(*p.shape, seed=10 * s + i)
            opt.step()

    a, c = weights(), weights()
    oa, oc = (b.AdamW(w, lr=0.01, states=states, seed=5) for w in (a, c))
    run(a, oa, range(3))
    for p, q in zip(c, a):
        p.data.copy_(q.data)
    oc.load_state_dict(copy.deepcopy(oa.state_dict()))
    if states == "e4m3":
        assert oc.state[c[0]]["m"].dtype == torch.float8_e4m3fn
    run(a, oa, range(3, 6))
    run(c, oc, range(3, 6))
    assert all(torch.equal(p, q) for p, q in zip(a, c))
    with pytest.raises(ValueError, match="another kind"):
        b.AdamW(weights(), states="f32" if states == "e4m3" else "e4m3").load_state_dict(oa.state_dict())


def test_adamw_states_follow_their_weights():
    """Weights whose memory order changes between steps, by a conversion, a view or a checkpoint of another model."""
    b = blocks()
    values = [gen(16, 8, 3, 3, seed=1), gen(20, 20, seed=2), gen(6, 5, 1, 1, seed=3)]
    mine = [torch.nn.Parameter(v.clone()) for v in values]
    theirs = [torch.nn.Parameter(v.double()) for v in values]
    kw = dict(lr=0.01, betas=(0.8, 0.95), weight_decay=0.1)
    opt, ref = b.AdamW(mine, **kw), torch.optim.AdamW(theirs, **kw)

    def steps(opt, weights, seed):
        for s in range(2):
            for i, (p, q) in enumerate(zip(weights, theirs)):
                g = gen(*p.shape, seed=seed + 10 * s + i)
                p.grad, q.grad = g, g.double()
            opt.step()
            ref.step()
        for p, q in zip(weights, theirs):                  # (the formula's float32 roundings, a few of 2^-24 a step)
            assert (p.double() - q).abs().max() <= 4e-6 * max(1, q.abs().max().item())
    steps(opt, mine, 100)
    mine[0].data = mine[0].data.to(memory_format=torch.channels_last)
    mine[2].data = mine[2].data.to(memory_format=torch.channels_last)
    steps(opt, mine, 200)
    assert opt.state[mine[0]]["m"].stride() == mine[0].stride()
    for p in (mine[1], theirs[1]):
        p.data = p.data.t()                                # at the same address
    steps(opt, mine, 300)
    other = [torch.nn.Parameter(p.detach().clone(memory_format=torch.contiguous_format)) for p in mine]
    again = b.AdamW(other, **kw)
    again.load_state_dict(copy.deepcopy(opt.state_dict()))
    steps(again, other, 400)
    # states of other shapes
    wrong = [torch.nn.Parameter(p.detach().flatten()) for p in mine]
    refused = b.AdamW(wrong, **kw)
    refused.load_state_dict(copy.deepcopy(opt.state_dict()))
    for p in wrong:
        p.grad = torch.ones_like(p)
    before = [p.detach().clone() for p in wrong]
    with pytest.raises(ValueError, match="states of shapes"):
        refused.step()
    assert all(torch.equal(p, q) for p, q in zip(wrong, before))


def test_adamw_8_bit_states_of_another_memory_order():
    b = blocks()
    conv, point, rest = (torch.nn.Parameter(gen(*n, seed=i)) for i, n in enumerate([(16, 8, 3, 3), (6, 5, 1, 1), (9,)]))
    opt = b.AdamW([rest, point, conv], states="e4m3")

    def step():
        for p in (conv, point, rest):
            p.grad = torch.ones_like(p)
        opt.step()
    step()
    point.data = point.data.to(memory_format=torch.channels_last)      # the same memory order
    step()
    contiguous = conv.data
    conv.data = conv.data.to(memory_format=torch.channels_last)
    before = [p.detach().clone() for p in (conv, point, rest)]
    with pytest.raises(ValueError, match="8-bit states of weights with strides"):
        step()
    assert all(torch.equal(p, q) for p, q in zip((conv, point, rest), before))
    assert {s["step"] for s in opt.state.values()} == {2}
    conv.data = contiguous
    step()
    other = [torch.nn.Parameter(p.detach().clone()) for p in (rest, point, conv)]
    again = b.AdamW(other, states="e4m3")
    again.load_state_dict(copy.deepcopy(opt.state_dict()))
    for p, q in zip(other, (rest, point, conv)):
        p.grad = q.grad = torch.ones_like(p)
    again.step()
    opt.step()
    assert all(torch.equal(p, q) for p, q in zip(other, (rest, point, conv)))


def test_adamw_copies_and_gradients_of_some():
    """A deep copy goes on like its original; weights with and without gradients change from step to step; gradients
    are not held after a step."""
    import gc
    import weakref
    b = blocks()
    params = weights()
    opt = b.AdamW(params, lr=0.01, states="e4m3", max_norm=1.0)
    for s in range(4):
        for i, p in enumerate(params):
            p.grad = gen(*p.shape, seed=10 * s + i) if (i + s) % 2 else None
        held = [weakref.ref(p.grad) for p in params if p.grad is not None]
        opt.step()
        for p in params:
            p.grad = None
        gc.collect()
        assert all(r() is None for r in held)
        assert len(opt._lists) <= 2
    both = copy.deepcopy((params, opt))
    for q, o in ((params, opt), both):
        for i, p in enumerate(q):
            p.grad = gen(*p.shape, seed=50 + i)
        o.step()
    assert all(torch.equal(p, q) for p, q in zip(params, both[0]))


def test_adamw_refusals():
    b = blocks()
    for bad in (torch.zeros(3, device="cuda").double(), torch.zeros(3, 4, device="cuda")[:, :2]):
        with pytest.raises(ValueError, match="float32 weights"):
            b.AdamW([torch.nn.Parameter(bad)])
    p = torch.nn.Parameter(gen(10))
    for kw in (dict(lr=-1), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=math.nan), dict(weight_decay=-1),
               dict(states="int8"), dict(max_norm=0.0), dict(max_norm=-1.0)):
        with pytest.raises(ValueError):
            b.AdamW([p], **kw)
    opt = b.AdamW([p, torch.nn.Parameter(torch.zeros(4))])
    opt.param_groups[0]["params"][1].grad = torch.zeros(4)
    p.grad = torch.ones(10, device="cuda")
    before = p.detach().clone()
    with pytest.raises(ValueError, match="current device"):
        opt.step()
    assert torch.equal(p, before)                        # nothing was updated
    for kind in ("f32", "e4m3"):                         # and nothing is left that a checkpoint would carry
        opt = b.AdamW([p, torch.nn.Parameter(torch.zeros(4))], states=kind)
        opt.param_groups[0]["params"][1].grad = torch.zeros(4)
        with pytest.raises(ValueError):
            opt.step()
        b.AdamW([p, torch.nn.Parameter(torch.zeros(4))], states=kind).load_state_dict(opt.state_dict())
    from paper_2408_14267_amd import train
    with pytest.raises(ValueError, match="autocast"):
        train.train_step(b.ResidualMLP(8, 3, width=16, hidden=16, depth=0).cuda(), b.Optimizers(), None, None,
                         autocast_dtype=torch.bfloat16, fused_loss=True)
    with pytest.raises(ValueError, match="max_norm"):
        b.muon_and_adam(torch.nn.Linear(3, 3), max_norm=1.0)


def test_grad_norm():
    b = blocks()
    params = weights()
    with pytest.raises(ValueError, match="no gradients"):
        b.grad_norm(params)
    for i, p in enumerate(params[:-1]):
        p.grad = gen(*p.shape, seed=i)
    want = math.sqrt(sum(p.grad.double().square().sum().item() for p in params[:-1]))
    norm, factor = b.grad_norm(params, 0.5)
    assert abs(norm.item() - want) < 1e-6 * want and abs(factor.item() - 0.5 / want) < 1e-6


# ----------------------------------------------------------------------------- together

@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_training_steps(states):
    """Loss, its gradients, norm and AdamW over a whole network with binary layers, beside the same with torch's
    cross entropy and Adam: the first step has the same gradients, up to bf16."""
    from paper_2408_14267_amd import train
    b = blocks()
    torch.manual_seed(0)
    model = b.ResidualMLP(48, 10, width=64, hidden=96, depth=2, operands="bf16").cuda()
    other = copy.deepcopy(model)
    opt = b.AdamW(model.parameters(), lr=1e-3, states=states, max_norm=1.0)
    x, y = gen(70, 48, seed=1), torch.randint(10, (70,), device="cuda")
    loss = train.train_step(model, opt, x, y, fused_loss=True)
    want = torch.nn.functional.cross_entropy(other(x), y)
    want.backward()
    assert abs(loss.item() - want.item()) < 1e-4
    for (name, p), q in zip(model.named_parameters(), other.parameters()):
        assert rel(p.grad, q.grad) < 0.05, name
    norm = math.sqrt(sum(p.grad.double().square().sum().item() for p in model.parameters()))
    assert abs(opt.grad_norm[0].item() - norm) < 1e-5 * norm
    for _ in range(3):
        loss = train.train_step(model, opt, x, y, fused_loss=True)
    assert torch.isfinite(loss) and all(torch.isfinite(p).all() for p in model.parameters())


@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_a_captured_training_step(states):
    """Forward, loss, backward, clipping and the step in one graph, replayed beside eager steps."""
    b = blocks()

    def make():
        torch.manual_seed(0)
        m = torch.nn.Sequential(b.NormLinear(40, 64, act="gelu", operands="bf16"), b.Linear(64, 30)).cuda()
        return m, b.AdamW(m.parameters(), lr=0.01, states=states, max_norm=0.5, capturable=True)

    def one(m, o, x, t):
        # (nothing of the autograd graph is kept: its accumulators belong to the stream of the call)
        grads = torch.autograd.grad(m[1].loss(m[0](x), t), list(m.parameters()))
        for p, g in zip(m.parameters(), grads):
            p.grad = g
        o.step()

    (ma, oa), (mb, ob) = make(), make()
    x, t = gen(50, 40), targets((50,), 30)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one(ma, oa, x, t)
    torch.cuda.current_stream().wait_stream(side)
    one(mb, ob, x, t)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(ma, oa, x, t)
    for s in range(1, 5):
        x.copy_(gen(50, 40, seed=s))
        t.copy_(targets((50,), 30, seed=s))
        graph.replay()
        one(mb, ob, x, t)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(ma.parameters(), mb.parameters())), s
        assert torch.equal(oa.grad_norm, ob.grad_norm)


def test_two_graphs_of_a_loss():
    """Each graph has workspaces of its own: replayed one after the other, on streams side by side, and between eager calls."""
    b = blocks()
    mods = [b.Linear(64, n, operands=o).cuda() for n, o in ((300, "bf16"), (5000, "int8"))]
    xs, ts = [gen(m, 64, seed=m) for m in (200, 40)], [targets((m,), n) for m, n in ((200, 300), (40, 5000))]

    def call(i):
        return torch.autograd.grad(mods[i].loss(xs[i], ts[i]), list(mods[i].parameters()))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i in range(2):
            call(i)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call(i))
        graphs.append(graph)
    for s in range(3):
        for i in range(2):
            xs[i].copy_(gen(*xs[i].shape, seed=10 * s + i))
        want = [[g.clone() for g in call(i)] for i in range(2)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(p, q) for p, q in zip(want[i], outs[i])), (s, i)


def test_adamw_on_another_stream_and_with_other_states():
    b = blocks()
    (pa, pb) = (weights(), weights())
    oa, ob = (b.AdamW(p, lr=0.01, max_norm=0.5) for p in (pa, pb))
    side = torch.cuda.Stream()
    for s in range(3):
        for i, (p, q) in enumerate(zip(pa, pb)):
            p.grad, q.grad = gen(*p.shape, seed=10 * s + i), gen(*p.shape, seed=10 * s + i)
        oa.step()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            ob.step()
        torch.cuda.current_stream().wait_stream(side)
        if s == 0:                                           # the same states in other tensors
            ob.state[pb[0]] = {k: v.clone() if torch.is_tensor(v) else v for k, v in ob.state[pb[0]].items()}
    assert all(torch.equal(p, q) for p, q in zip(pa, pb))


def test_a_first_step_is_not_captured():
    b = blocks()
    p = torch.nn.Parameter(gen(100))
    p.grad = torch.ones_like(p)
    for capturable, match in ((True, "before a capture"), (False, "capturable")):
        opt = b.AdamW([p], capturable=capturable)
        with pytest.raises(RuntimeError, match=match):
            with torch.cuda.graph(torch.cuda.CUDAGraph()):
                opt.step()
    torch.cuda.synchronize()


def test_example_runs():
    spec = importlib.util.spec_from_file_location("example", os.path.join(ROOT, "examples", "train_residual_mlp.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.main(["--steps", "4", "--fused-loss", "--states", "e4m3", "--clip", "1.0"])
    assert len(losses) == 4 and all(math.isfinite(v) for v in losses)
