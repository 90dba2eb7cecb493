"""Workspaces of the modules: bounded over batch sizes, and no two streams or graphs at one of them."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def modules():
    from paper_2408_14267_amd import blocks, dense
    return blocks, dense


def gen(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + sum(shape))
    return torch.randn(shape, generator=g, device="cuda")


@pytest.fixture
def workspaces(monkeypatch):
    """The addresses of the workspaces that the calls get, by call."""
    _, dense = modules()
    seen = []
    for name, at in (("fqt_linear_forward", 4), ("fqt_linear_backward", 4), ("fqt_rmsnorm_backward", 7)):
        def call(*args, _f=getattr(dense, name), _name=name, _at=at, **kw):
            seen.append((_name, args[_at].data_ptr()))
            return _f(*args, **kw)
        monkeypatch.setattr(dense, name, call)
    return seen


def passes(mod, x, dy):
    """Output and gradients.  Nothing of the autograd graph is kept: its accumulators belong to the stream of
    the pass that made them, and a capture that met them would take that stream in."""
    y = mod(x)
    return (y.detach(), *torch.autograd.grad(y, [x, *mod.parameters()], dy))


@pytest.mark.parametrize("operands", ["int8", "e4m3", "bf16"])
def test_memory_is_bounded_over_batch_sizes(operands):
    b, _ = modules()
    mod = b.NormLinear(515, 300, act="gelu", operands=operands).cuda()
    x = gen(600, 515, seed=1)
    passes(mod, x[:600].requires_grad_(), gen(600, 300))
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for M in range(5, 600, 7):
        passes(mod, x[:M].detach().requires_grad_(), gen(M, 300))
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() <= before


def test_optimizer_holds_no_workspace():
    b, _ = modules()
    ps = [torch.nn.Parameter(gen(64 + i, 200 + 40 * i, seed=i)) for i in range(6)]
    opt = b.Muon(ps)
    for p in ps:
        p.grad = gen(*p.shape, seed=9)
    before = torch.cuda.memory_allocated()
    opt.step()
    torch.cuda.synchronize()
    momentum = sum((4 * p.numel() + 511) // 512 * 512 for p in ps)
    assert torch.cuda.memory_allocated() <= before + momentum


@pytest.mark.parametrize("make", ["linear", "norm_linear"])
def test_streams_and_graphs_have_workspaces_of_their_own(make, workspaces):
    """One module, captured twice on top of eager use: three buffers a call, and every replay equals the eager
    result with eager work in between."""
    b, _ = modules()
    mod = (b.Linear(511, 130, act="silu", operands="e4m3") if make == "linear" else
           b.NormLinear(511, 130, act="gelu")).cuda()
    x, dy = gen(40, 511, seed=1).requires_grad_(), gen(40, 130, seed=2)
    want = [t.clone() for t in passes(mod, x, dy)]
    torch.cuda.synchronize()
    workspaces.clear()
    passes(mod, x, dy)
    torch.cuda.synchronize()
    eager = list(workspaces)
    graphs, captured = [], []
    for _ in range(2):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):                       # (torch asks for a warm-up on the side stream)
            passes(mod, x, dy)
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        workspaces.clear()
        with torch.cuda.graph(graph):
            out = passes(mod, x, dy)
        graphs.append((graph, out))
        captured.append(list(workspaces))
    first, second = captured
    for (name, a), (_, c), (_, e) in zip(first, second, eager):
        assert len({a, c, e}) == 3, name
    for i in range(3):
        for graph, out in graphs:
            for t in out:
                t.fill_(float(i))
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(out, want)), i
            assert all(torch.equal(p, q) for p, q in zip(passes(mod, x, dy), want))
