"""Modules with frozen parameters: the products that nothing asks for are not computed, the others keep their bits."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def gen(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + sum(shape))
    return torch.randn(shape, generator=g, device="cuda")


@pytest.fixture
def asked(monkeypatch):
    """What each backward of a product was asked for."""
    from paper_2408_14267_amd import dense
    calls = []

    def call(*args, _f=dense.fqt_linear_backward, **kw):
        calls.append({k for k in ("dx", "dw", "dbias") if kw.get(k) is not None})
        return _f(*args, **kw)
    monkeypatch.setattr(dense, "fqt_linear_backward", call)
    return calls


@pytest.mark.parametrize("kind", ["linear", "norm_linear"])
@pytest.mark.parametrize("operands", ["int8", "bf16"])
@pytest.mark.parametrize("frozen", [("weight",), ("bias",), ("weight", "bias"), ("x",), ("x", "weight"),
                                    ("x", "norm_weight"), ("x", "norm_weight", "weight")])
def test_frozen(kind, operands, frozen, asked):
    from paper_2408_14267_amd import blocks as b
    if kind == "linear" and "norm_weight" in frozen:
        frozen = tuple(f for f in frozen if f != "norm_weight")
    mod = (b.Linear if kind == "linear" else b.NormLinear)(96, 56, act="gelu", operands=operands).cuda()
    dy = gen(70, 56, seed=2)

    def grads(off):
        x = gen(70, 96, seed=1)
        named = {"x": x, **dict(mod.named_parameters())}
        for n, t in named.items():
            t.grad = None
            t.requires_grad_(n not in off)
        mod(x).backward(dy)
        return {n: None if t.grad is None else t.grad.clone() for n, t in named.items()}

    full = grads(())
    part = grads(frozen)
    for n, g in part.items():
        assert (g is None) == (n in frozen), n
        assert g is None or torch.equal(g, full[n]), n
    assert asked[0] == {"dx", "dw", "dbias"}
    through = "x" not in frozen or (kind == "norm_linear" and "norm_weight" not in frozen)
    want = {"dx"} if through else set()
    want |= {d for d, n in (("dw", "weight"), ("dbias", "bias")) if n not in frozen}
    assert asked[1] == want
