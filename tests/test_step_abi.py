"""Host-side checks of the C ABI in include/fqt_step.h: exports, layouts, refusals before any launch, and the
binding's checks of tensors (no GPU needed)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fqt_step.h")

torch = pytest.importorskip("torch")
fqt = pytest.importorskip("paper_2408_14267_amd.fqt", reason="libfqt.so not built")
from paper_2408_14267_amd import dense, step  # noqa: E402

FAKE = 1 << 20          # never dereferenced: validation fails first
BIG = 1 << 50
NAN, INF = float("nan"), float("inf")


def test_exports_every_declared_symbol():
    names = sorted(set(re.findall(r"^int\s+(fqt_\w+)\(", open(HEADER).read(), flags=re.M)))
    assert sorted(step.EXPORTED) == names
    lib = ctypes.CDLL(fqt.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


def test_constants_match_header():
    text = open(HEADER).read()
    for name in ("FQT_STATE_BLOCK", "FQT_MAX_PARAMS"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(step, name)


# ----------------------------------------------------------------------------- loss

def _loss(**kw):
    d = step.loss_desc(8, 16, 32)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _forward(d, x=FAKE, w=FAKE, xs=None, ws_=None, bias=None, target=FAKE, loss=FAKE, lse=FAKE, mean=None, ws=FAKE,
             size=BIG):
    return step._lib.fqt_loss_forward(d, x, w, xs, ws_, bias, target, loss, lse, mean, ws, size, None)


def _backward(d, x=FAKE, w=FAKE, xs=None, ws_=None, bias=None, target=FAKE, lse=FAKE, dloss=FAKE, dmean=None,
              mean=None, dx=FAKE, dw=FAKE, dbias=FAKE, ws=FAKE, size=BIG):
    return step._lib.fqt_loss_backward(d, x, w, xs, ws_, bias, target, lse, dloss, dmean, mean, dx, dw, dbias, ws,
                                       size, None)


@pytest.mark.parametrize("field,value,status", [
    ("x_dtype", 0, fqt.FQT_E_DTYPE), ("x_dtype", 4, fqt.FQT_E_DTYPE), ("dx_dtype", 3, fqt.FQT_E_DTYPE),
    ("dw_dtype", -1, fqt.FQT_E_DTYPE), ("M", -1, fqt.FQT_E_SHAPE), ("N", 0, fqt.FQT_E_SHAPE),
    ("N", -1, fqt.FQT_E_SHAPE), ("K", -1, fqt.FQT_E_SHAPE), ("M", 1 << 31, fqt.FQT_E_SHAPE),
    ("N", (1 << 22) + 1, fqt.FQT_E_SHAPE), ("K", (1 << 22) + 1, fqt.FQT_E_SHAPE), ("ldx", 31, fqt.FQT_E_SHAPE),
    ("ldw", 31, fqt.FQT_E_SHAPE), ("lddx", 8, fqt.FQT_E_SHAPE), ("lddw", -8, fqt.FQT_E_SHAPE),
    ("smoothing", -0.1, fqt.FQT_E_INVAL), ("smoothing", 1.5, fqt.FQT_E_INVAL), ("smoothing", NAN, fqt.FQT_E_INVAL)])
def test_loss_descriptor_refusals(field, value, status):
    d = _loss(**{field: value})
    for backward in (False, True):
        with pytest.raises(fqt.FqtError) as e:
            step.fqt_loss_workspace_size(d, backward)
        assert e.value.status == status
    assert _forward(d) == status and _backward(d) == status


def test_loss_size_limits():
    for M, N, K in ((1 << 30, 1 << 22, 1), (1 << 30, 1, 1 << 22), (1, 1 << 22, 1 << 22)):
        with pytest.raises(fqt.FqtError) as e:
            step.fqt_loss_workspace_size(step.loss_desc(M, N, K))
        assert e.value.status == fqt.FQT_E_SHAPE
    assert step.fqt_loss_workspace_size(step.loss_desc(1, 1, 133144, x_dtype="int8")) > 0
    with pytest.raises(fqt.FqtError):
        step.fqt_loss_workspace_size(step.loss_desc(1, 1, 133145, x_dtype="int8"))


def test_loss_pointer_refusals():
    d, q = _loss(), _loss(x_dtype=dense.FQT_I8)
    for name in ("x", "w", "target", "loss", "lse", "ws"):
        assert _forward(d, **{name: None}) == fqt.FQT_E_NULL, name
    for name in ("x", "w", "target", "lse", "ws", "dloss"):
        assert _backward(d, **{name: None}) == fqt.FQT_E_NULL, name
    for call in (_forward, _backward):
        assert call(q, xs=FAKE) == fqt.FQT_E_NULL and call(q, ws_=FAKE) == fqt.FQT_E_NULL
        assert call(d, xs=FAKE, ws_=FAKE) == fqt.FQT_E_DTYPE
        for name, off in (("x", 8), ("w", 2), ("bias", 2), ("target", 4), ("lse", 2), ("mean", 1), ("ws", 64)):
            more = {} if call is _forward or name != "mean" else {"dloss": None, "dmean": FAKE}
            assert call(d, **{name: FAKE + off}, **more) == fqt.FQT_E_ALIGN, name
    assert _forward(d, loss=FAKE + 2) == fqt.FQT_E_ALIGN
    assert _backward(d, dloss=None, dmean=FAKE + 2, mean=FAKE) == fqt.FQT_E_ALIGN
    for name in ("dx", "dw", "dbias"):
        assert _backward(d, **{name: FAKE + 1}) == fqt.FQT_E_ALIGN
    # either dloss, or dmean with mean
    assert _backward(d, dmean=FAKE, mean=FAKE) == fqt.FQT_E_INVAL
    assert _backward(d, dloss=None, dmean=FAKE) == fqt.FQT_E_INVAL
    assert _backward(d, mean=FAKE) == fqt.FQT_E_INVAL
    for backward, call in ((False, _forward), (True, _backward)):
        for desc in (d, _loss(M=2), _loss(K=31)):
            need = step.fqt_loss_workspace_size(desc, backward)
            if need > 256:
                assert call(desc, size=need - 256) == fqt.FQT_E_WORKSPACE
    assert _backward(d, dx=None, dw=None, dbias=None, ws=None) == fqt.FQT_OK      # nothing asked for


def test_loss_workspace_stays_below_the_outputs():
    # a piece of dz and a pair for 64 columns, not M x N outputs
    d = step.loss_desc(16384, 1 << 20, 64)
    assert step.fqt_loss_workspace_size(d) < 16384 * (1 << 20) // 4
    assert step.fqt_loss_workspace_size(d, True) < 16384 * (1 << 20) // 16


@pytest.mark.parametrize("M", [131072, 1 << 20])
@pytest.mark.parametrize("kind,codes", [("bf16", 1), ("int8", 2)])
def test_loss_workspace_of_many_rows(M, kind, codes):
    """dz of a piece has 4096 classes at least (up to 5120 where that is all of them), so of many rows it takes more than 256 MB;
    what else there is: copies and a float32 dx, sums of dbias, a float32 a row."""
    for N, K in ((32768, 512), (65536, 512), (1 << 18, 64), (5120, 512), (4096, 64), (1000, 512)):
        most = 5120 if N <= 5120 else 4096 + 256
        rest = M * K * 8 + most * K * 2 + M * 4 + (M // 32 + 1) * most * 4 + (1 << 28)
        size = step.fqt_loss_workspace_size(step.loss_desc(M, N, K, x_dtype=kind), True)
        assert size <= M * (min(N, most) + 128) * 2 * codes + rest


def test_loss_binding_checks():
    bf = torch.bfloat16
    d = step.loss_desc(4, 8, 16)
    x, w, t = torch.empty(4, 16, dtype=bf), torch.empty(8, 16, dtype=bf), torch.zeros(4, dtype=torch.int64)
    f, ws = torch.empty(4), torch.empty(256, dtype=torch.uint8)
    for bad, match in ((dict(x=x.float()), "x: dtype"), (dict(w=w[:7]), "w: shape"), (dict(w=w.t()), "w: shape"),
                       (dict(target=t.int()), "target"), (dict(target=t[:3]), "target"),
                       (dict(target=t.expand(2, 4).t()[:, 0].contiguous().float()), "target"),
                       (dict(loss=f[:3]), "loss"), (dict(lse=f.double()), "lse"), (dict(mean=f), "mean"),
                       (dict(bias=f), "bias"), (dict(x=None), "required"), (dict(), "device tensor")):
        args = dict(x=x, w=w, target=t, loss=f, lse=f.clone(), ws=ws)
        args.update(bad)
        with pytest.raises(ValueError, match=match):
            step.fqt_loss_forward(d, **args)
    for bad, match in ((dict(), "either"), (dict(dloss=f, dmean=f[:1]), "either"), (dict(dmean=f[:1]), "either"),
                       (dict(dloss=f[:3]), "dloss"), (dict(dmean=f[:2], mean=f[:2]), "dmean"),
                       (dict(dloss=f, dx=x.float()), "dx: dtype"), (dict(dloss=f, dw=w[:3]), "dw: shape"),
                       (dict(dloss=f, dbias=f), "dbias"), (dict(dloss=f), "device tensor")):
        with pytest.raises(ValueError, match=match):
            step.fqt_loss_backward(d, x, w, t, f, ws, **bad)


def test_loss_logp_checks():
    d = _loss()
    for off, status in ((2, fqt.FQT_E_ALIGN), (0, fqt.FQT_E_WORKSPACE)):
        at = FAKE + off
        assert step._lib.fqt_loss_forward_logp(d, FAKE, FAKE, None, None, None, FAKE, FAKE, FAKE, at, None, FAKE, 0,
                                               None) == status
        assert step._lib.fqt_loss_backward_logp(d, FAKE, FAKE, None, None, None, FAKE, FAKE, at, FAKE, None, None, FAKE,
                                                FAKE, FAKE, FAKE, 0, None) == status
    bf = torch.bfloat16
    d = step.loss_desc(4, 8, 16)
    x, w, t = torch.empty(4, 16, dtype=bf), torch.empty(8, 16, dtype=bf), torch.zeros(4, dtype=torch.int64)
    f, ws = torch.empty(4), torch.empty(256, dtype=torch.uint8)
    for bad in (f[:3], f.double(), torch.empty(8)[::2]):
        with pytest.raises(ValueError, match="logp"):
            step.fqt_loss_forward(d, x, w, t, f, f.clone(), ws, logp=bad)
        with pytest.raises(ValueError, match="logp"):
            step.fqt_loss_backward(d, x, w, t, f, ws, dloss=f, logp=bad)


# ----------------------------------------------------------------------------- lists

def _params(count=1, **kw):
    a = (step.fqt_param * count)()
    for d in a:
        d.g = d.p = d.m = d.v = d.m_scale = d.v_scale = FAKE
        d.n, d.first, d.g_dtype = 100, 0, fqt.FQT_F32
        for k, v in kw.items():
            setattr(d, k, v)
    return a


def _norm(a, count=1, max_norm=1.0, out=FAKE, ws=FAKE, size=BIG):
    return step._lib.fqt_grad_norm(a, count, max_norm, out, ws, size, None)


def _adamw(a, count=1, number=1, at=None, scale=None, cfg=None, **kw):
    c = step.adamw_cfg(**({"states": "e4m3"} | kw)) if cfg is None else cfg
    return step._lib.fqt_adamw_step(c, a, count, number, at, scale, None)


def test_list_refusals():
    for kw, status in ((dict(g_dtype=2), fqt.FQT_E_DTYPE), (dict(g_dtype=-1), fqt.FQT_E_DTYPE),
                       (dict(n=-1), fqt.FQT_E_SHAPE), (dict(n=(1 << 40) + 1), fqt.FQT_E_SHAPE),
                       (dict(g=None), fqt.FQT_E_NULL), (dict(g=FAKE + 2), fqt.FQT_E_ALIGN)):
        a = _params(3, **kw)
        assert _norm(a, 3) == status and _adamw(a, 3) == status
    a = _params(1)
    for count, status in ((-1, fqt.FQT_E_SHAPE), (65537, fqt.FQT_E_SHAPE)):
        assert _norm(a, count) == status and _adamw(a, count) == status
    assert _norm(None) == fqt.FQT_E_NULL and _adamw(None) == fqt.FQT_E_NULL


def test_norm_refusals():
    a = _params(1)
    for v in (0.0, -1.0, NAN):
        assert _norm(a, max_norm=v) == fqt.FQT_E_INVAL
    assert _norm(a, out=None) == fqt.FQT_E_NULL and _norm(a, ws=None) == fqt.FQT_E_NULL
    assert _norm(a, out=FAKE + 2) == fqt.FQT_E_ALIGN and _norm(a, ws=FAKE + 8) == fqt.FQT_E_ALIGN
    assert _norm(a, size=8) == fqt.FQT_E_WORKSPACE


def test_adamw_refusals():
    a = _params(1)
    for kw in (dict(lr=-1.0), dict(lr=NAN), dict(lr=INF), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
               dict(beta2=NAN), dict(eps=-1e-8), dict(eps=NAN), dict(weight_decay=-1.0), dict(weight_decay=INF),
               dict(number=0), dict(number=-5)):
        assert _adamw(a, **kw) == fqt.FQT_E_INVAL, kw
    assert _adamw(a, states="int8") == fqt.FQT_E_DTYPE and _adamw(a, states="bf16") == fqt.FQT_E_DTYPE
    for name in ("p", "m", "v", "m_scale", "v_scale"):
        assert _adamw(_params(1, **{name: None})) == fqt.FQT_E_NULL, name
    for name in ("p", "m_scale", "v_scale"):
        assert _adamw(_params(1, **{name: FAKE + 2})) == fqt.FQT_E_ALIGN, name
    for name in ("m", "v"):
        assert _adamw(_params(1, **{name: FAKE + 2}), states="f32") == fqt.FQT_E_ALIGN, name
    for first in (-4, 2, 1 << 61):
        assert _adamw(_params(1, first=first)) == fqt.FQT_E_INVAL
    assert _adamw(a, at=FAKE + 4) == fqt.FQT_E_ALIGN and _adamw(a, scale=FAKE + 2) == fqt.FQT_E_ALIGN
    assert step._lib.fqt_adamw_step(None, a, 1, 1, None, None, None) == fqt.FQT_E_NULL
    assert _adamw(_params(1, n=0, g=None, p=None)) == fqt.FQT_OK       # nothing to do
    assert _adamw(None, 0) == fqt.FQT_OK


def test_param_list_checks():
    f = torch.zeros(8)
    with pytest.raises(ValueError, match="come together"):
        step.param_list([f], p=[f])
    with pytest.raises(ValueError, match="1 of p, 2 gradients"):
        step.param_list([f, f], p=[f], m=[f], v=[f])
    with pytest.raises(ValueError, match="dtype"):
        step.param_list([f.double()])
    with pytest.raises(ValueError, match="device tensor"):
        step.param_list([f])
    with pytest.raises(ValueError, match="come together"):
        step.param_list([f], p=[f], m=[f], v=[f], m_scale=[f])
    empty = step.param_list([])
    assert empty.count == 0 and step.fqt_grad_norm_workspace_size(empty) > 0
    with pytest.raises(ValueError, match="p, m and v"):
        step.fqt_adamw_step(step.adamw_cfg(), empty, 1)
    with pytest.raises(ValueError, match="differ"):
        step.fqt_adamw_step(step.adamw_cfg(states="e4m3"), step.param_list([], p=[], m=[], v=[]), 1)
