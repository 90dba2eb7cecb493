"""Host-side checks of the dense operators' C ABI (include/fqt_dense.h): exports, refusals before any
launch, and the binding's checks of tensors (no GPU needed)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fqt_dense.h")

torch = pytest.importorskip("torch")
fqt = pytest.importorskip("paper_2408_14267_amd.fqt", reason="libfqt.so not built")
from paper_2408_14267_amd import dense  # noqa: E402

FAKE = 1 << 20          # never dereferenced: validation fails first
BIG = 1 << 40


def test_exports_every_declared_symbol():
    names = sorted(set(re.findall(r"^int\s+(fqt_\w+)\(", open(HEADER).read(), flags=re.M)))
    assert sorted(dense.EXPORTED) == names
    lib = ctypes.CDLL(fqt.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


def test_constants_match_header():
    text = open(HEADER).read()
    for name in ("FQT_I8", "FQT_E4M3", "FQT_ACT_NONE", "FQT_ACT_RELU", "FQT_ACT_GELU",
                 "FQT_ACT_SILU", "FQT_ACT_HARDTANH"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(dense, name)


# ----------------------------------------------------------------------------- norm

def _norm(**kw):
    d = dense.norm_desc(4, 16, x_dtype="bf16", q_dtype="int8")
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("field,value,status", [
    ("x_dtype", 2, fqt.FQT_E_DTYPE), ("y_dtype", -1, fqt.FQT_E_DTYPE),
    ("q_dtype", 0, fqt.FQT_E_DTYPE), ("q_dtype", 4, fqt.FQT_E_DTYPE),
    ("rows", -1, fqt.FQT_E_SHAPE), ("cols", -1, fqt.FQT_E_SHAPE), ("rows", 1 << 31, fqt.FQT_E_SHAPE),
    ("cols", (1 << 22) + 1, fqt.FQT_E_SHAPE), ("ldx", 15, fqt.FQT_E_SHAPE),
    ("ldq", -1, fqt.FQT_E_SHAPE), ("ldy", (1 << 22) + 1, fqt.FQT_E_SHAPE),
    ("eps", 0.0, fqt.FQT_E_INVAL), ("eps", -1.0, fqt.FQT_E_INVAL),
    ("eps", float("inf"), fqt.FQT_E_INVAL), ("eps", float("nan"), fqt.FQT_E_INVAL)])
def test_norm_descriptor_refusals(field, value, status):
    with pytest.raises(fqt.FqtError) as e:
        dense.fqt_norm_workspace_size(_norm(**{field: value}))
    assert e.value.status == status
    d = _norm(**{field: value})
    assert dense._lib.fqt_rmsnorm_forward(d, FAKE, None, FAKE, None, FAKE, None, None, None,
                                          None) == status
    assert dense._lib.fqt_rmsnorm_backward(d, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, BIG,
                                           None) == status


def test_norm_pointer_refusals():
    f, b, q = (dense._lib.fqt_rmsnorm_forward, dense._lib.fqt_rmsnorm_backward,
               dense._lib.fqt_quantize_rows)
    d = _norm()
    assert f(d, None, None, FAKE, None, FAKE, None, None, None, None) == fqt.FQT_E_NULL
    assert f(d, FAKE, None, None, None, FAKE, None, None, None, None) == fqt.FQT_E_NULL
    assert f(d, FAKE, None, FAKE, None, None, FAKE, None, None, None) == fqt.FQT_E_NULL   # scale
    assert f(d, FAKE, None, FAKE, None, None, None, FAKE, None, None) == fqt.FQT_E_NULL   # codes
    assert f(d, FAKE + 1, None, FAKE, None, FAKE, None, None, None, None) == fqt.FQT_E_ALIGN
    assert f(d, FAKE, None, FAKE + 2, None, FAKE, None, None, None, None) == fqt.FQT_E_ALIGN
    n = _norm(q_dtype=dense.FQT_NO_CODES)
    assert f(n, FAKE, None, FAKE, None, None, FAKE, FAKE, None, None) == fqt.FQT_E_DTYPE
    assert q(n, FAKE, FAKE, FAKE, None) == fqt.FQT_E_DTYPE
    assert q(d, FAKE, None, FAKE, None) == fqt.FQT_E_NULL
    assert f(None, FAKE, None, FAKE, None, FAKE, None, None, None, None) == fqt.FQT_E_NULL
    need = dense.fqt_norm_workspace_size(d)
    assert b(d, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, need - 1, None) == fqt.FQT_E_WORKSPACE
    assert b(d, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE + 16, need, None) == fqt.FQT_E_ALIGN
    assert b(d, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, need, None) == fqt.FQT_E_NULL
    assert b(d, FAKE, FAKE, FAKE, FAKE, None, FAKE, None, FAKE, need, None) == fqt.FQT_E_NULL


# ----------------------------------------------------------------------------- linear

def _linear(**kw):
    d = dense.linear_desc(8, 16, 32)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("field,value,status", [
    ("x_dtype", 0, fqt.FQT_E_DTYPE), ("x_dtype", 4, fqt.FQT_E_DTYPE),
    ("y_dtype", 2, fqt.FQT_E_DTYPE), ("dx_dtype", 3, fqt.FQT_E_DTYPE),
    ("dw_dtype", -1, fqt.FQT_E_DTYPE), ("act", 5, fqt.FQT_E_INVAL), ("act", -1, fqt.FQT_E_INVAL),
    ("M", -1, fqt.FQT_E_SHAPE), ("N", -1, fqt.FQT_E_SHAPE), ("K", -1, fqt.FQT_E_SHAPE),
    ("M", 1 << 31, fqt.FQT_E_SHAPE), ("N", (1 << 22) + 1, fqt.FQT_E_SHAPE), ("ldx", 31, fqt.FQT_E_SHAPE),
    ("ldw", 31, fqt.FQT_E_SHAPE), ("ldr", 15, fqt.FQT_E_SHAPE), ("ldz", -8, fqt.FQT_E_SHAPE),
    ("lddx", 8, fqt.FQT_E_SHAPE), ("lddw", 8, fqt.FQT_E_SHAPE), ("ldy", 15, fqt.FQT_E_SHAPE)])
def test_linear_descriptor_refusals(field, value, status):
    d = _linear(**{field: value})
    for backward in (False, True):
        with pytest.raises(fqt.FqtError) as e:
            dense.fqt_linear_workspace_size(d, backward)
        assert e.value.status == status
    assert dense._lib.fqt_linear_forward(d, FAKE, FAKE, None, None, None, None, None, FAKE, FAKE,
                                         BIG, None) == status
    assert dense._lib.fqt_linear_backward(d, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, FAKE, FAKE,
                                          FAKE, BIG, None) == status


@pytest.mark.parametrize("K,ok", [(133144, True), (133145, False)])
def test_int8_sums_stay_in_32_bits(K, ok):
    assert (127 * 127 * K < 2 ** 31) == ok
    d = dense.linear_desc(1, 1, K, x_dtype="int8")
    if ok:
        assert dense.fqt_linear_workspace_size(d) > 0
    else:
        with pytest.raises(fqt.FqtError) as e:
            dense.fqt_linear_workspace_size(d)
        assert e.value.status == fqt.FQT_E_SHAPE
    assert dense.fqt_linear_workspace_size(dense.linear_desc(1, 1, K)) > 0      # bf16: no such bound


def test_linear_size_limits():
    for M, N, K in ((1 << 30, 1 << 22, 1), (1 << 30, 1, 1 << 22), (1, 1 << 22, 1 << 22)):
        with pytest.raises(fqt.FqtError) as e:
            dense.fqt_linear_workspace_size(dense.linear_desc(M, N, K))
        assert e.value.status == fqt.FQT_E_SHAPE


def test_linear_pointer_refusals():
    f, b = dense._lib.fqt_linear_forward, dense._lib.fqt_linear_backward
    d, q = _linear(), _linear(x_dtype=dense.FQT_I8)
    assert f(d, None, FAKE, None, None, None, None, None, FAKE, FAKE, BIG, None) == fqt.FQT_E_NULL
    assert f(d, FAKE, FAKE, None, None, None, None, None, None, FAKE, BIG, None) == fqt.FQT_E_NULL
    assert f(d, FAKE, FAKE, None, None, None, None, None, FAKE, None, BIG, None) == fqt.FQT_E_NULL
    assert f(q, FAKE, FAKE, None, FAKE, None, None, None, FAKE, FAKE, BIG, None) == fqt.FQT_E_NULL
    assert f(d, FAKE, FAKE, FAKE, FAKE, None, None, None, FAKE, FAKE, BIG, None) == fqt.FQT_E_DTYPE
    assert f(d, FAKE + 8, FAKE, None, None, None, None, None, FAKE, FAKE, BIG, None) == fqt.FQT_E_ALIGN
    assert f(d, FAKE, FAKE, None, None, FAKE + 2, None, None, FAKE, FAKE, BIG, None) == fqt.FQT_E_ALIGN
    assert f(d, FAKE, FAKE, None, None, None, None, None, FAKE, FAKE + 64, BIG, None) == fqt.FQT_E_ALIGN
    odd = _linear(K=31)                       # rows that are not whole 16-byte pieces are copied
    need = dense.fqt_linear_workspace_size(odd)
    assert need >= (8 + 16) * 32 * 2
    assert f(odd, FAKE, FAKE, None, None, None, None, None, FAKE, FAKE, need - 1, None) == fqt.FQT_E_WORKSPACE
    g = _linear(act=dense.FQT_ACT_GELU)
    assert b(g, FAKE, FAKE, None, None, None, FAKE, FAKE, None, None, FAKE, BIG, None) == fqt.FQT_E_NULL
    assert b(d, FAKE, None, None, None, None, FAKE, FAKE, None, None, FAKE, BIG, None) == fqt.FQT_E_NULL
    assert b(d, None, FAKE, None, None, None, FAKE, None, FAKE, None, FAKE, BIG, None) == fqt.FQT_E_NULL
    assert b(q, FAKE, FAKE, None, FAKE, None, FAKE, None, FAKE, None, FAKE, BIG, None) == fqt.FQT_E_NULL
    assert b(q, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, None, None, FAKE, BIG, None) == fqt.FQT_E_NULL
    need = dense.fqt_linear_workspace_size(d, True)
    assert b(d, FAKE, FAKE, None, None, None, FAKE, FAKE, None, None, FAKE, need - 1,
             None) == fqt.FQT_E_WORKSPACE


# ----------------------------------------------------------------------------- orthogonalisation

@pytest.mark.parametrize("field,value,status", [
    ("g_dtype", 2, fqt.FQT_E_DTYPE), ("o_dtype", -1, fqt.FQT_E_DTYPE), ("rows", -1, fqt.FQT_E_SHAPE),
    ("cols", (1 << 22) + 1, fqt.FQT_E_SHAPE), ("ldg", 15, fqt.FQT_E_SHAPE),
    ("ldm", 3, fqt.FQT_E_SHAPE), ("ldo", 3, fqt.FQT_E_SHAPE), ("steps", 0, fqt.FQT_E_INVAL),
    ("steps", 33, fqt.FQT_E_INVAL), ("eps", 0.0, fqt.FQT_E_INVAL), ("eps", float("nan"), fqt.FQT_E_INVAL)])
def test_ortho_descriptor_refusals(field, value, status):
    d = dense.ortho_desc(8, 16)
    setattr(d, field, value)
    with pytest.raises(fqt.FqtError) as e:
        dense.fqt_ortho_workspace_size(d)
    assert e.value.status == status
    assert dense._lib.fqt_orthogonalize(d, FAKE, FAKE, FAKE, BIG, None) == status
    c = dense.fqt_muon_cfg(0.1, 0.9, 0.0, 1.0, 1)
    assert dense._lib.fqt_muon_step(d, c, FAKE, FAKE, FAKE, FAKE, BIG, None) == status


def test_ortho_size_limits():
    for rows, cols in ((65537, 65537), (1 << 22, 1 << 15)):
        with pytest.raises(fqt.FqtError) as e:
            dense.fqt_ortho_workspace_size(dense.ortho_desc(rows, cols))
        assert e.value.status == fqt.FQT_E_SHAPE


def test_ortho_pointer_refusals():
    o, s = dense._lib.fqt_orthogonalize, dense._lib.fqt_muon_step
    d = dense.ortho_desc(8, 16)
    need = dense.fqt_ortho_workspace_size(d)
    c = dense.fqt_muon_cfg(0.1, 0.9, 0.0, 1.0, 1)
    assert o(d, None, FAKE, FAKE, BIG, None) == fqt.FQT_E_NULL
    assert o(d, FAKE, None, FAKE, BIG, None) == fqt.FQT_E_NULL
    assert o(d, FAKE + 2, FAKE, FAKE, BIG, None) == fqt.FQT_E_ALIGN
    assert o(d, FAKE, FAKE, FAKE, need - 1, None) == fqt.FQT_E_WORKSPACE
    assert s(d, None, FAKE, FAKE, FAKE, FAKE, BIG, None) == fqt.FQT_E_NULL
    assert s(d, c, FAKE, None, FAKE, FAKE, BIG, None) == fqt.FQT_E_NULL
    assert s(d, c, FAKE, FAKE, FAKE, FAKE + 8, BIG, None) == fqt.FQT_E_ALIGN
    assert s(dense.ortho_desc(8, 16, o_dtype="bf16"), c, FAKE, FAKE, FAKE, FAKE, BIG,
             None) == fqt.FQT_E_DTYPE
    for field in ("lr", "momentum", "weight_decay", "scale"):
        bad = dense.fqt_muon_cfg(0.1, 0.9, 0.0, 1.0, 1)
        setattr(bad, field, float("nan"))
        assert s(d, bad, FAKE, FAKE, FAKE, FAKE, BIG, None) == fqt.FQT_E_INVAL


# ----------------------------------------------------------------------------- binding

def test_binding_rejects_mismatched_tensors_before_launch():
    bf, f32 = torch.bfloat16, torch.float32
    d = dense.norm_desc(4, 16, q_dtype="int8")
    x, g, y = torch.empty(4, 16, dtype=bf), torch.empty(16), torch.empty(4, 16, dtype=bf)
    with pytest.raises(ValueError, match="dtype"):
        dense.fqt_rmsnorm_forward(d, x.float(), g, y=y)
    with pytest.raises(ValueError, match="shape"):
        dense.fqt_rmsnorm_forward(d, x[:3], g, y=y)
    with pytest.raises(ValueError, match="strides"):
        dense.fqt_rmsnorm_forward(d, torch.empty(16, 4, dtype=bf).t(), g, y=y)
    with pytest.raises(ValueError, match="strides"):
        dense.fqt_rmsnorm_forward(d, torch.empty(1, 16, dtype=bf).expand(4, 16), g, y=y)
    with pytest.raises(ValueError, match="g: .*float32"):
        dense.fqt_rmsnorm_forward(d, x, g.to(bf), y=y)
    with pytest.raises(ValueError, match="come together"):
        dense.fqt_rmsnorm_forward(d, x, g, q=torch.empty(4, 16, dtype=torch.int8))
    with pytest.raises(ValueError, match="required"):
        dense.fqt_rmsnorm_forward(d, None, g)
    with pytest.raises(ValueError, match="device tensor"):
        dense.fqt_rmsnorm_forward(d, x, g, y=y)          # everything right, but host memory
    l = dense.linear_desc(4, 8, 16)
    w, yl, ws = torch.empty(8, 16, dtype=bf), torch.empty(4, 8, dtype=bf), torch.empty(256, dtype=torch.uint8)
    with pytest.raises(ValueError, match="shape"):
        dense.fqt_linear_forward(l, x, w.t(), yl, ws)
    with pytest.raises(ValueError, match="bias"):
        dense.fqt_linear_forward(l, x, w, yl, ws, bias=torch.empty(4))
    with pytest.raises(ValueError, match="device tensor"):
        dense.fqt_linear_forward(l, x, w, yl, ws)
    with pytest.raises(ValueError, match="unknown activation"):
        dense.linear_desc(4, 8, 16, act="tanh")
    with pytest.raises(ValueError, match="unsupported dtype"):
        dense.norm_desc(4, 16, x_dtype=torch.float16)
    o = dense.ortho_desc(4, 16)
    with pytest.raises(ValueError, match="m: dtype"):
        dense.fqt_muon_step(o, torch.empty(4, 16), torch.empty(4, 16), torch.empty(4, 16, dtype=bf), ws, lr=0.1)
    with pytest.raises(ValueError, match="device tensor"):
        dense.fqt_orthogonalize(o, torch.empty(4, 16, dtype=f32), torch.empty(4, 16), ws)
