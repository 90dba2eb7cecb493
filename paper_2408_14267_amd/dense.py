"""ctypes binding of the dense operators of libfqt (the C ABI declared in include/fqt_dense.h).

RMS norm of a residual sum with 8-bit codes, matrix product with bias, activation and residual in
its epilogue, their backward passes, and the Newton-Schulz orthogonalisation with the optimizer step
on it.  As in `fqt`, this is argument marshalling only: functions keep the C names, tensors are torch
tensors on the current HIP device, `stream` defaults to torch's current stream, and a non-zero status
raises FqtError.  Tensors are matrices [rows][cols] with unit stride along cols and the row stride of
the descriptor (its ld* fields, 0 for dense rows); every tensor is checked against the descriptor
before anything is launched.
"""
import ctypes
from ctypes import POINTER, Structure, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p

import torch

from . import fqt
from .fqt import FQT_BF16, FQT_F32, FqtError  # noqa: F401

FQT_I8, FQT_E4M3, FQT_NO_CODES = 2, 3, -1
FQT_ACT_NONE, FQT_ACT_RELU, FQT_ACT_GELU, FQT_ACT_SILU, FQT_ACT_HARDTANH = range(5)
FQT_MAX_LD = 1 << 22
ACTIVATIONS = {"none": FQT_ACT_NONE, "relu": FQT_ACT_RELU, "gelu": FQT_ACT_GELU,
               "silu": FQT_ACT_SILU, "hardtanh": FQT_ACT_HARDTANH}
EXPORTED = ("fqt_rmsnorm_forward", "fqt_norm_workspace_size", "fqt_rmsnorm_backward",
            "fqt_quantize_rows", "fqt_linear_plan", "fqt_linear_workspace_size",
            "fqt_linear_forward", "fqt_linear_backward", "fqt_ortho_plan",
            "fqt_ortho_workspace_size", "fqt_orthogonalize", "fqt_muon_step")
LINEAR_PRODUCTS, ORTHO_PRODUCTS = ("forward", "dx", "dw"), ("gram", "poly", "apply")

_CODES = {torch.float32: FQT_F32, "f32": FQT_F32, torch.bfloat16: FQT_BF16, "bf16": FQT_BF16,
          torch.int8: FQT_I8, "int8": FQT_I8, torch.float8_e4m3fn: FQT_E4M3, "e4m3": FQT_E4M3,
          None: FQT_NO_CODES}
_TORCH_OF = {FQT_F32: torch.float32, FQT_BF16: torch.bfloat16, FQT_I8: torch.int8,
             FQT_E4M3: torch.float8_e4m3fn}


def dtype_code(dt):
    if isinstance(dt, int):
        return dt
    if dt not in _CODES:
        raise ValueError(f"unsupported dtype {dt}")
    return _CODES[dt]


class fqt_norm_desc(Structure):
    _fields_ = [("rows", c_int64), ("cols", c_int64), ("ldx", c_int64), ("ldr", c_int64),
                ("ldh", c_int64), ("ldy", c_int64), ("ldq", c_int64), ("x_dtype", c_int32),
                ("y_dtype", c_int32), ("q_dtype", c_int32), ("eps", c_float)]


class fqt_linear_desc(Structure):
    _fields_ = [("M", c_int64), ("N", c_int64), ("K", c_int64), ("ldx", c_int64),
                ("ldw", c_int64), ("ldr", c_int64), ("ldy", c_int64), ("ldz", c_int64),
                ("lddx", c_int64), ("lddw", c_int64), ("x_dtype", c_int32), ("y_dtype", c_int32),
                ("dx_dtype", c_int32), ("dw_dtype", c_int32), ("act", c_int32)]


class fqt_ortho_desc(Structure):
    _fields_ = [("rows", c_int64), ("cols", c_int64), ("ldg", c_int64), ("ldo", c_int64),
                ("ldm", c_int64), ("g_dtype", c_int32), ("o_dtype", c_int32), ("steps", c_int32),
                ("eps", c_float)]


class fqt_muon_cfg(Structure):
    _fields_ = [("lr", c_float), ("momentum", c_float), ("weight_decay", c_float),
                ("scale", c_float), ("nesterov", c_int32)]


class fqt_product_plan(Structure):
    _fields_ = [("launches", c_int32), ("splits", c_int32), ("tile", c_int32 * 2),
                ("threads", c_int32 * 2), ("workgroups", c_int64 * 2)]


def _bind(lib):
    N, L, O, U, P = (POINTER(t) for t in (fqt_norm_desc, fqt_linear_desc, fqt_ortho_desc,
                                          fqt_muon_cfg, fqt_product_plan))
    p, size = c_void_p, POINTER(c_size_t)
    for name, args in {
            "fqt_rmsnorm_forward": [N] + [p] * 9,
            "fqt_norm_workspace_size": [N, size],
            "fqt_rmsnorm_backward": [N] + [p] * 8 + [c_size_t, p],
            "fqt_quantize_rows": [N] + [p] * 4,
            "fqt_linear_plan": [L, c_int32, P],
            "fqt_linear_workspace_size": [L, c_int32, size],
            "fqt_linear_forward": [L] + [p] * 9 + [c_size_t, p],
            "fqt_linear_backward": [L] + [p] * 10 + [c_size_t, p],
            "fqt_ortho_plan": [O, c_int32, P],
            "fqt_ortho_workspace_size": [O, size],
            "fqt_orthogonalize": [O] + [p] * 3 + [c_size_t, p],
            "fqt_muon_step": [O, U] + [p] * 4 + [c_size_t, p]}.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = c_int, args
    return lib


_lib = _bind(fqt._lib)


# ----------------------------------------------------------------------------- descriptors

def norm_desc(rows, cols, x_dtype=FQT_BF16, y_dtype=None, q_dtype=None, eps=1e-6, ldx=0, ldr=0,
              ldh=0, ldy=0, ldq=0):
    x = dtype_code(x_dtype)
    return fqt_norm_desc(rows, cols, ldx, ldr, ldh, ldy, ldq, x,
                         x if y_dtype is None else dtype_code(y_dtype), dtype_code(q_dtype), eps)


def linear_desc(M, N, K, x_dtype=FQT_BF16, y_dtype=FQT_BF16, act="none", dx_dtype=FQT_BF16,
                dw_dtype=FQT_BF16, ldx=0, ldw=0, ldr=0, ldy=0, ldz=0, lddx=0, lddw=0):
    if act not in ACTIVATIONS and not isinstance(act, int):
        raise ValueError(f"unknown activation {act!r}: {', '.join(ACTIVATIONS)}")
    return fqt_linear_desc(M, N, K, ldx, ldw, ldr, ldy, ldz, lddx, lddw, dtype_code(x_dtype),
                           dtype_code(y_dtype), dtype_code(dx_dtype), dtype_code(dw_dtype),
                           ACTIVATIONS.get(act, act))


def ortho_desc(rows, cols, g_dtype=FQT_F32, o_dtype=FQT_F32, steps=5, eps=1e-7, ldg=0, ldo=0,
               ldm=0):
    return fqt_ortho_desc(rows, cols, ldg, ldo, ldm, dtype_code(g_dtype), dtype_code(o_dtype),
                          steps, eps)


# ----------------------------------------------------------------------------- checks

def _matrix(where, name, t, dtype, rows, cols, ld, dev):
    """Raise unless t is the matrix that the descriptor describes, on device `dev` (a kernel would
    read or write outside it)."""
    dt = _TORCH_OF.get(dtype)
    if (t.dtype is dt and t.shape == (rows, cols) and t.get_device() == dev and
            (t.stride() == (ld, 1) if ld else t.is_contiguous())):
        return
    if t.dtype is not dt:
        raise ValueError(f"{where}: {name}: dtype {t.dtype} does not match the descriptor's {dt}")
    if t.shape != (rows, cols):
        raise ValueError(f"{where}: {name}: shape {tuple(t.shape)}, the descriptor has "
                         f"({rows}, {cols})")
    if (cols > 1 and t.stride(1) != 1) or (rows > 1 and t.stride(0) != (ld or cols)):
        raise ValueError(f"{where}: {name}: strides {t.stride()}, the descriptor has "
                         f"({ld or cols}, 1)")
    if t.get_device() != dev:
        raise ValueError(f"{where}: {name}: expected a device tensor on device {dev}, got one on "
                         f"{t.device}")


def _vector(where, name, t, n, dev):
    if t.dtype is torch.float32 and t.shape == (n,) and t.is_contiguous() and t.get_device() == dev:
        return
    if t.dtype is not torch.float32:
        raise ValueError(f"{where}: {name}: dtype {t.dtype}, float32 is needed")
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{where}: {name}: shape {tuple(t.shape)}, strides {t.stride()}: "
                         f"{n} contiguous elements are needed")
    raise ValueError(f"{where}: {name}: expected a device tensor on device {dev}, got one on "
                     f"{t.device}")


def _current(where, dev):
    """Raise unless `dev`, where all tensors of a call are, is the current HIP device."""
    if dev < 0:
        raise ValueError(f"{where}: expected device tensors")
    if dev != torch.cuda.current_device():
        raise ValueError(f"{where}: tensors on device {dev}, the current device is "
                         f"{torch.cuda.current_device()}")


def _required(where, **tensors):
    for name, t in tensors.items():
        if t is None:
            raise ValueError(f"{where}: {name}: a tensor is required")


def _workspace(where, ws, dev):
    if ws is None:
        raise ValueError(f"{where}: ws: a workspace is required")
    if ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError(f"{where}: ws: a contiguous workspace on device {dev} is needed, got one on "
                         f"{ws.device}")
    return ws.data_ptr(), ws.numel() * ws.element_size()


# torch's current device, without the initialisation check that a device tensor makes needless.
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream(stream, dev):
    """The stream's handle; dev is the current device."""
    if stream is None and fqt._raw_stream is not None:
        return fqt._raw_stream(dev)
    return fqt._stream(stream)


def _check(status, where):
    if status:
        raise FqtError(status, where)


# ----------------------------------------------------------------------------- RMS norm

def fqt_rmsnorm_forward(desc, x, g, residual=None, h=None, y=None, q=None, scale=None, rstd=None,
                        stream=None):
    where, R, C = "fqt_rmsnorm_forward", desc.rows, desc.cols
    if x is None or g is None:
        _required(where, x=x, g=g)
    dev = x.get_device()
    if (q is None) != (scale is None):
        raise ValueError(f"{where}: q and scale come together")
    _matrix(where, "x", x, desc.x_dtype, R, C, desc.ldx, dev)
    _vector(where, "g", g, C, dev)
    if residual is not None:
        _matrix(where, "residual", residual, desc.x_dtype, R, C, desc.ldr, dev)
    if h is not None:
        _matrix(where, "h", h, desc.x_dtype, R, C, desc.ldh, dev)
    if y is not None:
        _matrix(where, "y", y, desc.y_dtype, R, C, desc.ldy, dev)
    if q is not None:
        _matrix(where, "q", q, desc.q_dtype, R, C, desc.ldq, dev)
        _vector(where, "scale", scale, R, dev)
    if rstd is not None:
        _vector(where, "rstd", rstd, R, dev)
    if dev < 0 or dev != _device():
        _current(where, dev)
    _check(_lib.fqt_rmsnorm_forward(
        desc, x.data_ptr(), None if residual is None else residual.data_ptr(), g.data_ptr(),
        None if h is None else h.data_ptr(), None if y is None else y.data_ptr(),
        None if q is None else q.data_ptr(), None if scale is None else scale.data_ptr(),
        None if rstd is None else rstd.data_ptr(), _stream(stream, dev)), where)


def fqt_norm_workspace_size(desc):
    n = c_size_t()
    _check(_lib.fqt_norm_workspace_size(desc, ctypes.byref(n)), "fqt_norm_workspace_size")
    return n.value


def fqt_rmsnorm_backward(desc, h, g, rstd, dy, dx, dg, ws, dres=None, stream=None):
    where, R, C = "fqt_rmsnorm_backward", desc.rows, desc.cols
    if h is None or g is None or rstd is None or dy is None or dx is None or dg is None:
        _required(where, h=h, g=g, rstd=rstd, dy=dy, dx=dx, dg=dg)
    dev = h.get_device()
    _matrix(where, "h", h, desc.x_dtype, R, C, desc.ldh, dev)
    _vector(where, "g", g, C, dev)
    _vector(where, "rstd", rstd, R, dev)
    _matrix(where, "dy", dy, desc.y_dtype, R, C, desc.ldy, dev)
    _matrix(where, "dx", dx, desc.x_dtype, R, C, desc.ldx, dev)
    _vector(where, "dg", dg, C, dev)
    if dres is not None:
        _matrix(where, "dres", dres, desc.x_dtype, R, C, desc.ldr, dev)
    if dev < 0 or dev != _device():
        _current(where, dev)
    _check(_lib.fqt_rmsnorm_backward(
        desc, h.data_ptr(), g.data_ptr(), rstd.data_ptr(), dy.data_ptr(),
        None if dres is None else dres.data_ptr(), dx.data_ptr(), dg.data_ptr(),
        *_workspace(where, ws, dev), _stream(stream, dev)), where)


def fqt_quantize_rows(desc, x, q, scale, stream=None):
    where, R, C = "fqt_quantize_rows", desc.rows, desc.cols
    if x is None or q is None or scale is None:
        _required(where, x=x, q=q, scale=scale)
    dev = x.get_device()
    _matrix(where, "x", x, desc.x_dtype, R, C, desc.ldx, dev)
    _matrix(where, "q", q, desc.q_dtype, R, C, desc.ldq, dev)
    _vector(where, "scale", scale, R, dev)
    if dev < 0 or dev != _device():
        _current(where, dev)
    _check(_lib.fqt_quantize_rows(
        desc, x.data_ptr(), q.data_ptr(), scale.data_ptr(), _stream(stream, dev)), where)


# ----------------------------------------------------------------------------- linear

def _plan(fn, desc, product, products):
    if product not in products:
        raise ValueError(f"unknown product {product!r}: {', '.join(products)}")
    plan = fqt_product_plan()
    _check(fn(desc, products.index(product), ctypes.byref(plan)), fn.__name__)
    return plan


def fqt_linear_plan(desc, product="forward"):
    """The fqt_product_plan of "forward", "dx" or "dw" (host only)."""
    return _plan(_lib.fqt_linear_plan, desc, product, LINEAR_PRODUCTS)


def fqt_linear_workspace_size(desc, backward=False):
    n = c_size_t()
    _check(_lib.fqt_linear_workspace_size(desc, int(backward), ctypes.byref(n)),
           "fqt_linear_workspace_size")
    return n.value


def _operands(where, desc, x, w, x_scale, w_scale, dev):
    if x is not None:
        _matrix(where, "x", x, desc.x_dtype, desc.M, desc.K, desc.ldx, dev)
    if w is not None:
        _matrix(where, "w", w, desc.x_dtype, desc.N, desc.K, desc.ldw, dev)
    if x_scale is not None:
        _vector(where, "x_scale", x_scale, desc.M, dev)
    if w_scale is not None:
        _vector(where, "w_scale", w_scale, desc.N, dev)


def fqt_linear_forward(desc, x, w, y, ws, bias=None, residual=None, x_scale=None, w_scale=None,
                       z=None, stream=None):
    where, M, N = "fqt_linear_forward", desc.M, desc.N
    if x is None or w is None or y is None:
        _required(where, x=x, w=w, y=y)
    dev = y.get_device()
    _operands(where, desc, x, w, x_scale, w_scale, dev)
    _matrix(where, "y", y, desc.y_dtype, M, N, desc.ldy, dev)
    if bias is not None:
        _vector(where, "bias", bias, N, dev)
    if residual is not None:
        _matrix(where, "residual", residual, desc.y_dtype, M, N, desc.ldr, dev)
    if z is not None:
        _matrix(where, "z", z, desc.y_dtype, M, N, desc.ldz, dev)
    if dev < 0 or dev != _device():
        _current(where, dev)
    _check(_lib.fqt_linear_forward(
        desc, x.data_ptr(), w.data_ptr(), None if x_scale is None else x_scale.data_ptr(),
        None if w_scale is None else w_scale.data_ptr(), None if bias is None else bias.data_ptr(),
        None if residual is None else residual.data_ptr(), None if z is None else z.data_ptr(),
        y.data_ptr(), *_workspace(where, ws, dev), _stream(stream, dev)), where)


def fqt_linear_backward(desc, x, w, dy, ws, z=None, x_scale=None, w_scale=None, dx=None, dw=None,
                        dbias=None, stream=None):
    where, M, N, K = "fqt_linear_backward", desc.M, desc.N, desc.K
    if dy is None:
        _required(where, dy=dy)
    dev = dy.get_device()
    _operands(where, desc, x, w, x_scale, w_scale, dev)
    _matrix(where, "dy", dy, desc.y_dtype, M, N, desc.ldy, dev)
    if z is not None:
        _matrix(where, "z", z, desc.y_dtype, M, N, desc.ldz, dev)
    if dx is not None:
        _matrix(where, "dx", dx, desc.dx_dtype, M, K, desc.lddx, dev)
    if dw is not None:
        _matrix(where, "dw", dw, desc.dw_dtype, N, K, desc.lddw, dev)
    if dbias is not None:
        _vector(where, "dbias", dbias, N, dev)
    if dev < 0 or dev != _device():
        _current(where, dev)
    _check(_lib.fqt_linear_backward(
        desc, None if x is None else x.data_ptr(), None if w is None else w.data_ptr(),
        None if x_scale is None else x_scale.data_ptr(),
        None if w_scale is None else w_scale.data_ptr(), None if z is None else z.data_ptr(),
        dy.data_ptr(), None if dx is None else dx.data_ptr(), None if dw is None else dw.data_ptr(),
        None if dbias is None else dbias.data_ptr(), *_workspace(where, ws, dev),
        _stream(stream, dev)), where)


# ----------------------------------------------------------------------------- orthogonalisation

def fqt_ortho_plan(desc, product):
    """The fqt_product_plan of "gram", "poly" or "apply" (host only)."""
    return _plan(_lib.fqt_ortho_plan, desc, product, ORTHO_PRODUCTS)


def fqt_ortho_workspace_size(desc):
    n = c_size_t()
    _check(_lib.fqt_ortho_workspace_size(desc, ctypes.byref(n)), "fqt_ortho_workspace_size")
    return n.value


def fqt_orthogonalize(desc, g, o, ws, stream=None):
    where, R, C = "fqt_orthogonalize", desc.rows, desc.cols
    if g is None or o is None:
        _required(where, g=g, o=o)
    dev = g.get_device()
    _matrix(where, "g", g, desc.g_dtype, R, C, desc.ldg, dev)
    _matrix(where, "o", o, desc.o_dtype, R, C, desc.ldo, dev)
    if dev < 0 or dev != _device():
        _current(where, dev)
    _check(_lib.fqt_orthogonalize(
        desc, g.data_ptr(), o.data_ptr(), *_workspace(where, ws, dev), _stream(stream, dev)), where)


def fqt_muon_step(desc, w, g, m, ws, lr, momentum=0.95, weight_decay=0.0, scale=1.0, nesterov=True,
                  stream=None):
    where, R, C = "fqt_muon_step", desc.rows, desc.cols
    if w is None or g is None or m is None:
        _required(where, w=w, g=g, m=m)
    dev = w.get_device()
    _matrix(where, "g", g, desc.g_dtype, R, C, desc.ldg, dev)
    _matrix(where, "m", m, FQT_F32, R, C, desc.ldm, dev)
    _matrix(where, "w", w, desc.o_dtype, R, C, desc.ldo, dev)
    cfg = fqt_muon_cfg(lr, momentum, weight_decay, scale, int(nesterov))
    if dev < 0 or dev != _device():
        _current(where, dev)
    _check(_lib.fqt_muon_step(
        desc, cfg, g.data_ptr(), m.data_ptr(), w.data_ptr(), *_workspace(where, ws, dev),
        _stream(stream, dev)), where)


# ----------------------------------------------------------------------------- workspaces

def _bytes(n, device):
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device)


def norm_workspace(desc, device="cuda"):
    """The workspace of fqt_rmsnorm_backward."""
    return _bytes(fqt_norm_workspace_size(desc), device)


def linear_workspace(desc, backward=False, device="cuda"):
    """The workspace of fqt_linear_forward, or of fqt_linear_backward."""
    return _bytes(fqt_linear_workspace_size(desc, backward), device)


def ortho_workspace(desc, device="cuda"):
    """The workspace of fqt_orthogonalize and fqt_muon_step."""
    return _bytes(fqt_ortho_workspace_size(desc), device)
