"""ctypes binding of the operators around a training step (the C ABI declared in include/fqt_step.h).

Softmax cross entropy of a linear layer without its outputs, its gradients, the norm of all gradients, and AdamW
over a list of tensors with states in float32 or 8 bits.  As in `dense`, this is argument marshalling only:
functions keep the C names, tensors are torch tensors on the current HIP device, `stream` defaults to torch's
current stream, every tensor is checked against its descriptor before anything is launched, and a non-zero
status raises FqtError.

A ParamList (param_list) holds the tensors of a list and their descriptors, checked once when it is made; a
program makes it once and passes it to every step.  set_gradients puts other gradients in.
"""
import ctypes
from ctypes import POINTER, Structure, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_uint64, c_void_p

import torch

from . import fqt
from .dense import (_bytes, _check, _current, _device, _matrix, _required, _stream, _vector, _workspace, dtype_code)
from .fqt import FQT_BF16, FQT_F32, FqtError  # noqa: F401

FQT_STATE_BLOCK, FQT_MAX_PARAMS = 256, 65536
EXPORTED = ("fqt_loss_workspace_size", "fqt_loss_forward", "fqt_loss_backward", "fqt_loss_forward_logp",
            "fqt_loss_backward_logp", "fqt_grad_norm_workspace_size", "fqt_grad_norm", "fqt_adamw_step")


class fqt_loss_desc(Structure):
    _fields_ = [("M", c_int64), ("N", c_int64), ("K", c_int64), ("ldx", c_int64), ("ldw", c_int64),
                ("lddx", c_int64), ("lddw", c_int64), ("ignore", c_int64), ("x_dtype", c_int32),
                ("dx_dtype", c_int32), ("dw_dtype", c_int32), ("smoothing", c_float)]


class fqt_param(Structure):
    _fields_ = [("g", c_void_p), ("p", c_void_p), ("m", c_void_p), ("v", c_void_p), ("m_scale", c_void_p),
                ("v_scale", c_void_p), ("n", c_int64), ("first", c_int64), ("g_dtype", c_int32)]


class fqt_adamw_cfg(Structure):
    _fields_ = [("lr", c_double), ("beta1", c_double), ("beta2", c_double), ("eps", c_double),
                ("weight_decay", c_double), ("seed", c_uint64), ("state_dtype", c_int32)]


def _bind(lib):
    L, T, A = (POINTER(t) for t in (fqt_loss_desc, fqt_param, fqt_adamw_cfg))
    p, size = c_void_p, POINTER(c_size_t)
    for name, args in {
            "fqt_loss_workspace_size": [L, c_int32, size],
            "fqt_loss_forward": [L] + [p] * 10 + [c_size_t, p],
            "fqt_loss_backward": [L] + [p] * 14 + [c_size_t, p],
            "fqt_loss_forward_logp": [L] + [p] * 11 + [c_size_t, p],
            "fqt_loss_backward_logp": [L] + [p] * 15 + [c_size_t, p],
            "fqt_grad_norm_workspace_size": [T, c_int32, size],
            "fqt_grad_norm": [T, c_int32, c_float, p, p, c_size_t, p],
            "fqt_adamw_step": [A, T, c_int32, c_int64, p, p, p]}.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = c_int, args
    return lib


_lib = _bind(fqt._lib)


def _ptr(t):
    return None if t is None else t.data_ptr()


# ----------------------------------------------------------------------------- loss of a linear layer

def loss_desc(M, N, K, x_dtype=FQT_BF16, dx_dtype=FQT_BF16, dw_dtype=FQT_BF16, smoothing=0.0, ignore=-100, ldx=0,
              ldw=0, lddx=0, lddw=0):
    return fqt_loss_desc(M, N, K, ldx, ldw, lddx, lddw, ignore, dtype_code(x_dtype), dtype_code(dx_dtype),
                         dtype_code(dw_dtype), smoothing)


def fqt_loss_workspace_size(desc, backward=False):
    n = c_size_t()
    _check(_lib.fqt_loss_workspace_size(desc, int(backward), ctypes.byref(n)), "fqt_loss_workspace_size")
    return n.value


def loss_workspace(desc, backward=False, device="cuda"):
    """The workspace of fqt_loss_forward, or of fqt_loss_backward."""
    return _bytes(fqt_loss_workspace_size(desc, backward), device)


def _loss_inputs(where, desc, x, w, target, bias, x_scale, w_scale, dev):
    M, N, K = desc.M, desc.N, desc.K
    _matrix(where, "x", x, desc.x_dtype, M, K, desc.ldx, dev)
    _matrix(where, "w", w, desc.x_dtype, N, K, desc.ldw, dev)
    if target.dtype is not torch.int64 or target.shape != (M,) or not target.is_contiguous():
        raise ValueError(f"{where}: target: {target.dtype} {tuple(target.shape)}, strides {target.stride()}: {M} "
                         f"contiguous int64 are needed")
    if target.get_device() != dev:
        raise ValueError(f"{where}: target: expected a device tensor on device {dev}, got one on {target.device}")
    if bias is not None:
        _vector(where, "bias", bias, N, dev)
    if x_scale is not None:
        _vector(where, "x_scale", x_scale, M, dev)
    if w_scale is not None:
        _vector(where, "w_scale", w_scale, N, dev)


def fqt_loss_forward(desc, x, w, target, loss, lse, ws, bias=None, x_scale=None, w_scale=None, mean=None, stream=None,
                     logp=None):
    """logp: log p of the targets, for the backward (fqt_loss_forward_logp)."""
    where = "fqt_loss_forward"
    if x is None or w is None or target is None or loss is None or lse is None:
        _required(where, x=x, w=w, target=target, loss=loss, lse=lse)
    dev = x.get_device()
    _loss_inputs(where, desc, x, w, target, bias, x_scale, w_scale, dev)
    _vector(where, "loss", loss, desc.M, dev)
    _vector(where, "lse", lse, desc.M, dev)
    if mean is not None:
        _vector(where, "mean", mean, 2, dev)
    if logp is not None:
        _vector(where, "logp", logp, desc.M, dev)
    if dev < 0 or dev != _device():
        _current(where, dev)
    _check(_lib.fqt_loss_forward_logp(
        desc, x.data_ptr(), w.data_ptr(), _ptr(x_scale), _ptr(w_scale), _ptr(bias), target.data_ptr(),
        loss.data_ptr(), lse.data_ptr(), _ptr(logp), _ptr(mean), *_workspace(where, ws, dev),
        _stream(stream, dev)), where)


def fqt_loss_backward(desc, x, w, target, lse, ws, dloss=None, dmean=None, mean=None, bias=None, x_scale=None,
                      w_scale=None, dx=None, dw=None, dbias=None, stream=None, logp=None):
    """logp: as the forward left it (fqt_loss_backward_logp)."""
    where = "fqt_loss_backward"
    if x is None or w is None or target is None or lse is None:
        _required(where, x=x, w=w, target=target, lse=lse)
    if (dloss is None) == (dmean is None) or (dmean is None) != (mean is None):
        raise ValueError(f"{where}: either dloss, or dmean and mean")
    dev = x.get_device()
    M, N, K = desc.M, desc.N, desc.K
    _loss_inputs(where, desc, x, w, target, bias, x_scale, w_scale, dev)
    _vector(where, "lse", lse, M, dev)
    if logp is not None:
        _vector(where, "logp", logp, M, dev)
    if dloss is not None:
        _vector(where, "dloss", dloss, M, dev)
    else:
        _vector(where, "dmean", dmean, 1, dev)
        _vector(where, "mean", mean, 2, dev)
    if dx is not None:
        _matrix(where, "dx", dx, desc.dx_dtype, M, K, desc.lddx, dev)
    if dw is not None:
        _matrix(where, "dw", dw, desc.dw_dtype, N, K, desc.lddw, dev)
    if dbias is not None:
        _vector(where, "dbias", dbias, N, dev)
    if dev < 0 or dev != _device():
        _current(where, dev)
    _check(_lib.fqt_loss_backward_logp(
        desc, x.data_ptr(), w.data_ptr(), _ptr(x_scale), _ptr(w_scale), _ptr(bias), target.data_ptr(),
        lse.data_ptr(), _ptr(logp), _ptr(dloss), _ptr(dmean), _ptr(mean), _ptr(dx), _ptr(dw), _ptr(dbias),
        *_workspace(where, ws, dev), _stream(stream, dev)), where)


# ----------------------------------------------------------------------------- lists of tensors

class ParamList:
    """The descriptors of a list of tensors, and the tensors (so that they live as long)."""

    def __init__(self, array, tensors, device, states):
        self.array, self.tensors, self.device, self.states = array, tensors, device, states
        self.count = len(array)
        self.sizes = [d.n for d in array]

    def set_gradients(self, g):
        """Other gradients for the same tensors: of their sizes, float32 or bfloat16, contiguous."""
        if len(g) != self.count:
            raise ValueError(f"set_gradients: {len(g)} gradients for {self.count} tensors")
        f32, bf16, device = torch.float32, torch.bfloat16, self.device
        for i, (t, n) in enumerate(zip(g, self.sizes)):
            if not ((t.dtype is f32 or t.dtype is bf16) and t.numel() == n and t.is_contiguous() and
                    t.get_device() == device):
                _flat("set_gradients", f"g[{i}]", t, (f32, bf16), n, device)
        for d, t in zip(self.array, g):
            d.g, d.g_dtype = t.data_ptr(), FQT_F32 if t.dtype is f32 else FQT_BF16
        self.tensors["g"] = list(g)

    def drop_gradients(self):
        """Forgets the gradients, whose memory may then be used again; others have to be set before the next call."""
        for d in self.array:
            d.g = None
        self.tensors["g"] = []


def _flat(where, name, t, dtypes, n, dev):
    if t.dtype not in dtypes:
        raise ValueError(f"{where}: {name}: dtype {t.dtype}, {' or '.join(str(d) for d in dtypes)} is needed")
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{where}: {name}: shape {tuple(t.shape)}, strides {t.stride()}: {n} contiguous elements "
                         f"are needed")
    if dev < 0 or t.get_device() != dev:
        raise ValueError(f"{where}: {name}: expected a device tensor on device {max(dev, 0)}, got one on {t.device}")


def param_list(g, p=None, m=None, v=None, m_scale=None, v_scale=None, first=None):
    """The ParamList of gradients g (float32 or bfloat16) and, for fqt_adamw_step, weights p (float32) with
    their states m and v: float32, or float8_e4m3fn with the scales of their blocks.  first: the place of each tensor in the
    random sequence (multiples of 4), one after the other by default."""
    where = "param_list"
    lists = dict(p=p, m=m, v=v, m_scale=m_scale, v_scale=v_scale, first=first)
    for name, t in lists.items():
        if t is not None and len(t) != len(g):
            raise ValueError(f"{where}: {len(t)} of {name}, {len(g)} gradients")
    if (p is None) != (m is None) or (p is None) != (v is None):
        raise ValueError(f"{where}: p, m and v come together")
    if (m_scale is None) != (v_scale is None) or (m_scale is not None and m is None):
        raise ValueError(f"{where}: m_scale and v_scale come together, with m and v")
    if len(g) > FQT_MAX_PARAMS:
        raise ValueError(f"{where}: {len(g)} tensors, at most {FQT_MAX_PARAMS}")
    states = None if m is None else FQT_F32 if m_scale is None else dtype_code("e4m3")
    kind = (torch.float32,) if m_scale is None else (torch.float8_e4m3fn,)
    dev = g[0].get_device() if g else 0
    array = (fqt_param * len(g))()
    at, ranges = 0, []
    for i, t in enumerate(g):
        n = t.numel()
        _flat(where, f"g[{i}]", t, (torch.float32, torch.bfloat16), n, dev)
        array[i].g, array[i].g_dtype, array[i].n = t.data_ptr(), FQT_F32 if t.dtype is torch.float32 else FQT_BF16, n
        if p is not None:
            blocks = -(-n // FQT_STATE_BLOCK)
            for name, dtypes, count in (("p", (torch.float32,), n), ("m", kind, n), ("v", kind, n),
                                        ("m_scale", (torch.float32,), blocks), ("v_scale", (torch.float32,), blocks)):
                if lists[name] is None:
                    continue
                o = lists[name][i]
                _flat(where, f"{name}[{i}]", o, dtypes, count, dev)
                setattr(array[i], name, o.data_ptr())
                if count:
                    ranges.append((o.data_ptr(), o.data_ptr() + count * o.element_size(), f"{name}[{i}]"))
        array[i].first = at if first is None else first[i]
        at += -(-n // FQT_STATE_BLOCK) * FQT_STATE_BLOCK
    ranges.sort()
    for (_, end, a), (begin, _, b) in zip(ranges, ranges[1:]):
        if begin < end:
            raise ValueError(f"{where}: {a} and {b} overlap")
    tensors = {"g": list(g), **{k: list(t) for k, t in lists.items() if t is not None and k != "first"}}
    return ParamList(array, tensors, dev, states)


def joined(lists):
    """The gradients of several lists on one device as a ParamList for fqt_grad_norm, until theirs change."""
    if len(lists) == 1:
        return lists[0]
    array, at = (fqt_param * sum(p.count for p in lists))(), 0
    for p in lists:
        if p.device != lists[0].device:
            raise ValueError(f"joined: lists on devices {lists[0].device} and {p.device}")
        ctypes.memmove(ctypes.byref(array, at * ctypes.sizeof(fqt_param)), p.array, ctypes.sizeof(p.array))
        at += p.count
    return ParamList(array, {"g": [t for p in lists for t in p.tensors["g"]]}, lists[0].device, None)


def fqt_grad_norm_workspace_size(params):
    n = c_size_t()
    _check(_lib.fqt_grad_norm_workspace_size(params.array, params.count, ctypes.byref(n)),
           "fqt_grad_norm_workspace_size")
    return n.value


def grad_norm_workspace(params, device="cuda"):
    """The workspace of fqt_grad_norm."""
    return _bytes(fqt_grad_norm_workspace_size(params), device)


def fqt_grad_norm(params, out, ws, max_norm=float("inf"), stream=None):
    where = "fqt_grad_norm"
    if out is None:
        _required(where, out=out)
    dev = out.get_device()
    _vector(where, "out", out, 2, dev)
    if params.count and dev != params.device:
        raise ValueError(f"{where}: out on {out.device}, the tensors on device {params.device}")
    if dev < 0 or dev != _device():
        _current(where, dev)
    _check(_lib.fqt_grad_norm(params.array, params.count, max_norm, out.data_ptr(), *_workspace(where, ws, dev),
                              _stream(stream, dev)), where)


def adamw_cfg(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, seed=0, states="f32"):
    return fqt_adamw_cfg(lr, beta1, beta2, eps, weight_decay, seed, dtype_code(states))


def fqt_adamw_step(cfg, params, step, grad_scale=None, stream=None):
    """One step on every tensor of the list, in place.  step: the number of this step, from 1, or an int64
    tensor of one element on the device, which the kernels read (for captured graphs)."""
    where = "fqt_adamw_step"
    if params.states is None:
        raise ValueError(f"{where}: a list with p, m and v is needed")
    if params.states != cfg.state_dtype:
        raise ValueError(f"{where}: the list's states and the configuration's state_dtype differ")
    dev, number, at = params.device, 0, None
    if isinstance(step, torch.Tensor):
        if step.dtype is not torch.int64 or step.numel() != 1 or step.get_device() != dev:
            raise ValueError(f"{where}: step: one int64 on device {dev} is needed, got {step.numel()} {step.dtype} on "
                             f"{step.device}")
        at = step.data_ptr()
    else:
        number = step
    if grad_scale is not None:
        _vector(where, "grad_scale", grad_scale, 1, dev)
    if dev < 0 or dev != _device():
        _current(where, dev)
    _check(_lib.fqt_adamw_step(cfg, params.array, params.count, number, at, _ptr(grad_scale), _stream(stream, dev)),
           where)
