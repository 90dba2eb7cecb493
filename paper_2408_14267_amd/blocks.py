"""Residual blocks, a loss and optimizers around binary layers: torch modules over the dense operators.

RMSNorm, Linear and NormLinear call fqt_rmsnorm_*, fqt_quantize_rows and fqt_linear_* (forward and
backward); NormLinear keeps the activations between the norm and the product as 8-bit codes.  Muon
updates latent weight matrices (and convolution weights, unfolded) by fqt_muon_step.  Linear.loss is the softmax
cross entropy of a layer's outputs without computing them as a matrix (fqt_loss_*); AdamW updates all tensors of a model
by fqt_adamw_step, with states in float32 or 8 bits, clipped by fqt_grad_norm.  ResidualMLP puts them together with
BinaryLinear: a float32 residual stream, blocks of a normed 8-bit expansion with GELU and a binary projection, the
first and last layers at full width as in the networks of `train`.

Modules take [..., features] inputs of float32 or bfloat16, keep float32 parameters, and cast or
quantize the weight in every forward pass.  Gradients come in the type of what they belong to (the products
of the backward take dz in bf16, as fqt_linear_backward says) and cannot be differentiated again.
"""
import math

import torch
import torch.nn as nn
from torch.autograd.function import once_differentiable

from . import dense, step, train

_BF16, _F32 = torch.bfloat16, torch.float32


def _workspace(size, device):
    """A call's workspace, from torch's allocator for that call alone: the calls of a stream take the same
    memory one after the other, those of other streams, threads and graphs (a capture's comes from the
    graph's pool) never, and nothing is held between calls."""
    return torch.empty(max(size, 1), dtype=torch.uint8, device=device)


def _rows(t, cols, name):
    """t as a matrix [rows][cols]: dense rows on 16 bytes."""
    if t.dtype not in (_F32, _BF16) or t.shape[-1] != cols:
        raise ValueError(f"{name}: float32 or bfloat16 with {cols} features is needed, got "
                         f"{t.dtype} {tuple(t.shape)}")
    t = t.reshape(-1, cols).contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class _NormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, g, mod):
        rows, cols = x.shape
        desc = dense.norm_desc(rows, cols, x_dtype=x.dtype, y_dtype=mod.out_dtype or x.dtype, eps=mod.eps)
        h = torch.empty_like(x) if residual is not None else x
        y = torch.empty(rows, cols, dtype=mod.out_dtype or x.dtype, device=x.device)
        rstd = torch.empty(rows, device=x.device)
        dense.fqt_rmsnorm_forward(desc, x, g, residual=residual, h=h if residual is not None else None,
                                  y=y, rstd=rstd)
        ctx.save_for_backward(h, g, rstd)
        ctx.desc, ctx.residual = desc, residual is not None
        return (y, h) if ctx.residual else y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh=None):
        h, g, rstd = ctx.saved_tensors
        desc = ctx.desc
        dx, dg = torch.empty_like(h), torch.empty_like(g)
        ws = _workspace(dense.fqt_norm_workspace_size(desc), h.device)
        dense.fqt_rmsnorm_backward(desc, h, g, rstd, dy.contiguous(), dx, dg, ws,
                                   dres=dh.contiguous() if ctx.residual else None)
        return dx, dx if ctx.residual else None, dg, None


class RMSNorm(nn.Module):
    """y = h / sqrt(mean h^2 + eps) * weight for h = x + residual; forward(x) returns y, forward(x,
    residual) returns (y, h)."""

    def __init__(self, features, eps=1e-6, out_dtype=None):
        super().__init__()
        self.weight = nn.Parameter(torch.ones(features))
        self.features, self.eps, self.out_dtype = features, eps, out_dtype

    def forward(self, x, residual=None):
        m = _rows(x, self.features, "x")
        r = None if residual is None else _rows(residual, self.features, "residual").to(m.dtype)
        if r is None:
            return _NormFn.apply(m, None, self.weight, self).view(x.shape)
        y, h = _NormFn.apply(m, r, self.weight, self)
        return y.view(x.shape), h.view(x.shape)


def _quantized(w, kind):
    """Codes and scales of a matrix's rows, or its bf16 copy."""
    w = w.contiguous()
    if kind == "bf16":
        return w.to(_BF16), None
    q = torch.empty(w.shape, dtype=dense._TORCH_OF[dense.dtype_code(kind)], device=w.device)
    scale = torch.empty(w.shape[0], device=w.device)
    dense.fqt_quantize_rows(dense.norm_desc(*w.shape, x_dtype=w.dtype, q_dtype=kind), w, q, scale)
    return q, scale


def _linear_forward(mod, x, x_scale, w, bias, residual, out_dtype, stream_dtype):
    """y, the pre-activation (None without an activation), the operand form of w, and the descriptor.
    stream_dtype: the type of the module's input, which its gradient has."""
    (M, K), N = x.shape, w.shape[0]
    wq, w_scale = _quantized(w, mod.operands)
    desc = dense.linear_desc(M, N, K, x_dtype=mod.operands, y_dtype=out_dtype, act=mod.act,
                             dx_dtype=stream_dtype, dw_dtype=_F32)
    y = torch.empty(M, N, dtype=out_dtype, device=x.device)
    z = torch.empty_like(y) if mod.act != "none" else None
    ws = _workspace(dense.fqt_linear_workspace_size(desc), x.device)
    dense.fqt_linear_forward(desc, x, wq, y, ws, bias=bias, residual=residual, x_scale=x_scale,
                             w_scale=w_scale, z=z)
    return y, z, wq, w_scale, desc


def _linear_backward(desc, x, x_scale, wq, w_scale, z, dy, need_x, need_w, need_bias):
    """The gradients that are needed, None for the others."""
    dy = dy.contiguous()
    dx = torch.empty(desc.M, desc.K, dtype=dense._TORCH_OF[desc.dx_dtype], device=dy.device) if need_x else None
    dw = torch.empty(desc.N, desc.K, device=dy.device) if need_w else None
    db = torch.empty(desc.N, device=dy.device) if need_bias else None
    ws = _workspace(dense.fqt_linear_workspace_size(desc, True), dy.device)
    dense.fqt_linear_backward(desc, x, wq, dy, ws, z=z, x_scale=x_scale, w_scale=w_scale, dx=dx, dw=dw,
                              dbias=db)
    return dx, dw, db


class _LinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, w, bias, mod):
        xq, x_scale = _quantized(x, mod.operands)
        y, z, wq, w_scale, desc = _linear_forward(mod, xq, x_scale, w, bias, residual,
                                                  residual.dtype if residual is not None else x.dtype, x.dtype)
        ctx.save_for_backward(xq, x_scale, wq, w_scale, z)
        ctx.desc, ctx.residual = desc, residual is not None
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        xq, x_scale, wq, w_scale, z = ctx.saved_tensors
        need_x, _, need_w, need_bias, _ = ctx.needs_input_grad
        dx, dw, db = _linear_backward(ctx.desc, xq, x_scale, wq, w_scale, z, dy, need_x, need_w, need_bias)
        return dx, (dy if ctx.residual else None), dw, db, None


class _LossFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, target, mod, smoothing, ignore, mean):
        (M, K), N = x.shape, w.shape[0]
        xq, x_scale = _quantized(x, mod.operands)
        wq, w_scale = _quantized(w, mod.operands)
        desc = step.loss_desc(M, N, K, x_dtype=mod.operands, dx_dtype=x.dtype, dw_dtype=_F32, smoothing=smoothing,
                              ignore=ignore)
        loss, lse, logp = (torch.empty(M, device=x.device) for _ in range(3))
        average = torch.empty(2, device=x.device) if mean else None
        step.fqt_loss_forward(desc, xq, wq, target, loss, lse, _workspace(step.fqt_loss_workspace_size(desc), x.device),
                              bias=bias, x_scale=x_scale, w_scale=w_scale, mean=average, logp=logp)
        ctx.save_for_backward(xq, x_scale, wq, w_scale, bias, target, lse, logp, average)
        ctx.desc = desc
        return average[0].clone() if mean else loss

    @staticmethod
    @once_differentiable
    def backward(ctx, d):
        xq, x_scale, wq, w_scale, bias, target, lse, logp, average = ctx.saved_tensors
        desc, (need_x, need_w, need_bias) = ctx.desc, ctx.needs_input_grad[:3]
        dx = torch.empty(desc.M, desc.K, dtype=dense._TORCH_OF[desc.dx_dtype], device=d.device) if need_x else None
        dw = torch.empty(desc.N, desc.K, device=d.device) if need_w else None
        db = torch.empty(desc.N, device=d.device) if need_bias else None
        given = dict(dloss=d.contiguous()) if average is None else dict(dmean=d.reshape(1), mean=average)
        ws = _workspace(step.fqt_loss_workspace_size(desc, True), d.device)
        step.fqt_loss_backward(desc, xq, wq, target, lse, ws, bias=bias, x_scale=x_scale, w_scale=w_scale, dx=dx, dw=dw,
                               dbias=db, logp=logp, **given)
        return dx, dw, db, None, None, None, None, None


class Linear(nn.Module):
    """act(x W^T + bias) + residual with bf16, int8 or e4m3 operands (quantized per row, gradients passed
    through the rounding)."""

    def __init__(self, fin, fout, bias=True, act="none", operands="bf16"):
        super().__init__()
        dense.linear_desc(1, fout, fin, x_dtype=operands, act=act)       # refuses what does not exist
        self.weight = nn.Parameter(torch.empty(fout, fin))
        nn.init.kaiming_uniform_(self.weight, a=5 ** 0.5)
        self.bias = nn.Parameter(torch.zeros(fout)) if bias else None
        self.fin, self.fout, self.act, self.operands = fin, fout, act, operands

    def forward(self, x, residual=None):
        r = None if residual is None else _rows(residual, self.fout, "residual")
        y = _LinearFn.apply(_rows(x, self.fin, "x"), r, self.weight, self.bias, self)
        return y.view(*x.shape[:-1], self.fout)

    def loss(self, x, target, smoothing=0.0, ignore=-100, reduction="mean"):
        """The softmax cross entropy of this layer's outputs for x against class numbers (int64, of x's shape
        without its last dimension), without computing the outputs as a matrix.  Rows whose target is `ignore` are left
        out; any other target that is no class gives NaN.  reduction: "mean" over the rows that count (0 if none
        does) or "none"."""
        if self.act != "none":
            raise ValueError(f"loss: the outputs of a layer with activation {self.act} are no logits")
        if reduction not in ("mean", "none"):
            raise ValueError(f"loss: unknown reduction {reduction!r}: mean, none")
        if target.dtype != torch.int64 or target.shape != x.shape[:-1] or target.device != x.device:
            raise ValueError(f"loss: target: int64 {tuple(x.shape[:-1])} on {x.device} is needed, got {target.dtype} "
                             f"{tuple(target.shape)} on {target.device}")
        y = _LossFn.apply(_rows(x, self.fin, "x"), self.weight, self.bias, target.reshape(-1).contiguous(), self,
                          smoothing, ignore, reduction == "mean")
        return y if reduction == "mean" else y.view(target.shape)


class _NormLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, g, w, bias, mod):
        rows, cols = x.shape
        kind = mod.operands
        desc = dense.norm_desc(rows, cols, x_dtype=x.dtype, y_dtype=_BF16,
                               q_dtype=None if kind == "bf16" else kind, eps=mod.eps)
        h = torch.empty_like(x) if residual is not None else x
        rstd = torch.empty(rows, device=x.device)
        out = dict(residual=residual, h=h if residual is not None else None, rstd=rstd)
        scale = None
        if kind == "bf16":
            n = torch.empty(rows, cols, dtype=_BF16, device=x.device)
            dense.fqt_rmsnorm_forward(desc, x, g, y=n, **out)
        else:
            n = torch.empty(rows, cols, dtype=dense._TORCH_OF[dense.dtype_code(kind)], device=x.device)
            scale = torch.empty(rows, device=x.device)
            dense.fqt_rmsnorm_forward(desc, x, g, q=n, scale=scale, **out)
        y, z, wq, w_scale, ldesc = _linear_forward(mod, n, scale, w, bias, None, mod.out_dtype, x.dtype)
        ctx.save_for_backward(h, g, rstd, n, scale, wq, w_scale, z)
        # (the norm's own y is the product's operand; its gradient has the stream's type)
        ctx.descs = dense.norm_desc(rows, cols, x_dtype=x.dtype, eps=mod.eps), ldesc
        ctx.residual = residual is not None
        return (y, h) if ctx.residual else y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh=None):
        h, g, rstd, n, scale, wq, w_scale, z = ctx.saved_tensors
        desc, ldesc = ctx.descs
        need_w, need_bias = ctx.needs_input_grad[3:5]
        need_norm = any(ctx.needs_input_grad[:3])
        dn, dw, db = _linear_backward(ldesc, n, scale, wq, w_scale, z, dy, need_norm, need_w, need_bias)
        if not need_norm:
            return None, None, None, dw, db, None
        dx, dg = torch.empty_like(h), torch.empty_like(g)
        ws = _workspace(dense.fqt_norm_workspace_size(desc), h.device)
        dense.fqt_rmsnorm_backward(desc, h, g, rstd, dn, dx, dg, ws,
                                   dres=dh.contiguous() if ctx.residual else None)
        return dx, dx if ctx.residual else None, dg, dw, db, None


class NormLinear(nn.Module):
    """act(norm(x + residual) W^T + bias), the normed rows as 8-bit codes (operands "int8" or "e4m3") or
    bf16.  forward(x) returns y, forward(x, residual) returns (y, h) with h = x + residual."""

    def __init__(self, fin, fout, bias=True, act="none", operands="int8", eps=1e-6, out_dtype=_F32):
        super().__init__()
        dense.linear_desc(1, fout, fin, x_dtype=operands, act=act)
        self.norm_weight = nn.Parameter(torch.ones(fin))
        self.weight = nn.Parameter(torch.empty(fout, fin))
        nn.init.kaiming_uniform_(self.weight, a=5 ** 0.5)
        self.bias = nn.Parameter(torch.zeros(fout)) if bias else None
        self.fin, self.fout, self.act, self.operands = fin, fout, act, operands
        self.eps, self.out_dtype = eps, out_dtype

    def forward(self, x, residual=None):
        m = _rows(x, self.fin, "x")
        r = None if residual is None else _rows(residual, self.fin, "residual").to(m.dtype)
        shape = (*x.shape[:-1], self.fout)
        if r is None:
            return _NormLinearFn.apply(m, None, self.norm_weight, self.weight, self.bias, self).view(shape)
        y, h = _NormLinearFn.apply(m, r, self.norm_weight, self.weight, self.bias, self)
        return y.view(shape), h.view(x.shape)


class Muon(torch.optim.Optimizer):
    """Orthogonalised momentum for float32 weights of two or more dimensions (a convolution's is unfolded to
    [out][in kh kw]): m = momentum m + g, u = g + momentum m (nesterov) or m, w = (1 - lr weight_decay) w
    - lr sqrt(max(1, rows / cols)) NS(u), one fqt_muon_step per weight.  Weights of another memory order
    (channels_last) are updated through a copy.  What cannot be updated is refused when its group is added or,
    where it has changed since, before a step updates anything."""

    def __init__(self, params, lr=0.02, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5, eps=1e-7):
        super().__init__(params, dict(lr=lr, momentum=momentum, weight_decay=weight_decay,
                                      nesterov=nesterov, steps=steps, eps=eps))

    def add_param_group(self, param_group):
        super().add_param_group(param_group)
        group = self.param_groups[-1]
        try:
            self._check_rates(group)
            for p in group["params"]:
                if p.dim() < 2 or p.dtype != _F32:
                    raise ValueError(f"Muon updates float32 matrices, got {p.dtype} {tuple(p.shape)}")
                dense.fqt_ortho_workspace_size(self._desc(p, group))     # refuses sizes, steps and eps
        except Exception:
            self.param_groups.pop()
            raise

    @staticmethod
    def _check_rates(group):
        lr, momentum, weight_decay = group["lr"], group["momentum"], group["weight_decay"]
        if not (0 <= lr < math.inf and 0 <= momentum < 1 and 0 <= weight_decay < math.inf):
            raise ValueError(f"lr {lr}, momentum {momentum}, weight_decay {weight_decay}: out of range")

    @staticmethod
    def _desc(p, group):
        return dense.ortho_desc(p.shape[0], math.prod(p.shape[1:]), steps=group["steps"], eps=group["eps"])

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        todo = []
        for group in self.param_groups:
            self._check_rates(group)
            for p in group["params"]:
                if p.grad is None or p.numel() == 0:
                    continue
                if p.grad.layout != torch.strided or p.device.type != "cuda" or \
                        p.device.index != torch.cuda.current_device():
                    raise ValueError(f"Muon updates weights with dense gradients on the current device, got "
                                     f"{p.grad.layout} on {p.device}")
                desc = self._desc(p, group)
                todo.append((group, p, desc, dense.fqt_ortho_workspace_size(desc)))
        for group, p, desc, size in todo:
            state = self.state[p]
            if "momentum" not in state:
                state["momentum"] = torch.zeros_like(p)
            held = p, state["momentum"]
            w, m = (t.contiguous() for t in held)
            shape = desc.rows, desc.cols
            dense.fqt_muon_step(desc, w.view(shape), p.grad.contiguous().view(shape), m.view(shape),
                                _workspace(size, p.device), lr=group["lr"], momentum=group["momentum"],
                                weight_decay=group["weight_decay"],
                                scale=math.sqrt(max(1.0, desc.rows / desc.cols)), nesterov=group["nesterov"])
            for t, dense_t in zip(held, (w, m)):
                if dense_t is not t:
                    t.copy_(dense_t)
        return loss


def _flat(t):
    """The elements of t in memory order, or None where they have gaps or overlap."""
    if t.numel() == 0:
        return t.detach().reshape(-1)
    expected = 1
    for stride, size in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n != 1):
        if stride != expected:
            return None
        expected *= size
    return t.detach().as_strided((t.numel(),), (1,))


def _same_order(p, strides):
    """Whether p's elements lie in memory as those of a tensor of its shape with these strides."""
    have = p.stride()
    return have == strides or (len(have) == len(strides) and
                               all(a == b or n == 1 for a, b, n in zip(have, strides, p.shape)))


_MOST = 1e30                   # of the settings of fqt_adamw_step, and of lr * weight_decay


class AdamW(torch.optim.Optimizer):
    """AdamW for float32 weights of any shape, all tensors of a group in one fqt_adamw_step.  states: "f32", or "e4m3"
    for 8-bit states, stochastically rounded with the random sequence of `seed` (2 bytes a weight instead of 8).
    max_norm: the gradients are clipped to this norm over all groups; `grad_norm` holds the last step's norm
    and factor (on the device).  capturable: the step number is counted on the device (one for each group, weights without a
    gradient included), so that step() may be captured into a graph; the learning rate is then the captured one, and a
    checkpoint is loaded before the capture.  A checkpoint of either kind goes on in the other: the states' step number becomes
    the group's counter (it has to be one number for the group's weights) or the other way.  States lie in memory as their weights do: those in float32 follow weights whose
    memory order has changed, 8-bit ones, whose blocks are of memory order, are refused then.
    What cannot be updated is refused when its group is added or before a step updates anything."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, states="f32", seed=0,
                 max_norm=None, capturable=False):
        if states not in ("f32", "e4m3"):
            raise ValueError(f"states {states!r}: f32, e4m3")
        if max_norm is not None and not max_norm > 0:
            raise ValueError(f"max_norm {max_norm}: out of range")
        self.states, self.seed, self.max_norm, self.capturable = states, seed, max_norm, capturable
        self.grad_norm = None
        self._lists = {}
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay))

    def add_param_group(self, param_group):
        super().add_param_group(param_group)
        group = self.param_groups[-1]
        try:
            self._config(group)
            for p in group["params"]:
                if p.dtype != _F32 or _flat(p) is None:
                    raise ValueError(f"AdamW updates float32 weights without gaps, got {p.dtype} {tuple(p.shape)}, "
                                     f"strides {p.stride()}")
        except Exception:
            self.param_groups.pop()
            raise

    def _config(self, group):
        lr, (beta1, beta2), eps, decay = group["lr"], group["betas"], group["eps"], group["weight_decay"]
        if not (0 <= lr <= _MOST and 0 <= beta1 < 1 and 0 <= beta2 < 1 and 0 <= eps <= _MOST and 0 <= decay <= _MOST and
                lr * decay <= _MOST):
            raise ValueError(f"lr {lr}, betas {group['betas']}, eps {eps}, weight_decay {decay}: out of range")
        return step.adamw_cfg(lr=lr, beta1=beta1, beta2=beta2, eps=eps, weight_decay=decay, seed=self.seed,
                              states=self.states)

    def _state(self, p):
        state = self.state[p]
        if "m" not in state:
            self._not_captured("states are made")
            state["step"] = 0
            if self.states == "f32":
                state["m"], state["v"] = torch.zeros_like(p), torch.zeros_like(p)
            else:
                blocks = -(-p.numel() // step.FQT_STATE_BLOCK)
                for name in ("m", "v"):
                    state[name] = torch.zeros(p.numel(), dtype=torch.float8_e4m3fn, device=p.device)
                    state[name + "_scale"] = torch.zeros(blocks, device=p.device)
                state["strides"] = p.stride()
        elif self.states == "f32":
            for name in ("m", "v"):
                if not _same_order(p, state[name].stride()):
                    self._not_captured("states are laid out again")
                    state[name] = torch.empty_like(p).copy_(state[name])
        return state

    def _check_state(self, p, state):
        if self.states == "f32":
            if state["m"].shape != p.shape or state["v"].shape != p.shape:
                raise ValueError(f"AdamW: states of shapes {tuple(state['m'].shape)}, {tuple(state['v'].shape)} for "
                                 f"weights of {tuple(p.shape)}")
        elif not _same_order(p, state["strides"]):
            raise ValueError(f"AdamW: 8-bit states of weights with strides {state['strides']}, got {p.stride()}")

    @staticmethod
    def _not_captured(what):
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError(f"AdamW: {what} in the first step: take one before a capture")

    def _clock(self, group, device):
        """The group's counter of steps on the device, made before the first one."""
        if group.get("clock") is None:
            self._not_captured("the step counter is made")
            group["clock"] = torch.zeros(1, dtype=torch.int64, device=device)
        if group["clock"].device != device:
            raise ValueError(f"AdamW: a step counter on {group['clock'].device}, weights on {device}")

    def _gradient(self, p, g, device):
        """g, the gradient of p, its elements in p's memory order.  device: the current one."""
        if (g.layout is not torch.strided or g.dtype not in (_F32, _BF16) or p.dtype is not _F32 or
                p.get_device() != device):
            raise ValueError(f"AdamW updates float32 weights with dense float32 or bfloat16 gradients on the current device, "
                             f"got {p.dtype} with {g.layout} {g.dtype} on {p.device}")
        if g.is_contiguous() and p.is_contiguous():
            return g
        if _flat(p) is None:
            raise ValueError(f"AdamW updates weights without gaps, got {tuple(p.shape)}, strides {p.stride()}")
        if g.stride() != p.stride():
            g = torch.empty_like(p, dtype=g.dtype).copy_(g)
        return g if g.is_contiguous() else _flat(g)

    def _list(self, key, params, starts):
        """The ParamList of some weights and their states, made again when any of them has moved."""
        at = self._lists.get(key)
        if at is None or any(p.data_ptr() != where or p.stride() != strides or self.state[p] is not s or
                             s["m"] is not m or s["v"] is not v
                             for p, (where, strides, s, m, v) in zip(params, at[0])):
            states = [self._state(p) for p in params]
            held = [(p.data_ptr(), p.stride(), s, s["m"], s["v"]) for p, s in zip(params, states)]
            flat = {k: [_flat(s[k]) for s in states] for k in ("m", "v")}
            for k in ("m_scale", "v_scale"):
                flat[k] = [s[k] for s in states] if self.states == "e4m3" else None
            weights = [_flat(p) for p in params]
            at = held, step.param_list(weights, weights, flat["m"], flat["v"], flat["m_scale"], flat["v_scale"],
                                       first=starts)
        return at

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        if not self.capturable and torch.cuda.is_available() and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("AdamW: a captured step would keep its number: make the optimizer capturable")
        # weights with a gradient, by group and by how many steps they have taken
        todo, at, device = {}, 0, dense._device() if torch.cuda.is_available() else None
        for i, group in enumerate(self.param_groups):
            cfg = self._config(group)
            for p in group["params"]:
                n, g = p.numel(), p.grad
                if g is not None and n:
                    g = self._gradient(p, g, device)
                    state = self.state.get(p)                # (none is made before all are checked)
                    if state:
                        self._check_state(p, state)
                    key = i, state["step"] if state and not self.capturable else 0
                    if key not in todo:
                        todo[key] = cfg, [], [], []
                    _, params, grads, starts = todo[key]
                    params.append(p)
                    grads.append(g)
                    starts.append(at)
                at += -(-n // step.FQT_STATE_BLOCK) * step.FQT_STATE_BLOCK
        if not todo:
            return loss
        lists, kept = [], {}
        for (i, t), (cfg, params, g, starts) in todo.items():
            key = i, tuple(starts)
            kept[key] = self._list(key, params, starts)
            params_list = kept[key][1]
            params_list.set_gradients(g)
            lists.append((i, t, cfg, params, params_list))
            if self.capturable:
                self._clock(self.param_groups[i], params[0].device)
        self._lists = kept                   # (those of this step: other sets of weights with gradients go)
        scale = None
        if self.max_norm is not None:
            whole = step.joined([at[4] for at in lists])
            if self.grad_norm is None:
                self.grad_norm = torch.empty(2, device=lists[0][3][0].device)
            step.fqt_grad_norm(whole, self.grad_norm, _workspace(step.fqt_grad_norm_workspace_size(whole),
                                                                 self.grad_norm.device), max_norm=self.max_norm)
            scale = self.grad_norm[1:]
        for i, t, cfg, params, params_list in lists:
            if self.capturable:
                number = self.param_groups[i]["clock"].add_(1)
            else:
                number = t + 1
                for p in params:
                    self.state[p]["step"] = number
            step.fqt_adamw_step(cfg, params_list, number, grad_scale=scale)
            params_list.drop_gradients()     # (their memory is free for the next backward pass)
        return loss

    def __getstate__(self):
        return {**super().__getstate__(), "states": self.states, "seed": self.seed, "max_norm": self.max_norm,
                "capturable": self.capturable, "grad_norm": None, "_lists": {}}

    def _steps_taken(self, group, states):
        """The number of steps that a saved group's weights have taken, from its counter or their states; None where it
        has no states, or where each state keeps its own."""
        if group.get("clock") is not None:
            return int(group["clock"])
        numbers = {states[i]["step"] for i in group["params"] if states.get(i)}
        if not self.capturable or not numbers:
            return None
        if len(numbers) > 1:
            raise ValueError(f"AdamW: weights of a group that have taken different numbers of steps, {sorted(numbers)}: a "
                             f"capturable optimizer counts one number for a group")
        return numbers.pop()

    def load_state_dict(self, state_dict):
        if any(s and ("m_scale" in s) != (self.states == "e4m3") for s in state_dict["state"].values()):
            raise ValueError(f"a state of another kind than {self.states}")
        needed = ("step", "m", "v") if self.states == "f32" else ("step", "m", "v", "m_scale", "v_scale", "strides")
        for state in state_dict["state"].values():
            missing = [name for name in needed if state and name not in state]
            if missing:
                raise ValueError(f"AdamW: a state without {', '.join(missing)}: it has {', '.join(map(str, state))}")
        taken = [self._steps_taken(group, state_dict["state"]) for group in state_dict["param_groups"]]
        super().load_state_dict(state_dict)
        self._lists = {}
        for group, number in zip(self.param_groups, taken):
            group.pop("clock", None)
            if self.capturable and number is not None:
                group["clock"] = torch.full((1,), number, dtype=torch.int64, device=group["params"][0].device)
            for p in group["params"]:
                if number is not None and self.state.get(p):
                    self.state[p]["step"] = 0 if self.capturable else number
        for state in self.state.values():
            if "m_scale" in state:             # (loading casts to the weights' type, which holds the codes exactly)
                for name in ("m", "v"):
                    state[name] = state[name].to(torch.float8_e4m3fn)


def grad_norm(params, max_norm=math.inf):
    """The norm of the gradients of params, and the factor that clips them to max_norm: two scalars on the device."""
    g = [p.grad if p.grad.is_contiguous() else p.grad.contiguous() for p in params if p.grad is not None]
    if not g:
        raise ValueError("grad_norm: no gradients")
    listed = step.param_list(g)
    out = torch.empty(2, device=g[0].device)
    step.fqt_grad_norm(listed, out, _workspace(step.fqt_grad_norm_workspace_size(listed), out.device), max_norm=max_norm)
    return out[0], out[1]


class Optimizers:
    """Several optimizers behind the interface that train.train_step uses, with one checkpoint.  A scheduler
    takes one of `optimizers`; param_groups has the groups of all."""

    def __init__(self, *optimizers):
        self.optimizers = optimizers

    def zero_grad(self, set_to_none=True):
        for o in self.optimizers:
            o.zero_grad(set_to_none=set_to_none)

    def step(self):
        for o in self.optimizers:
            o.step()

    @property
    def param_groups(self):
        return [group for o in self.optimizers for group in o.param_groups]

    def state_dict(self):
        return {"optimizers": [o.state_dict() for o in self.optimizers]}

    def load_state_dict(self, state):
        states = state["optimizers"]
        if len(states) != len(self.optimizers):
            raise ValueError(f"a state of {len(states)} optimizers, there are {len(self.optimizers)}")
        for o, s in zip(self.optimizers, states):
            o.load_state_dict(s)


def muon_and_adam(model, lr=0.02, adam_lr=1e-3, first_last=(), states=None, max_norm=None):
    """Muon for the weight matrices of a model, Adam for its vectors and for the modules in first_last
    (input and output layers, whose singular values carry meaning).  states: None for torch's Adam, "f32" or "e4m3" for
    AdamW here, with max_norm (over the gradients that it takes: Muon's update does not go by the size of its own)."""
    if states is None and max_norm is not None:
        raise ValueError("max_norm comes with states")
    apart = {id(p) for m in first_last for p in m.parameters()}
    matrices = [p for p in model.parameters() if p.dim() >= 2 and id(p) not in apart]
    chosen = {id(p) for p in matrices}
    rest = [p for p in model.parameters() if id(p) not in chosen]
    return Optimizers(*([Muon(matrices, lr=lr)] if matrices else []),
                      *([torch.optim.Adam(rest, lr=adam_lr) if states is None else
                         AdamW(rest, lr=adam_lr, states=states, max_norm=max_norm)] if rest else []))


class ResidualMLP(nn.Module):
    """features -> width, `depth` residual blocks, norm, classes.  A block norms the stream, expands it by
    an 8-bit product with GELU, and projects back by a binary layer (1-bit FQT backward) whose input is
    brought into its straight-through range by Hardtanh."""

    def __init__(self, features, classes, width=256, hidden=512, depth=3, bits=4, operands="int8"):
        super().__init__()
        self.stem = Linear(features, width)
        self.up = nn.ModuleList(NormLinear(width, hidden, act="gelu", operands=operands) for _ in range(depth))
        self.down = nn.ModuleList(train.BinaryLinear(hidden, width, bits=bits, layer_id=i) for i in range(depth))
        self.norm = RMSNorm(width)
        self.head = Linear(width, classes)

    def features(self, x):
        """What the head reads."""
        h, add = self.stem(x), None
        for up, down in zip(self.up, self.down):
            if add is None:
                z = up(h)
            else:
                z, h = up(add, h)
            add = down(nn.functional.hardtanh(z))
        return self.norm(h) if add is None else self.norm(add, h)[0]

    def forward(self, x):
        return self.head(self.features(x))

    def loss(self, x, target, **kw):
        """The loss of forward(x), without its logits (Linear.loss)."""
        return self.head.loss(self.features(x), target, **kw)
