"""Residual blocks and an optimizer around binary layers: torch modules over the dense operators.

RMSNorm, Linear and NormLinear call fqt_rmsnorm_*, fqt_quantize_rows and fqt_linear_* (forward and
backward); NormLinear keeps the activations between the norm and the product as 8-bit codes.  Muon
updates latent weight matrices (and convolution weights, unfolded) by fqt_muon_step.  ResidualMLP puts
them together with BinaryLinear: a float32 residual stream, blocks of a normed 8-bit expansion with
GELU and a binary projection, the first and last layers at full width as in the networks of `train`.

Modules take [..., features] inputs of float32 or bfloat16, keep float32 parameters, and cast or
quantize the weight in every forward pass.  Gradients come in the type of what they belong to (the products
of the backward take dz in bf16, as fqt_linear_backward says) and cannot be differentiated again.
"""
import math

import torch
import torch.nn as nn
from torch.autograd.function import once_differentiable

from . import dense, train

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


def muon_and_adam(model, lr=0.02, adam_lr=1e-3, first_last=()):
    """Muon for the weight matrices of a model, Adam for its vectors and for the modules in first_last
    (input and output layers, whose singular values carry meaning)."""
    apart = {id(p) for m in first_last for p in m.parameters()}
    matrices = [p for p in model.parameters() if p.dim() >= 2 and id(p) not in apart]
    chosen = {id(p) for p in matrices}
    rest = [p for p in model.parameters() if id(p) not in chosen]
    return Optimizers(*([Muon(matrices, lr=lr)] if matrices else []),
                      *([torch.optim.Adam(rest, lr=adam_lr)] if rest else []))


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

    def forward(self, x):
        h, add = self.stem(x), None
        for up, down in zip(self.up, self.down):
            if add is None:
                z = up(h)
            else:
                z, h = up(add, h)
            add = down(nn.functional.hardtanh(z))
        y = self.norm(h) if add is None else self.norm(add, h)[0]
        return self.head(y)
