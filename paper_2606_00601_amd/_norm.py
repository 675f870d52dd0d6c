"""The norms before and after a block: the binding of sw_residual_norm_* and
sw_gated_norm_* (include/scanweaver.h).

Tensors are (..., D), in fp32 or bf16, contiguous along D; leading dimensions
that one stride does not cover are copied first.  Weights and scales are (D,)
fp32; outputs are dense.
"""
from __future__ import annotations

import torch

from ._bind import _dense_like, _differentiable_once, _need, _on, _ptr
from ._lib import SW_DTYPE_BF16, SW_DTYPE_F32, SW_GATE_AFTER, check, fast

_DTYPES = {torch.float32: SW_DTYPE_F32, torch.bfloat16: SW_DTYPE_BF16}


def _rows(t, name, dtype, shape):
    """(t as rows of D, elements from row to row)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU (got {t.device})")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    D = shape[-1]
    if t.is_contiguous():
        return t, D
    if D > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} must be contiguous along its last dimension")
    t = t.reshape(-1, D)  # a view where one stride covers the leading dimensions
    return t, t.stride(0) if t.shape[0] > 1 else D


def _of(x, name):
    if not isinstance(x, torch.Tensor) or x.dim() < 1:
        raise ValueError(f"{name} must be a (..., D) tensor")
    if x.dtype not in _DTYPES:
        raise TypeError(f"{name} must be float32 or bfloat16")
    D = x.shape[-1]
    if D == 0:
        raise ValueError(f"{name} has no columns")
    return x.shape, x.numel() // D, D, x.dtype


def _res_type(t, name, dtype):
    if not isinstance(t, torch.Tensor) or t.dtype not in (dtype, torch.float32):
        raise TypeError(f"{name} must be a {dtype} or float32 tensor")
    return t.dtype


def _workspace(M, D, width, grads, device):
    n = fast().sw_norm_bwd_workspace(M, D, width, grads)
    return (torch.empty((n,), dtype=torch.uint8, device=device) if n else None), n


def residual_norm_fwd(x, weight, residual=None, *, res_scale=None, eps=1e-6):
    """The norm before a block; returns ``(y, residual_out)``:

        residual_out = residual + res_scale * x     (x itself without residual)
        y = weight * residual_out / sqrt(mean(residual_out ** 2) + eps)

    x (..., D) fp32 or bf16; residual of x's type or fp32, residual_out of its
    type (y is the norm of the values as stored there); weight, res_scale (D,)
    fp32, D at most 16384.
    """
    shape, M, D, dt = _of(x, "x")
    _need(weight, "weight", torch.float32, (D,))
    if residual is None and res_scale is not None:
        raise ValueError("res_scale scales x on its way into a residual: pass residual too")
    if res_scale is not None:
        _need(res_scale, "res_scale", torch.float32, (D,))
    xr, x_st = _rows(x, "x", dt, shape)
    rt, rr, r_st, out = dt, None, D, None
    if residual is not None:
        rt = _res_type(residual, "residual", dt)
        rr, r_st = _rows(residual, "residual", rt, shape)
        out = _dense_like(residual)
    y = _dense_like(x)
    with _on(x.device):
        check(fast().sw_residual_norm_fwd(
            _ptr(xr), _ptr(rr), _ptr(weight), _ptr(res_scale), _ptr(y), _ptr(out), M, D, x_st, r_st,
            _DTYPES[dt], _DTYPES[rt], eps), "sw_residual_norm_fwd")
    return y, x if out is None else out


def residual_norm_bwd(dy, dres, residual_out, weight, *, x=None, res_scale=None, eps=1e-6):
    """Backward of :func:`residual_norm_fwd`: the gradients of sum(dy * y) +
    sum(dres * residual_out) (dres None: no second term) from residual_out, and
    from x where there is a res_scale.  Returns a dict: ``dx`` in dy's type,
    ``dresidual`` in residual_out's (one tensor where both are the same), and
    ``dweight``, ``dres_scale`` (D,) fp32.
    """
    shape, M, D, dt = _of(dy, "dy")
    _need(weight, "weight", torch.float32, (D,))
    rt = _res_type(residual_out, "residual_out", dt)
    d, d_st = _rows(dy, "dy", dt, shape)
    o, o_st = _rows(residual_out, "residual_out", rt, shape)
    e, e_st, xr, x_st = None, D, None, D
    if dres is not None:
        e, e_st = _rows(dres, "dres", rt, shape)
    if res_scale is not None:
        _need(res_scale, "res_scale", torch.float32, (D,))
        xr, x_st = _rows(x, "x", dt, shape)
    f32 = dict(dtype=torch.float32, device=dy.device)
    same = res_scale is None and rt is dt
    out = {"dresidual": _dense_like(residual_out),
           "dweight": torch.empty((D,), **f32)}
    out["dx"] = out["dresidual"] if same else _dense_like(dy)
    if res_scale is not None:
        out["dres_scale"] = torch.empty((D,), **f32)
    with _on(dy.device):
        ws, nws = _workspace(M, D, D, 1 if res_scale is None else 2, dy.device)
        check(fast().sw_residual_norm_bwd(
            _ptr(d), _ptr(e), _ptr(o), _ptr(weight), _ptr(xr), _ptr(res_scale),
            None if same else _ptr(out["dx"]), _ptr(out["dresidual"]), _ptr(out["dweight"]),
            _ptr(out.get("dres_scale")), M, D, d_st, e_st, o_st, x_st, _DTYPES[dt], _DTYPES[rt],
            eps, _ptr(ws), nws), "sw_residual_norm_bwd")
    return out


def _grad_like(d, like):
    """An incoming gradient in its tensor's type, contiguous along the last dimension."""
    if d is None:
        return None
    d = d.to(like)
    return d.contiguous() if d.shape[-1] > 1 and d.stride(-1) != 1 else d


class _ResidualNormFn(torch.autograd.Function):
    """Autograd glue; no arithmetic happens here."""

    @staticmethod
    def forward(ctx, x, weight, residual, res_scale, eps):
        y, out = residual_norm_fwd(x, weight, residual, res_scale=res_scale, eps=eps)
        ctx.save_for_backward(out, weight, x if res_scale is not None else None, res_scale)
        ctx.eps, ctx.alone, ctx.dtype = eps, residual is None, x.dtype
        ctx.set_materialize_grads(False)
        return (y, None) if residual is None else (y, out)

    @staticmethod
    def backward(ctx, dy, dres):
        out, weight, x, res_scale = ctx.saved_tensors
        if dy is None:  # only the residual reached the loss
            dy = torch.zeros(out.shape, dtype=ctx.dtype, device=out.device)
        r = residual_norm_bwd(_grad_like(dy, ctx.dtype), _grad_like(dres, out.dtype), out, weight,
                              x=x, res_scale=res_scale, eps=ctx.eps)
        grads = (r["dx"], r["dweight"], None if ctx.alone else r["dresidual"],
                 r.get("dres_scale"), None)
        return _differentiable_once("residual_norm_fn", grads, (out, weight, x, res_scale, dy, dres))


def residual_norm_fn(x, weight, residual=None, *, res_scale=None, eps=1e-6):
    """Differentiable :func:`residual_norm_fwd`; returns ``(y, residual_out)``."""
    y, out = _ResidualNormFn.apply(x, weight, residual, res_scale, eps)
    return y, x if residual is None else out


def _gated(x, z, weight, group, gate_after):
    shape, M, D, dt = _of(x, "x")
    _need(weight, "weight", torch.float32, (D,))
    group = D if group is None else int(group)
    if group < 1 or D % group:
        raise ValueError(f"D = {D} is no multiple of group = {group}")
    xr, x_st = _rows(x, "x", dt, shape)
    zr, z_st = (None, D) if z is None else _rows(z, "z", dt, shape)
    return shape, M, D, dt, group, xr, x_st, zr, z_st, SW_GATE_AFTER if gate_after else 0


def gated_norm_fwd(x, z, weight, *, group=None, gate_after=False, eps=1e-6):
    """The norm after a block's mixer, with its gate, over groups of ``group``
    columns (the whole row if None; a head's width for a norm of each head):

        y = weight * u / sqrt(mean(u ** 2) + eps),  u = x * silu(z)

    or, with ``gate_after``, weight * x / sqrt(mean(x ** 2) + eps) * silu(z).  x, z
    (..., D) fp32 or bf16, z None for no gate; weight (D,) fp32.  Returns y.
    """
    shape, M, D, dt, group, xr, x_st, zr, z_st, flags = _gated(x, z, weight, group, gate_after)
    y = _dense_like(x)
    with _on(x.device):
        check(fast().sw_gated_norm_fwd(
            _ptr(xr), _ptr(zr), _ptr(weight), _ptr(y), M, D, group, x_st, z_st, _DTYPES[dt], flags,
            eps), "sw_gated_norm_fwd")
    return y


def gated_norm_bwd(dy, x, z, weight, *, group=None, gate_after=False, eps=1e-6):
    """Backward of :func:`gated_norm_fwd`: a dict of ``dx``, ``dz`` (with z) in the
    inputs' type and ``dweight`` (D,) fp32."""
    shape, M, D, dt, group, xr, x_st, zr, z_st, flags = _gated(x, z, weight, group, gate_after)
    d, d_st = _rows(dy, "dy", dt, shape)
    out = {"dx": _dense_like(x),
           "dweight": torch.empty((D,), dtype=torch.float32, device=x.device)}
    if z is not None:
        out["dz"] = _dense_like(z)
    with _on(x.device):
        ws, nws = _workspace(M, D, group, 1, x.device)
        check(fast().sw_gated_norm_bwd(
            _ptr(d), _ptr(xr), _ptr(zr), _ptr(weight), _ptr(out["dx"]), _ptr(out.get("dz")),
            _ptr(out["dweight"]), M, D, group, d_st, x_st, z_st, _DTYPES[dt], flags, eps, _ptr(ws),
            nws), "sw_gated_norm_bwd")
    return out


class _GatedNormFn(torch.autograd.Function):
    """Autograd glue; no arithmetic happens here."""

    @staticmethod
    def forward(ctx, x, z, weight, group, gate_after, eps):
        ctx.save_for_backward(x, z, weight)
        ctx.how = dict(group=group, gate_after=gate_after, eps=eps)
        return gated_norm_fwd(x, z, weight, **ctx.how)

    @staticmethod
    def backward(ctx, dy):
        x, z, weight = ctx.saved_tensors
        r = gated_norm_bwd(_grad_like(dy, x.dtype), x, z, weight, **ctx.how)
        grads = r["dx"], r.get("dz"), r["dweight"], None, None, None
        return _differentiable_once("gated_norm_fn", grads, (x, z, weight, dy))


def gated_norm_fn(x, z, weight, *, group=None, gate_after=False, eps=1e-6):
    """Differentiable :func:`gated_norm_fwd`; returns y."""
    return _GatedNormFn.apply(x, z, weight, group, bool(gate_after), eps)
