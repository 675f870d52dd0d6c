"""A gated linear recurrence for each channel: the binding of sw_gated_scan_*
(include/scanweaver.h).

    m_t = c softplus(lam) sigmoid(r_t),    a_t = e^{-m_t}
    h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(i_t) x_t

x, r, i: (B, L, D) in fp32 or bf16, any strides whose last is one; lam (D,) fp32;
states (sequences, D) fp32.
"""
from __future__ import annotations

import torch

from ._bind import _dense_like, _differentiable_once, _need, _on, _ptr
from ._lib import SW_DTYPE_BF16, SW_DTYPE_F32, SW_GATED_CKPT, check, fast

_DTYPES = {torch.float32: SW_DTYPE_F32, torch.bfloat16: SW_DTYPE_BF16}


def _rate(c):
    c = float(c)
    if not 0.0 < c < float("inf"):
        raise ValueError(f"c must be positive and finite (got {c})")
    return c


def _same_rows(ts, names, dt, shape):
    """The strides of tensors of one type and shape, one after the other's, without the
    last, which is one."""
    st = ()
    for t, name in zip(ts, names):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a torch.Tensor")
        if not t.is_cuda:
            raise ValueError(f"{name} must be on a GPU (got {t.device})")
        if t.dtype is not dt:
            raise TypeError(f"{name} must be {dt} (got {t.dtype})")
        if t.shape != shape:
            raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
        s = t.stride()
        if s[-1] != 1 and shape[-1] > 1 and t.numel():
            raise ValueError(f"{name} must be contiguous along its last dimension")
        st += s[:-1]
    return st


def _operands(x, r, i, lam, c, h0, cu_seqlens, *dh):
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        raise ValueError("x must be a (B, L, D) tensor")
    dt = x.dtype
    if dt not in _DTYPES:
        raise TypeError("x must be float32 or bfloat16")
    shape = x.shape
    B, L, D = shape
    st = _same_rows((x, r, i, *dh), ("x", "r", "i", "dh"), dt, shape)
    _need(lam, "lam", torch.float32, (D,))
    n = B
    if cu_seqlens is not None:
        _need(cu_seqlens, "cu_seqlens", torch.int32)
        if cu_seqlens.dim() != 1 or cu_seqlens.shape[0] < 2 or B != 1:
            raise ValueError("cu_seqlens must be (sequences + 1,), with B = 1")
        n = cu_seqlens.shape[0] - 1
    if h0 is not None:
        _need(h0, "h0", torch.float32, (n, D))
    return (B, L, D, n), st, _DTYPES[dt], _rate(c)


def _workspace(n, device):
    """From torch's allocator, which takes it back after the call."""
    return (torch.empty((n,), dtype=torch.uint8, device=device) if n else None), n


def _forward(x, r, i, lam, c, h0, cu_seqlens, h, h_last, keep):
    """(h, h_last, the states that the backward starts from)."""
    sizes, st, dt, c = _operands(x, r, i, lam, c, h0, cu_seqlens)
    B, L, D, n = sizes
    f32 = dict(dtype=torch.float32, device=x.device)
    if h is None:
        h = _dense_like(x)
    else:
        _need(h, "h", x.dtype, (B, L, D))
    if h_last is True:
        h_last = torch.empty((n, D), **f32)
    elif h_last is not None:
        _need(h_last, "h_last", torch.float32, (n, D))
    ckpt = torch.empty((B, -(-L // SW_GATED_CKPT), D), **f32) if keep else None
    with _on(x.device):
        ws, nws = _workspace(fast().sw_gated_scan_fwd_workspace(B, L, D), x.device)
        check(fast().sw_gated_scan_fwd(
            _ptr(x), _ptr(r), _ptr(i), _ptr(lam), _ptr(h0), _ptr(cu_seqlens), _ptr(h), _ptr(h_last),
            _ptr(ckpt), B, L, D, n, st, dt, c, _ptr(ws), nws), "sw_gated_scan_fwd")
    return h, h_last, ckpt


def gated_scan_fwd(x, r, i, lam, *, c=8.0, h0=None, cu_seqlens=None, h=None, h_last=None,
                   want_h_last=True):
    """The gated recurrence over whole sequences; returns ``(h, h_last)`` (h_last None
    if not wanted).

    x, r, i: (B, L, D), all fp32 or all bf16, r and i before their sigmoids; lam (D,)
    fp32; c > 0.  ``h0`` (n, D) fp32 is the state before the first step, e.g. the
    h_last of an earlier part.  With ``cu_seqlens`` (n + 1,) int32, ascending within
    [0, L], B is 1 and the row holds n sequences one after the other (h is zero at
    steps that none of them covers, as are the gradients); else n = B.
    """
    if not want_h_last:
        h_last = None
    elif h_last is None:
        h_last = True
    return _forward(x, r, i, lam, c, h0, cu_seqlens, h, h_last, False)[:2]


def gated_scan_bwd(x, r, i, lam, dh, dh_last=None, *, c=8.0, h0=None, cu_seqlens=None,
                   want_dh0=True, ckpt=None):
    """Backward of :func:`gated_scan_fwd`: the gradients of sum(dh * h) + sum(dh_last *
    h_last).  ``dh`` (B, L, D) of the inputs' type, ``dh_last`` like h_last or None;
    ``ckpt`` what a training forward kept (formed again if None).  Returns a dict: dx,
    dr, di in the inputs' type, dlam (D,) and dh0 (n, D) (when ``want_dh0``) in fp32.
    """
    sizes, st, dt, c = _operands(x, r, i, lam, c, h0, cu_seqlens, dh)
    B, L, D, n = sizes
    if dh_last is not None:
        _need(dh_last, "dh_last", torch.float32, (n, D))
    if ckpt is not None:
        _need(ckpt, "ckpt", torch.float32, (B, -(-L // SW_GATED_CKPT), D))
    f32 = dict(dtype=torch.float32, device=x.device)
    out = {name: torch.empty((B, L, D), dtype=x.dtype, device=x.device) for name in ("dx", "dr", "di")}
    out["dlam"] = torch.empty((D,), **f32)
    if want_dh0:
        out["dh0"] = torch.empty((n, D), **f32)
    with _on(x.device):
        ws, nws = _workspace(fast().sw_gated_scan_bwd_workspace(B, L, D, ckpt is not None), x.device)
        check(fast().sw_gated_scan_bwd(
            _ptr(x), _ptr(r), _ptr(i), _ptr(lam), _ptr(h0), _ptr(cu_seqlens), _ptr(ckpt), _ptr(dh),
            _ptr(dh_last), _ptr(out["dx"]), _ptr(out["dr"]), _ptr(out["di"]), _ptr(out["dlam"]),
            _ptr(out.get("dh0")), B, L, D, n, st, dt, c, _ptr(ws), nws), "sw_gated_scan_bwd")
    return out


class _GatedScanFn(torch.autograd.Function):
    """Autograd glue; no arithmetic happens here."""

    @staticmethod
    def forward(ctx, x, r, i, lam, h0, cu_seqlens, c, want_h_last, keep):
        h, h_last, ckpt = _forward(x, r, i, lam, c, h0, cu_seqlens, None, want_h_last or None, keep)
        ctx.save_for_backward(x, r, i, lam, h0, cu_seqlens, ckpt)
        ctx.c = c
        ctx.set_materialize_grads(False)
        return h, h_last

    @staticmethod
    def backward(ctx, dh, dh_last):
        x, r, i, lam, h0, cu, ckpt = ctx.saved_tensors
        if dh is None:  # only h_last reached the loss
            dh = torch.zeros(x.shape, dtype=x.dtype, device=x.device)
        dh = dh.to(x.dtype)
        if dh.shape[-1] > 1 and dh.stride(-1) != 1:
            dh = dh.contiguous()
        if dh_last is not None:
            dh_last = dh_last.contiguous().to(torch.float32)
        g = gated_scan_bwd(x, r, i, lam, dh, dh_last, c=ctx.c, h0=h0, cu_seqlens=cu,
                           want_dh0=h0 is not None and ctx.needs_input_grad[4], ckpt=ckpt)
        grads = g["dx"], g["dr"], g["di"], g["dlam"], g.get("dh0"), None, None, None, None
        return _differentiable_once("gated_scan_fn", grads, (x, r, i, lam, h0, dh, dh_last))


def gated_scan_fn(x, r, i, lam, *, c=8.0, h0=None, cu_seqlens=None, return_last_state=False):
    """Differentiable gated recurrence: :func:`gated_scan_fwd` forward,
    :func:`gated_scan_bwd` backward through torch autograd.  With
    ``return_last_state`` returns ``(h, h_last)``, both differentiable."""
    # states for the backward only where there can be one
    keep = torch.is_grad_enabled() and any(getattr(t, "requires_grad", False) for t in (x, r, i, lam, h0))
    h, h_last = _GatedScanFn.apply(x, r, i, lam, h0, cu_seqlens, c, bool(return_last_state), keep)
    return (h, h_last) if return_last_state else h


def gated_scan_step(x, r, i, lam, state, *, c=8.0, slots=None, h=None):
    """One token of each sequence of a batch, its state updated in place; returns h (B, D).

    x, r, i: (B, D); ``state`` (pool, D) fp32, dense.  Sequence b's state is
    state[slots[b]] (state[b] without ``slots``, (B,) int32); a slot outside [0, pool)
    is no sequence: its h is zero and nothing is updated.  Two sequences must not share
    a slot.
    """
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("x must be a (B, D) tensor")
    dt = x.dtype
    if dt not in _DTYPES:
        raise TypeError("x must be float32 or bfloat16")
    B, D = x.shape
    st = _same_rows((x, r, i), ("x", "r", "i"), dt, x.shape)
    _need(lam, "lam", torch.float32, (D,))
    if not isinstance(state, torch.Tensor) or state.dim() != 2:
        raise ValueError("state must be a (pool, D) tensor")
    pool = state.shape[0]
    _need(state, "state", torch.float32, (pool, D))
    if slots is not None:
        _need(slots, "slots", torch.int32, (B,))
    elif pool < B:
        raise ValueError(f"state holds {pool} sequences (got {B})")
    if h is None:
        h = _dense_like(x)
    else:
        _need(h, "h", dt, (B, D))
    with _on(x.device):
        check(fast().sw_gated_scan_step(_ptr(x), _ptr(r), _ptr(i), _ptr(lam), _ptr(state), _ptr(slots),
                                        _ptr(h), B, D, pool, st, _DTYPES[dt], _rate(c)),
              "sw_gated_scan_step")
    return h
