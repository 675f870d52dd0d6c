"""Linear attention with a log decay for each head: the binding of
sw_linear_attn_* (include/scanweaver.h).

    S_t = e^{g_t} S_{t-1} + k_t v_t^T,    o_t = scale S_t^T q_t

q, k: (B, L, Hk, K), v: (B, L, H, V) in fp32 or bf16, any strides whose last is
one; g: (B, L, H) or (H,) fp32; states (sequences, H, K, V) fp32.
"""
from __future__ import annotations

import torch

from ._bind import _dense_like, _differentiable_once, _need, _on, _ptr
from ._lib import SW_DTYPE_BF16, SW_DTYPE_F32, SW_LINEAR_G_HEAD, check, fast

_DTYPES = {torch.float32: SW_DTYPE_F32, torch.bfloat16: SW_DTYPE_BF16}


def _steps(st, shape):
    """The strides of two or three leading dimensions, 0 along a dimension of one."""
    a, b = (st[0] if shape[0] > 1 else 0), (st[1] if shape[1] > 1 else 0)
    return (a, b) if len(shape) == 2 else (a, b, st[2] if shape[2] > 1 else 0)


def _need_rows(t, name, dtype, shape):
    """A GPU tensor of this type and shape whose last dimension is contiguous;
    returns its strides without the last (0 along a dimension of one)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU (got {t.device})")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    st = t.stride()
    if shape[-1] > 1 and st[-1] != 1 and t.numel():
        raise ValueError(f"{name} must be contiguous along its last dimension")
    return _steps(st, shape[:-1])


def _need_decay(g, lead, H):
    """(strides over (*lead, heads), flags) of g: (*lead, H) or (H,) fp32."""
    if not isinstance(g, torch.Tensor):
        raise TypeError("g must be a torch.Tensor")
    if not g.is_cuda:
        raise ValueError(f"g must be on a GPU (got {g.device})")
    if g.dtype is not torch.float32:
        raise TypeError(f"g must be torch.float32 (got {g.dtype})")
    if g.dim() == 1 and g.shape[0] == H:
        return (0,) * len(lead) + (g.stride(0) if H > 1 else 0,), SW_LINEAR_G_HEAD
    if g.shape != (*lead, H):
        raise ValueError(f"g must have shape {(*lead, H)} or {(H,)} (got {tuple(g.shape)})")
    return _steps(g.stride(), g.shape), 0


def _operands(q, k, v, g, h0, cu_seqlens):
    if not isinstance(q, torch.Tensor) or q.dim() != 4:
        raise ValueError("q must be a (B, L, Hk, K) tensor")
    dt = q.dtype
    if dt not in _DTYPES:
        raise TypeError("q must be float32 or bfloat16")
    if not isinstance(v, torch.Tensor) or v.dim() != 4:
        raise ValueError("v must be a (B, L, H, V) tensor")
    B, L, Hk, K = q.shape
    H, V = v.shape[2:]
    st = _need_rows(q, "q", dt, (B, L, Hk, K))
    st += _need_rows(k, "k", dt, (B, L, Hk, K))
    st += _need_rows(v, "v", dt, (B, L, H, V))
    gs, flags = _need_decay(g, (B, L), H)
    n = B
    if cu_seqlens is not None:
        _need(cu_seqlens, "cu_seqlens", torch.int32)
        if cu_seqlens.dim() != 1 or cu_seqlens.shape[0] < 2 or B != 1:
            raise ValueError("cu_seqlens must be (sequences + 1,), with B = 1")
        n = cu_seqlens.shape[0] - 1
    if h0 is not None:
        _need(h0, "h0", torch.float32, (n, H, K, V))
    return (B, L, Hk, H, K, V, n), st + gs, _DTYPES[dt], flags


def _workspace(query, sizes, dt, flags, packed, device):
    """From torch's allocator, which takes it back after the call."""
    n = query(*sizes, dt, flags, packed)
    return (torch.empty((n,), dtype=torch.uint8, device=device) if n else None), n


def linear_attn_fwd(q, k, v, g, *, scale=None, h0=None, cu_seqlens=None, o=None, h_last=None,
                    want_h_last=True):
    """Linear attention over whole sequences; returns ``(o, h_last)`` (h_last None
    if not wanted).

    q, k: (B, L, Hk, K); v: (B, L, H, V), H a multiple of Hk; all fp32 or all
    bf16, K and V at most 256; g: (B, L, H), or (H,) for one decay a head, fp32.
    ``scale`` is K ** -0.5 if not given.  ``h0`` (n, H, K, V) fp32 is the initial
    state, e.g. the h_last of an earlier part.  With ``cu_seqlens`` (n + 1,) int32,
    ascending within [0, L], B is 1 and the row holds n sequences one after the
    other (o is zero at steps that none of them covers, as are the gradients);
    else n = B.
    """
    sizes, st, dt, flags = _operands(q, k, v, g, h0, cu_seqlens)
    B, L, Hk, H, K, V, n = sizes
    if o is None:
        o = _dense_like(v)
    else:
        _need(o, "o", q.dtype, (B, L, H, V))
    if not want_h_last:
        h_last = None
    elif h_last is None:
        h_last = torch.empty((n, H, K, V), dtype=torch.float32, device=q.device)
    else:
        _need(h_last, "h_last", torch.float32, (n, H, K, V))
    with _on(q.device):
        ws, nws = _workspace(fast().sw_linear_attn_fwd_workspace, sizes, dt, flags,
                             cu_seqlens is not None, q.device)
        check(fast().sw_linear_attn_fwd(
            _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(h0), _ptr(cu_seqlens), _ptr(o),
            _ptr(h_last), *sizes, st, dt, flags, K ** -0.5 if scale is None else scale, _ptr(ws),
            nws), "sw_linear_attn_fwd")
    return o, h_last


def linear_attn_bwd(q, k, v, g, do, dh_last=None, *, scale=None, h0=None, cu_seqlens=None,
                    want_dh0=True):
    """Backward of :func:`linear_attn_fwd`: the gradients of sum(do * o) +
    sum(dh_last * h_last).  ``do`` (B, L, H, V) of the inputs' type, ``dh_last``
    like h_last or None.  Returns a dict: dq, dk, dv in the inputs' type, dg of
    g's shape and dh0 (n, H, K, V) (when ``want_dh0``) in fp32.
    """
    sizes, st, dt, flags = _operands(q, k, v, g, h0, cu_seqlens)
    B, L, Hk, H, K, V, n = sizes
    st += _need_rows(do, "do", q.dtype, (B, L, H, V))
    if dh_last is not None:
        _need(dh_last, "dh_last", torch.float32, (n, H, K, V))
    like = dict(dtype=q.dtype, device=q.device)
    f32 = dict(dtype=torch.float32, device=q.device)
    out = {"dq": torch.empty((B, L, Hk, K), **like), "dk": torch.empty((B, L, Hk, K), **like),
           "dv": torch.empty((B, L, H, V), **like),
           "dg": torch.empty((H,) if flags else (B, L, H), **f32)}
    if want_dh0:
        out["dh0"] = torch.empty((n, H, K, V), **f32)
    with _on(q.device):
        ws, nws = _workspace(fast().sw_linear_attn_bwd_workspace, sizes, dt, flags,
                             cu_seqlens is not None, q.device)
        check(fast().sw_linear_attn_bwd(
            _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(h0), _ptr(cu_seqlens), _ptr(do),
            _ptr(dh_last), _ptr(out["dq"]), _ptr(out["dk"]), _ptr(out["dv"]), _ptr(out["dg"]),
            _ptr(out.get("dh0")), *sizes, st, dt, flags, K ** -0.5 if scale is None else scale,
            _ptr(ws), nws), "sw_linear_attn_bwd")
    return out


class _LinearAttnFn(torch.autograd.Function):
    """Autograd glue; no arithmetic happens here."""

    @staticmethod
    def forward(ctx, q, k, v, g, h0, cu_seqlens, scale, want_h_last):
        o, h_last = linear_attn_fwd(q, k, v, g, scale=scale, h0=h0, cu_seqlens=cu_seqlens,
                                    want_h_last=want_h_last)
        ctx.save_for_backward(q, k, v, g, h0, cu_seqlens)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return o, h_last

    @staticmethod
    def backward(ctx, do, dh_last):
        q, k, v, g, h0, cu = ctx.saved_tensors
        if do is None:  # only h_last reached the loss
            do = torch.zeros(v.shape, dtype=v.dtype, device=v.device)
        do = do.to(v.dtype)
        if do.shape[-1] > 1 and do.stride(-1) != 1:
            do = do.contiguous()
        if dh_last is not None:
            dh_last = dh_last.contiguous().to(torch.float32)
        r = linear_attn_bwd(q, k, v, g, do, dh_last, scale=ctx.scale, h0=h0, cu_seqlens=cu,
                            want_dh0=h0 is not None and ctx.needs_input_grad[4])
        grads = r["dq"], r["dk"], r["dv"], r["dg"], r.get("dh0"), None, None, None
        return _differentiable_once("linear_attn_fn", grads, (q, k, v, g, h0, do, dh_last))


def linear_attn_fn(q, k, v, g, *, scale=None, h0=None, cu_seqlens=None, return_last_state=False):
    """Differentiable linear attention: :func:`linear_attn_fwd` forward,
    :func:`linear_attn_bwd` backward through torch autograd.  With
    ``return_last_state`` returns ``(o, h_last)``, both differentiable."""
    o, h_last = _LinearAttnFn.apply(q, k, v, g, h0, cu_seqlens, scale, bool(return_last_state))
    return (o, h_last) if return_last_state else o


def linear_attn_step(q, k, v, g, state, *, scale=None, slots=None, o=None):
    """One token of each sequence of a batch, its state updated in place; returns
    o (B, H, V).

    q, k: (B, Hk, K); v: (B, H, V); g: (B, H) or (H,) fp32; ``state`` (pool, H, K,
    V) fp32, dense.  Sequence b's state is state[slots[b]] (state[b] without
    ``slots``, (B,) int32); a slot outside [0, pool) is no sequence: its o is zero
    and nothing is updated.  Two sequences must not share a slot.
    """
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a (B, Hk, K) tensor")
    dt = q.dtype
    if dt not in _DTYPES:
        raise TypeError("q must be float32 or bfloat16")
    if not isinstance(v, torch.Tensor) or v.dim() != 3:
        raise ValueError("v must be a (B, H, V) tensor")
    B, Hk, K = q.shape
    H, V = v.shape[1:]
    st = _need_rows(q, "q", dt, (B, Hk, K))
    st += _need_rows(k, "k", dt, (B, Hk, K))
    st += _need_rows(v, "v", dt, (B, H, V))
    gs, flags = _need_decay(g, (B,), H)
    if not isinstance(state, torch.Tensor) or state.dim() != 4:
        raise ValueError("state must be a (pool, H, K, V) tensor")
    pool = state.shape[0]
    _need(state, "state", torch.float32, (pool, H, K, V))
    if slots is not None:
        _need(slots, "slots", torch.int32, (B,))
    elif pool < B:
        raise ValueError(f"state holds {pool} sequences (got {B})")
    if o is None:
        o = _dense_like(v)
    else:
        _need(o, "o", dt, (B, H, V))
    with _on(q.device):
        check(fast().sw_linear_attn_step(
            _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(state), _ptr(slots), _ptr(o), B, Hk, H, K, V,
            pool, st + gs, _DTYPES[dt], flags, K ** -0.5 if scale is None else scale),
            "sw_linear_attn_step")
    return o
