"""What a decoder does to its tokens' rows beside the blocks: the scaled embedding and
the norm of each head's query and key with the rotation by position; the binding of
sw_embedding_* and sw_head_norm_* (include/scanweaver.h).
"""
from __future__ import annotations

import torch

from ._bind import _differentiable_once, _need, _on, _ptr
from ._lib import (SW_DTYPE_BF16, SW_DTYPE_F32, SW_EMBED_TOKENS_I64, SW_HEAD_ADJACENT, SW_HEAD_POS_I64,
                   check, fast)
from ._linear import _need_rows
from ._norm import _grad_like, _rows

_DTYPES = {torch.float32: SW_DTYPE_F32, torch.bfloat16: SW_DTYPE_BF16}


# ---- the norm of each head with the rotation


def _heads(t, name, dtype, lead):
    """The strides over (B, L, heads) of a (*lead, heads, K) tensor; one leading dimension
    is B, with L = 1."""
    if t.dtype is dtype and t.is_cuda and t.stride(-1) == 1:
        st = t.stride()
        return st[:-1] if len(lead) == 2 else (st[0], 0, st[1])
    return _need_rows(t if len(lead) == 2 else t.unsqueeze(1), name, dtype,
                      (lead[0], lead[1] if len(lead) == 2 else 1, *t.shape[-2:]))


def _head_operands(q, k, weight_q, weight_k, positions, inv_freq, adjacent):
    if not isinstance(q, torch.Tensor) or q.dim() not in (3, 4):
        raise ValueError("q must be a (B, L, H, K) or (B, H, K) tensor")
    dt = q.dtype
    if dt not in _DTYPES:
        raise TypeError("q must be float32 or bfloat16")
    lead, (H, K) = q.shape[:-2], q.shape[-2:]
    if not isinstance(k, torch.Tensor) or k.dim() != q.dim() or k.shape[:-2] != lead or k.shape[-1] != K:
        raise ValueError(f"k must have shape {tuple(lead)} + (Hk, {K}), as q has")
    st = _heads(q, "q", dt, lead) + _heads(k, "k", dt, lead)
    for w, name in ((weight_q, "weight_q"), (weight_k, "weight_k")):
        if w is not None:
            _need(w, name, torch.float32, (K,))
    R, flags = 0, SW_HEAD_ADJACENT if adjacent else 0
    if inv_freq is not None:
        _need(inv_freq, "inv_freq", torch.float32)
        R = 2 * inv_freq.shape[0] if inv_freq.dim() == 1 else K + 1
        if R > K:
            raise ValueError(f"inv_freq must be (R / 2,) with R at most {K} (got {tuple(inv_freq.shape)})")
    ps = (0, 0)
    if positions is not None:
        if not isinstance(positions, torch.Tensor) or positions.dtype not in (torch.int32, torch.int64):
            raise TypeError("positions must be an int32 or int64 tensor")
        if not positions.is_cuda:
            raise ValueError(f"positions must be on a GPU (got {positions.device})")
        if positions.shape != lead:
            raise ValueError(f"positions must have shape {tuple(lead)} (got {tuple(positions.shape)})")
        ps = tuple(s if n > 1 else 0 for s, n in zip(positions.stride(), lead))
        ps = ps if len(ps) == 2 else (ps[0], 0)
        if positions.dtype is torch.int64:
            flags |= SW_HEAD_POS_I64
    elif len(lead) == 1 and R:
        raise ValueError("single tokens (B, H, K) need their positions")
    B, L = lead if len(lead) == 2 else (lead[0], 1)
    return (B, L, H, k.shape[-2], K, R), st, ps, flags


def head_norm_fwd(q, k, weight_q=None, weight_k=None, *, positions=None, inv_freq=None, adjacent=False,
                  eps=1e-6):
    """The norm of each head's query and key with the rotation by the token's position;
    returns dense ``(q', k')``:

        u = weight * x / sqrt(mean(x ** 2) + eps)     over the K columns of a head
        y = u, its first R columns turned: pair j, (p, q) -> (p cos - q sin, q cos + p sin)
            by the angle position * inv_freq[j]

    q (B, L, H, K), k (B, L, Hk, K), or (B, H, K) and (B, Hk, K) for one token of each
    sequence; fp32 or bf16, any strides whose last is one, K at most 256.  Weights (K,)
    fp32 or None (ones).  ``inv_freq`` (R / 2,) fp32, None for no rotation; pair j is
    columns (j, j + R / 2), or (2 j, 2 j + 1) if ``adjacent``.  ``positions`` (B, L)
    int32 or int64 (expanded ones need no copy), 0 .. L - 1 if None.
    """
    sizes, st, ps, flags = _head_operands(q, k, weight_q, weight_k, positions, inv_freq, adjacent)
    yq, yk = (torch.empty(t.shape, dtype=q.dtype, device=q.device) for t in (q, k))
    with _on(q.device):
        check(fast().sw_head_norm_fwd(
            _ptr(q), _ptr(k), _ptr(weight_q), _ptr(weight_k), _ptr(positions), _ptr(inv_freq), _ptr(yq),
            _ptr(yk), *sizes, st + ps, _DTYPES[q.dtype], flags, eps), "sw_head_norm_fwd")
    return yq, yk


def head_norm_bwd(dq, dk, q, k, weight_q=None, weight_k=None, *, positions=None, inv_freq=None,
                  adjacent=False, eps=1e-6, want_dweight=True):
    """Backward of :func:`head_norm_fwd`, given the gradients of its results: a dict of
    ``dq``, ``dk`` in the inputs' type and, when ``want_dweight``, ``dweight_q``,
    ``dweight_k`` (K,) fp32."""
    sizes, st, ps, flags = _head_operands(q, k, weight_q, weight_k, positions, inv_freq, adjacent)
    lead = q.shape[:-2]
    for d, t, name in ((dq, q, "dq"), (dk, k, "dk")):
        if not isinstance(d, torch.Tensor) or d.shape != t.shape:
            raise ValueError(f"{name} must have shape {tuple(t.shape)}")
    st = _heads(dq, "dq", q.dtype, lead) + _heads(dk, "dk", q.dtype, lead) + st
    out = {n: torch.empty(t.shape, dtype=q.dtype, device=q.device) for n, t in (("dq", q), ("dk", k))}
    if want_dweight:
        for n in ("dweight_q", "dweight_k"):
            out[n] = torch.empty((sizes[4],), dtype=torch.float32, device=q.device)
    with _on(q.device):
        nws = fast().sw_head_norm_bwd_workspace(*sizes[:5]) if want_dweight else 0
        ws = torch.empty((nws,), dtype=torch.uint8, device=q.device) if nws else None
        check(fast().sw_head_norm_bwd(
            _ptr(dq), _ptr(dk), _ptr(q), _ptr(k), _ptr(weight_q), _ptr(weight_k), _ptr(positions),
            _ptr(inv_freq), _ptr(out["dq"]), _ptr(out["dk"]), _ptr(out.get("dweight_q")),
            _ptr(out.get("dweight_k")), *sizes, st + ps, _DTYPES[q.dtype], flags, eps, _ptr(ws), nws),
            "sw_head_norm_bwd")
    return out


class _HeadNormFn(torch.autograd.Function):
    """Autograd glue; no arithmetic happens here."""

    @staticmethod
    def forward(ctx, q, k, weight_q, weight_k, positions, inv_freq, adjacent, eps):
        ctx.save_for_backward(q, k, weight_q, weight_k, positions, inv_freq)
        ctx.how = dict(adjacent=adjacent, eps=eps)
        return head_norm_fwd(q, k, weight_q, weight_k, positions=positions, inv_freq=inv_freq, **ctx.how)

    @staticmethod
    def backward(ctx, dq, dk):
        q, k, wq, wk, positions, inv_freq = ctx.saved_tensors
        want = (wq is not None and ctx.needs_input_grad[2]) or (wk is not None and ctx.needs_input_grad[3])
        r = head_norm_bwd(_grad_like(dq, q.dtype), _grad_like(dk, q.dtype), q, k, wq, wk,
                          positions=positions, inv_freq=inv_freq, want_dweight=want, **ctx.how)
        grads = (r["dq"], r["dk"], r.get("dweight_q") if wq is not None else None,
                 r.get("dweight_k") if wk is not None else None, None, None, None, None)
        return _differentiable_once("head_norm_fn", grads, (q, k, wq, wk, dq, dk))


def head_norm_fn(q, k, weight_q=None, weight_k=None, *, positions=None, inv_freq=None, adjacent=False,
                 eps=1e-6):
    """Differentiable :func:`head_norm_fwd` (in q, k and the weights); returns ``(q', k')``."""
    return _HeadNormFn.apply(q, k, weight_q, weight_k, positions, inv_freq, bool(adjacent), eps)


# ---- the embedding


def _need_tokens(tokens):
    if not isinstance(tokens, torch.Tensor) or tokens.dtype not in (torch.int32, torch.int64):
        raise TypeError("tokens must be an int32 or int64 tensor")
    _need(tokens, "tokens", tokens.dtype)
    return SW_EMBED_TOKENS_I64 if tokens.dtype is torch.int64 else 0


def embedding_fwd(tokens, table, *, scale=1.0, dtype=None):
    """The tokens' rows of a table, scaled: (..., D) in ``dtype`` (the table's if None),
    ``scale * table[token]`` rounded once.

    tokens (...) int32 or int64, dense; table (V, D) fp32 or bf16, dense.  A token
    outside [0, V) is none (padding): its row is zero, and it adds to no gradient.
    """
    flags = _need_tokens(tokens)
    if not isinstance(table, torch.Tensor) or table.dim() != 2 or table.dtype not in _DTYPES:
        raise TypeError("table must be a (V, D) float32 or bfloat16 tensor")
    _need(table, "table", table.dtype)
    dtype = table.dtype if dtype is None else dtype
    if dtype not in _DTYPES:
        raise TypeError("dtype must be float32 or bfloat16")
    V, D = table.shape
    y = torch.empty((*tokens.shape, D), dtype=dtype, device=table.device)
    with _on(table.device):
        check(fast().sw_embedding_fwd(_ptr(tokens), _ptr(table), _ptr(y), tokens.numel(), V, D,
                                      _DTYPES[table.dtype], _DTYPES[dtype], flags, scale),
              "sw_embedding_fwd")
    return y


def embedding_bwd(tokens, dy, V, *, scale=1.0, dtype=None):
    """The gradient of :func:`embedding_fwd`'s table, dense (V, D) in ``dtype`` (dy's if
    None): row v is ``scale`` times the sum of dy (..., D) over the tokens equal to v, in
    fp32 and in a fixed order."""
    flags = _need_tokens(tokens)
    if not isinstance(dy, torch.Tensor) or dy.dtype not in _DTYPES:
        raise TypeError("dy must be a float32 or bfloat16 tensor")
    if dy.dim() != tokens.dim() + 1 or dy.shape[:-1] != tokens.shape:
        raise ValueError(f"dy must have shape {tuple(tokens.shape)} + (D,) (got {tuple(dy.shape)})")
    dtype = dy.dtype if dtype is None else dtype
    if dtype not in _DTYPES:
        raise TypeError("dtype must be float32 or bfloat16")
    T, D = tokens.numel(), dy.shape[-1]
    rows, st = _rows(dy, "dy", dy.dtype, dy.shape) if D else (dy, 0)
    out = torch.empty((V, D), dtype=dtype, device=dy.device)
    with _on(dy.device):
        nws = fast().sw_embedding_bwd_workspace(T, V, D)
        ws = torch.empty((nws,), dtype=torch.uint8, device=dy.device) if nws else None
        check(fast().sw_embedding_bwd(_ptr(tokens), _ptr(rows), _ptr(out), T, V, D, st, _DTYPES[dy.dtype],
                                      _DTYPES[dtype], flags, scale, _ptr(ws), nws), "sw_embedding_bwd")
    return out


class _EmbeddingFn(torch.autograd.Function):
    """Autograd glue; no arithmetic happens here."""

    @staticmethod
    def forward(ctx, tokens, table, scale, dtype):
        ctx.save_for_backward(tokens)
        y = embedding_fwd(tokens, table, scale=scale, dtype=dtype)
        ctx.how, ctx.V, ctx.dtype = dict(scale=scale, dtype=table.dtype), table.shape[0], y.dtype
        return y

    @staticmethod
    def backward(ctx, dy):
        (tokens,) = ctx.saved_tensors
        g = embedding_bwd(tokens, _grad_like(dy, ctx.dtype), ctx.V, **ctx.how)
        return _differentiable_once("embedding_fn", (None, g, None, None), (dy,))


def embedding_fn(tokens, table, *, scale=1.0, dtype=None):
    """Differentiable :func:`embedding_fwd` (in the table)."""
    return _EmbeddingFn.apply(tokens, table, scale, dtype)
