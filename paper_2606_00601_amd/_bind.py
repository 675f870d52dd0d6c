"""Checks and marshalling shared by the binding's modules."""
from __future__ import annotations

import torch

from ._lib import fast


def _ptr(t):
    return None if t is None else t.data_ptr()


def _need(t, name, dtype, shape=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU (got {t.device})")
    if t.dtype is not dtype:  # dtypes are singletons
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and t.shape != shape:  # torch.Size compares as a tuple
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")


def _dense_like(t):
    """A dense tensor of t's shape and type, not filled."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)


def _current_device():
    # the binding only runs once a GPU tensor exists, so torch's GPU state is
    # initialised and its raw query is enough
    if _get_device is not None:
        return _get_device()
    return torch.cuda.current_device()


def _stream_handle(idx):
    """torch's current HIP stream on GPU idx, as a raw handle."""
    if _raw_stream is not None:
        return _raw_stream(idx)
    return torch.cuda.current_stream(idx).cuda_stream


class _on:
    """``with _on(device):`` makes the tensor's GPU current (switching only when
    another one is) and hands torch's current stream on it to the library, for
    the library calls inside the block."""

    __slots__ = ("idx", "prev")

    def __init__(self, device):
        idx = device.index
        self.idx = idx if idx is not None else _current_device()
        self.prev = -1

    def __enter__(self):
        cur = _current_device()
        if cur != self.idx:
            torch.cuda.set_device(self.idx)
            self.prev = cur
        fast().sw_set_stream(_stream_handle(self.idx))
        return self

    def __exit__(self, *exc):
        if self.prev >= 0:
            torch.cuda.set_device(self.prev)
        return False


class _Once(torch.autograd.Function):
    """Gradients on their way out of a backward: themselves, and an error where they
    are differentiated again."""

    @staticmethod
    def forward(ctx, name, count, *tensors):
        ctx.name = name
        return tensors[:count]

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError(f"{ctx.name} cannot be differentiated twice: its backward is not "
                           "differentiable")


def _differentiable_once(name, grads, inputs):
    """``grads`` (tensors or None) of a backward that read ``inputs``.  Under
    ``create_graph`` they depend on those, so that a second derivative raises instead of
    coming out without their share."""
    if not torch.is_grad_enabled():
        return grads
    there = []
    for g in grads:
        if g is not None and not any(g is t for t in there):
            there.append(g)
    out = _Once.apply(name, len(there), *there, *(t for t in inputs if t is not None))
    return tuple(None if g is None else next(o for o, t in zip(out, there) if t is g) for g in grads)
