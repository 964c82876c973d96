"""Differentiable layers whose context is kept compressed (arXiv 2206.11357, Sec. 3.1: the context Q(h) that the backward
pass uses) and read as codes, never written out decompressed: a linear layer, whose weight gradient is
``gact_linear_weight_grad``, and ``gact_group_norm`` with an activation.  No arithmetic here: the steps run in the library's
kernels, the linear layer's other two products in torch's."""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import (GACT_BITS_UNCOMPRESSED, _map_strides, _rows, gact_compress, gact_group_norm, gact_group_norm_backward,
               gact_linear_weight_grad, make_group_norm_context)
from .heads import _itself, _refuse_tangents


def _changed(kept, versions) -> bool:
    return any(t is not None and t._version != v for t, v in zip(kept, versions))


def _versions(kept) -> list:
    return [t if t is None else t._version for t in kept]


def _laid_out(t: torch.Tensor, strides) -> torch.Tensor:
    """t, copied where its layout is not one that `strides` takes."""
    try:
        strides(t)
    except ValueError:
        return t.contiguous()
    return t


# ----------------------------------------------------------------- linear layer
class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, bits, group_size, seed, own):
        kept = x.contiguous()
        if kept.data_ptr() % 16:                # a view that begins inside 16 bytes, which the compressor loads at a time
            kept = kept.clone()
        context = gact_compress(kept, group_size, bits, seed)
        ctx.save_for_backward(weight, *context)
        ctx.versions = [weight._version] if own else ()
        ctx.bits, ctx.group_size, ctx.shape = bits, group_size, x.shape
        return torch.nn.functional.linear(x, weight, bias)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        weight, *context = ctx.saved_tensors
        if _changed((weight,), ctx.versions):
            raise RuntimeError("what the backward pass of linear needs was modified in place")
        need = ctx.needs_input_grad
        dy = _laid_out(dy, _rows)
        dx = torch.mm(dy.reshape(-1, dy.shape[-1]), weight).view(ctx.shape) if need[0] else None
        dw = db = None
        if need[1] or need[2]:
            dw, db = gact_linear_weight_grad(dy, *context, ctx.shape[-1], ctx.group_size, ctx.bits, w_dtype=weight.dtype,
                                             bias=need[2])
        return dx, dw if need[1] else None, db, None, None, None, None


def linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, bits: int = GACT_BITS_UNCOMPRESSED,
           group_size: int = 256, seed: int = 0, _own: bool = False) -> torch.Tensor:
    """``torch.nn.functional.linear`` of x, [..., in_features] in float32 or bfloat16, whose context (x) is kept compressed in
    `bits` bits, in groups of group_size with the noise of `seed`; with GACT_BITS_UNCOMPRESSED it is that function.
    ``Controller.linear`` chooses them from its scheme.  x, weight and bias have one type (under autocast: are cast to its
    type first).  Reverse mode, once: forward-mode tangents and second derivatives are refused."""
    if bits == GACT_BITS_UNCOMPRESSED or not (torch.is_grad_enabled() and weight.requires_grad):
        return torch.nn.functional.linear(x, weight, bias)
    _refuse_tangents(x, weight, bias, of="linear")
    if torch.is_autocast_enabled("cuda"):
        dtype = torch.get_autocast_dtype("cuda")
        x, weight, bias = x.to(dtype), weight.to(dtype), bias if bias is None else bias.to(dtype)
    if weight.dtype != x.dtype or (bias is not None and bias.dtype != x.dtype):
        raise ValueError("x, weight and bias must have one type, got %s, %s%s"
                         % (x.dtype, weight.dtype, "" if bias is None else ", %s" % bias.dtype))
    if x.dim() < 2:
        raise ValueError("gact needs [..., features]")
    args = (x, weight, bias, bits, group_size, seed, _own)
    with torch.autocast("cuda", enabled=False):
        if not _own:
            return _Linear.apply(*args)
        with torch.autograd.graph.saved_tensors_hooks(_itself, _itself):
            return _Linear.apply(*args)


# ------------------------------------------------------------------- group norm
class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, b, groups, eps, act, bits, group_size, seed, own):
        context = make_group_norm_context(x, groups, bits, group_size if bits != GACT_BITS_UNCOMPRESSED else 0, seed)
        y = gact_group_norm(x, groups, w, b, eps, act, context=context)
        # the context too is kept as autograd keeps what it needs, so that it goes after the backward pass
        kept = (x if bits == GACT_BITS_UNCOMPRESSED else None, w, b)
        ctx.save_for_backward(*kept, context.blob)
        ctx.versions = _versions(kept) if own else ()
        context.blob = None
        ctx.context, ctx.groups, ctx.act = context, groups, act
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        *kept, blob = ctx.saved_tensors
        if _changed(kept, ctx.versions):
            raise RuntimeError("what the backward pass of group_norm needs was modified in place")
        x, w, b = kept
        need = ctx.needs_input_grad
        dx, dw, db = gact_group_norm_backward(_laid_out(dy, _map_strides), ctx.groups, w, b, ctx.act,
                                              context=ctx.context.filled(blob), x=x, weight_grads=need[1:3])
        return (dx if need[0] else None, dw, db, *(None,) * 7)


def group_norm(x: torch.Tensor, groups: int, w: Optional[torch.Tensor] = None, b: Optional[torch.Tensor] = None,
               eps: float = 1e-5, act: str = "none", bits: int = GACT_BITS_UNCOMPRESSED, group_size: int = 0, seed: int = 0,
               _own: bool = False) -> torch.Tensor:
    """``gact_group_norm`` with gradients for x, w and b.  bits: width of the context, in groups of group_size with the
    noise of `seed`; GACT_BITS_UNCOMPRESSED keeps x itself through autograd.  ``Controller.group_norm`` chooses them from its
    scheme.  Reverse mode, once: forward-mode tangents and second derivatives are refused, and channels that are no multiple
    of eight and of the groups."""
    if groups < 1 or x.dim() == 0 or x.shape[-1] % 8 or x.shape[-1] % groups:
        raise ValueError("the channels must be a multiple of eight and of the groups, got %s in %d groups" % (tuple(x.shape), groups))
    _refuse_tangents(x, w, b, of="group_norm")
    if not (torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, w, b))):
        return gact_group_norm(x, groups, w, b, eps, act)
    args = (x, w, b, groups, eps, act, bits, group_size, seed, _own)
    if not _own:
        return _GroupNorm.apply(*args)
    # A context that a scheme has numbered: past all hooks (as head_norm_rotate's).
    with torch.autograd.graph.saved_tensors_hooks(_itself, _itself):
        return _GroupNorm.apply(*args)
