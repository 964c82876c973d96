"""Differentiable form of ``gact_head_norm_rotate``: RMS norms of queries and
keys for each head with the position rotation, one launch forward, whose context
(queries and keys before the norm) is kept compressed (arXiv 2206.11357, Sec. 3.1:
the context Q(h) that the backward pass uses) and never written out decompressed.
No arithmetic here: every step runs in the library's kernels."""
from __future__ import annotations

from typing import Optional, Sequence

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import (GACT_BITS_UNCOMPRESSED, gact_head_norm_rotate, gact_head_norm_rotate_backward, make_head_context)


def _empty_by_head(x: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """Of x's shape [..., tokens, heads, head_dim], laid out head by head."""
    if x is None:
        return None
    shape = x.shape
    return torch.empty(*shape[:-3], shape[-2], shape[-3], shape[-1], dtype=x.dtype, device=x.device).transpose(-3, -2)


def _consecutive(dy: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    return dy if dy is None or dy.stride(-1) == 1 else dy.contiguous()


def _itself(x: torch.Tensor) -> torch.Tensor:
    return x


class _HeadNormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, wq, wk, cos, sin, positions, eps, interleaved, by_head, bits, group_size, seeds, own):
        ctx.set_materialize_grads(False)
        context = [x if x is None else make_head_context(x, b, group_size if b != GACT_BITS_UNCOMPRESSED else 0, s)
                   for x, b, s in zip((q, k), bits, seeds)]
        out = (_empty_by_head(q), _empty_by_head(k)) if by_head else None
        yq, yk = gact_head_norm_rotate(q, k, cos, sin, wq, wk, positions, eps, interleaved, out=out, context=context)
        # The contexts too are kept as autograd keeps what it needs, so that they go after the backward pass.
        kept = (*(x if b == GACT_BITS_UNCOMPRESSED else None for x, b in zip((q, k), bits)), wq, wk, cos, sin, positions)
        ctx.save_for_backward(*kept, *(c if c is None else c.blob for c in context))
        ctx.versions = [t if t is None else t._version for t in kept] if own else ()
        for c in context:
            if c is not None:
                c.blob = None
        ctx.context, ctx.interleaved = context, interleaved
        return yq, yk

    @staticmethod
    @once_differentiable
    def backward(ctx, dyq, dyk):
        kept = ctx.saved_tensors
        if any(t is not None and t._version != v for t, v in zip(kept, ctx.versions)):
            raise RuntimeError("what the backward pass of head_norm_rotate needs was modified in place")
        q, k, wq, wk, cos, sin, positions, *blobs = kept
        need = ctx.needs_input_grad
        grads = gact_head_norm_rotate_backward(
            _consecutive(dyq), _consecutive(dyk), cos, sin, wq, wk, positions,
            context=[c if c is None else c.filled(blob) for c, blob in zip(ctx.context, blobs)], x=(q, k),
            interleaved=ctx.interleaved, weight_grads=need[2:4])
        return (*(g if n else None for g, n in zip(grads, need)), *(None,) * 10)


def _refuse_tangents(*tensors: Optional[torch.Tensor]) -> None:
    """The kernels pass no forward-mode derivatives on, and a result without one would stand for zero."""
    if getattr(forward_ad, "_current_level", 0) >= 0 and any(
            t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise NotImplementedError("head_norm_rotate has no forward-mode derivative")


def head_norm_rotate(q: torch.Tensor, k: Optional[torch.Tensor], cos: Optional[torch.Tensor], sin: Optional[torch.Tensor],
                     wq: Optional[torch.Tensor] = None, wk: Optional[torch.Tensor] = None,
                     positions: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                     by_head: bool = False, bits: Sequence[int] = (GACT_BITS_UNCOMPRESSED, GACT_BITS_UNCOMPRESSED),
                     group_size: int = 0, seeds: Sequence[int] = (0, 0), _own: bool = False):
    """``gact_head_norm_rotate`` with gradients for q, k, wq and wk.  by_head: the results lie head by head
    ([..., heads, tokens, head_dim] in memory, of q's shape), as attention reads them.  bits: widths of the contexts of q
    and k, in groups of group_size with the noise of `seeds`; GACT_BITS_UNCOMPRESSED keeps the tensor itself through
    autograd.  ``Controller.head_norm_rotate`` chooses them from its scheme.  Reverse mode, once: forward-mode tangents and
    second derivatives are refused."""
    _refuse_tangents(q, k, wq, wk, cos, sin)
    if not (torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (q, k, wq, wk))):
        out = (_empty_by_head(q), _empty_by_head(k)) if by_head else None
        return gact_head_norm_rotate(q, k, cos, sin, wq, wk, positions, eps, interleaved, out=out)
    args = (q, k, wq, wk, cos, sin, positions, eps, interleaved, by_head, tuple(bits), group_size, tuple(seeds), _own)
    if not _own:
        return _HeadNormRotate.apply(*args)
    # Contexts that a scheme has numbered: past all hooks, the scheme's own, which would number them again, and those of a region that
    # is computed twice, whose second time has other numbers.  (Autograd looks at no versions where there are hooks: backward does.)
    with torch.autograd.graph.saved_tensors_hooks(_itself, _itself):
        return _HeadNormRotate.apply(*args)
