"""The autograd form of the head norms: what it refuses, and what it keeps for how long."""
import contextlib

import pytest
import torch
from torch.autograd import forward_ad
from torch.multiprocessing.reductions import StorageWeakRef

import paper_2206_11357_amd as gact
from paper_2206_11357_amd import heads


@pytest.mark.parametrize("which", range(6))
@pytest.mark.parametrize("grad", (False, True))
def test_forward_mode_tangents_are_refused(monkeypatch, which, grad):
    """In whichever input they come, whether or not a gradient is wanted too: a result without a tangent would mean that the
    derivative is zero.  (Nothing is launched: the raw call hands its inputs back.)"""
    monkeypatch.setattr(heads, "gact_head_norm_rotate", lambda q, k, *a, **kw: (q.detach().clone(), k.detach().clone()))
    q, k = torch.zeros(1, 3, 2, 16), torch.zeros(1, 3, 1, 16)
    args = [q, k, torch.ones(3, 8), torch.zeros(3, 8), torch.ones(16), torch.ones(16)]
    heads.head_norm_rotate(*args)
    with forward_ad.dual_level():
        heads.head_norm_rotate(*args)                              # a level, but no tangents
        if grad:
            args[which].requires_grad_(True)
        args[which] = forward_ad.make_dual(args[which], torch.ones_like(args[which]))
        with pytest.raises(NotImplementedError):
            heads.head_norm_rotate(*args)
        with torch.no_grad(), pytest.raises(NotImplementedError):
            heads.head_norm_rotate(*args)


def test_transforms_of_functions_are_refused():
    """torch.func's own derivatives and batching."""
    q, k, t = torch.zeros(1, 3, 2, 16), torch.zeros(1, 3, 1, 16), torch.zeros(3, 8)
    with pytest.raises(Exception):
        torch.func.jvp(lambda x: heads.head_norm_rotate(x, k, t, t)[0], (q,), (q,))
    with pytest.raises(Exception):
        torch.func.vmap(lambda x: heads.head_norm_rotate(x, k, t, t)[0])(q)


@pytest.mark.parametrize("hooked", (False, True))
@pytest.mark.parametrize("own", (False, True))
@pytest.mark.parametrize("bits", ((4, 4), (32, 32), (2, 32)))
def test_contexts_go_with_the_backward_pass(monkeypatch, bits, own, hooked):
    """Compressed contexts, statistics and queries kept as they are: alive as long as a graph is retained, gone after the
    backward pass though the loss is held.  (Nothing is launched.)"""
    kept = []

    def make(x, *a, **kw):
        c = gact.make_head_context(x, *a, **kw)
        kept.append(StorageWeakRef(c.blob.untyped_storage()))
        return c
    seen = []

    def backward(dyq, dyk, *a, context, x, **kw):
        for c, t, b in zip(context, x, bits):
            assert c.blob is not None and c.bits == b and (t is None) == (b != 32)
            assert c.rstd.shape == c.shape[:-1] and c.rstd.data_ptr() % 4 == 0
        seen.append([c.addresses() for c in context])
        return torch.zeros_like(dyq), torch.zeros_like(dyk), None, None
    monkeypatch.setattr(heads, "make_head_context", make)
    monkeypatch.setattr(heads, "gact_head_norm_rotate", lambda q, k, *a, **kw: (torch.ones_like(q), torch.ones_like(k)))
    monkeypatch.setattr(heads, "gact_head_norm_rotate_backward", backward)
    leaf = torch.ones(2, 5, 6, 32, requires_grad=True)
    t = torch.ones(5, 16)

    def loss_of():
        projected = leaf * 2.0                          # what queries and keys are views of
        kept.append(StorageWeakRef(projected.untyped_storage()))
        y = heads.head_norm_rotate(projected[:, :, :4], projected[:, :, 4:], t, t, bits=bits, group_size=32, _own=own)
        return y[0].sum() + y[1].sum()
    with torch.autograd.graph.saved_tensors_hooks(lambda x: x, lambda x: x) if hooked else contextlib.nullcontext():
        loss = loss_of()
    assert len(kept) == 3 and [r.expired() for r in kept] == [32 not in bits, False, False]
    loss.backward(retain_graph=True)
    assert [r.expired() for r in kept] == [32 not in bits, False, False]
    loss.backward()
    assert seen[0] == seen[1]
    assert all(r.expired() for r in kept) and loss.grad_fn is not None
    with pytest.raises(RuntimeError):
        loss.backward()


@pytest.mark.parametrize("hooked", (False, True))
def test_modified_queries_are_noticed_with_and_without_hooks(monkeypatch, hooked):
    monkeypatch.setattr(heads, "gact_head_norm_rotate", lambda q, k, *a, **kw: (torch.ones_like(q), torch.ones_like(k)))
    monkeypatch.setattr(heads, "gact_head_norm_rotate_backward",
                        lambda dyq, dyk, *a, **kw: (torch.zeros_like(dyq), torch.zeros_like(dyk), None, None))
    leaf, t = torch.ones(2, 5, 4, 32, requires_grad=True), torch.ones(5, 16)
    for modified in (False, True):
        q, k = leaf * 1.0, leaf * 2.0
        q.add_(1.0)                                     # before: of no account
        with torch.autograd.graph.saved_tensors_hooks(lambda x: x, lambda x: x) if hooked else contextlib.nullcontext():
            y = heads.head_norm_rotate(q, k, t, t, _own=True)
        if modified:
            with torch.no_grad():
                k.add_(1.0)
            with pytest.raises(RuntimeError):
                (y[0].sum() + y[1].sum()).backward()
        else:
            (y[0].sum() + y[1].sum()).backward()
    # hooks that keep a copy: what they give back is what was there
    q, k = leaf * 1.0, leaf * 2.0
    q.add_(1.0)
    with torch.autograd.graph.saved_tensors_hooks(lambda x: x.clone(), lambda x: x):
        y = heads.head_norm_rotate(q, k, t, t, _own=True)
    with torch.no_grad():
        q.add_(1.0)
    (y[0].sum() + y[1].sum()).backward()
