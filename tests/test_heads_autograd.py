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
    # also behind hooks that would keep copies: a scheme's contexts go past them
    q, k = leaf * 1.0, leaf * 2.0
    with torch.autograd.graph.saved_tensors_hooks(lambda x: x.clone(), lambda x: x):
        y = heads.head_norm_rotate(q, k, t, t, _own=True)
    with torch.no_grad():
        q.add_(1.0)
    with pytest.raises(RuntimeError):
        (y[0].sum() + y[1].sum()).backward()


def test_a_buffer_of_another_layout_is_refused(monkeypatch):
    """A region that is computed again in the backward pass can come with other widths, and hooks can hand back anything: what
    does not hold this context is not read by its layout."""
    x = torch.zeros(1, 4, 2, 32)
    c = gact.make_head_context(x, 4, 32, 1)
    assert c.filled(c.blob.clone()).off == c.off
    for bad in (gact.make_head_context(x, 2, 32, 1).blob, gact.make_head_context(x, 8, 32, 1).blob, gact.make_head_context(x).blob,
                c.blob[:-1], c.blob.float(), torch.empty(2 * c.blob.numel(), dtype=torch.uint8)[::2], c.blob[:0]):
        with pytest.raises(ValueError):
            c.filled(bad)
    assert gact.make_head_context(x[:0], 4, 32, 1).filled(gact.make_head_context(x[:0], 4, 32, 1).blob).blob.numel() == 0
    # through autograd
    monkeypatch.setattr(heads, "gact_head_norm_rotate", lambda q, k, *a, **kw: (torch.ones_like(q), torch.ones_like(k)))
    q, t = torch.zeros(1, 4, 2, 32, requires_grad=True), torch.zeros(4, 16)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t[:-16] if t.dtype == torch.uint8 else t):
        y = heads.head_norm_rotate(q, q, t, t, bits=(4, 4), group_size=32)
    with pytest.raises(ValueError):
        y[0].sum().backward()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=str)
@pytest.mark.parametrize("Hq,Hk,D,G", [(16, 2, 64, 256), (2, 16, 64, 256), (4, 2, 80, 256)], ids=str)
def test_each_of_queries_and_keys_is_compressed(gact, Hq, Hk, D, G, dtype):
    """Slices of one projection under the controller, of which the group size fits one or none: the other is compressed by the
    hooks, nothing keeps the projection, and both gradients are those of what the contexts hold."""
    from paper_2206_11357_amd.hooks import Controller
    B, S = 2, 32
    g = torch.Generator("cuda").manual_seed(1)
    leaf = torch.randn(B, S, Hq + Hk, D, device="cuda", generator=g).to(dtype).requires_grad_(True)
    w = [(1 + 0.2 * torch.randn(D, device="cuda", generator=g)).requires_grad_(True) for _ in range(2)]
    angle = torch.rand(S, D // 16 * 8, device="cuda", generator=g)
    cos, sin = angle.cos(), angle.sin()
    ctl = Controller(w, group_size=G, bits=4, seed=3, min_numel=256)
    ctl.begin_iteration()
    projected = leaf * 1.0
    q, k = projected.detach()[:, :, :Hq].clone(), projected.detach()[:, :, Hq:].clone()
    held = StorageWeakRef(projected.untyped_storage())
    with ctl.hooks():
        yq, yk = ctl.head_norm_rotate(projected[:, :, :Hq], projected[:, :, Hq:], cos, sin, *w, by_head=True)
    own = [gact.head_context_fits(G, D, h) for h in (Hq, Hk)]
    del projected
    assert sum(own) < 2 and sorted(ctl.numel) == sorted((q.numel(), k.numel()))
    assert [h is not None for h in ctl._handles] == ([False] * sum(own) + [True] * (2 - sum(own)))
    dy = [torch.randn(y.shape, device="cuda", generator=g).to(dtype) for y in (yq, yk)]
    index = [0, 1] if own[0] == own[1] or own[0] else [1, 0]       # what the forward kernel compresses is numbered first
    seeds = [ctl.seed_of(i) for i in index]
    ctl._flush()
    assert held.expired()
    grads = torch.autograd.grad((yq, yk), [leaf, *w], dy)
    ctx, x = [], []
    for t, s, o in zip((q, k), seeds, own):
        ctx.append(gact.make_head_context(t, 4 if o else 32, G if o else 0, s))
        x.append(None if o else gact.gact_decompress(*gact.gact_compress(t.view(-1), G, 4, s), t.numel(), G, 4, dtype).view(t.shape))
    zq, zk = gact.gact_head_norm_rotate(q, k, cos, sin, *(t.detach() for t in w), context=ctx)
    assert torch.equal(yq, zq) and torch.equal(yk, zk)
    want = gact.gact_head_norm_rotate_backward(*dy, cos, sin, *(t.detach() for t in w), context=ctx, x=x)
    assert torch.equal(grads[0], torch.cat(want[:2], 2)) and torch.equal(grads[1], want[2]) and torch.equal(grads[2], want[3])
    # without gradients nothing is numbered, copied or kept
    before = len(ctl._handles)
    with torch.no_grad():
        assert torch.equal(ctl.head_norm_rotate(leaf[:, :, :Hq], leaf[:, :, Hq:], cos, sin, *w)[0], zq)
    assert len(ctl._handles) == before


@pytest.mark.gpu
def test_a_region_that_is_computed_twice(gact):
    """Under activation checkpointing the backward pass numbers the contexts anew; widths and seeds are those of the forward
    pass all the same, and so are the gradients."""
    from torch.utils.checkpoint import checkpoint
    from paper_2206_11357_amd.hooks import Controller
    g = torch.Generator("cuda").manual_seed(1)
    leaves = [torch.randn(2, 16, 4, 64, device="cuda", generator=g).requires_grad_(True) for _ in range(2)]
    angle = torch.rand(16, 32, device="cuda", generator=g)
    ctl = Controller(group_size=64, bits=4, seed=1, min_numel=16)

    def layer(q, k):
        q, k = ctl.head_norm_rotate(q * 1.0, k * 1.0, angle.cos(), angle.sin())
        return q * k, k

    def grads(run):
        ctl.set_iteration(0)
        ctl.begin_iteration()
        q, k = run(*run(*leaves))
        return torch.autograd.grad((q ** 2).sum() + (k ** 3).sum(), leaves)
    for bits in ({}, {0: 8, 1: 2, 2: 1, 3: 32, 4: 1, 5: 4, 6: 2, 7: 8}):
        ctl.bits = bits
        want = grads(layer)
        for a, b in zip(grads(lambda q, k: checkpoint(layer, q, k, use_reentrant=False)), want):
            assert torch.equal(a, b)
