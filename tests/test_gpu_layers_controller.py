"""What a controller's layers do with inputs that they do not take as they are."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2206_11357_amd as gact
from paper_2206_11357_amd import layers
from paper_2206_11357_amd.hooks import Controller

pytestmark = pytest.mark.gpu


def refused_calls():
    x = torch.randn(2, 9, 64, device="cuda", requires_grad=True)
    odd = torch.randn(2, 9, 60, device="cuda", requires_grad=True)
    w = torch.randn(16, 64, device="cuda", requires_grad=True)
    n = torch.ones(64, device="cuda", requires_grad=True)
    return [lambda c: c.group_norm(odd, 4), lambda c: c.group_norm(x, 7), lambda c: c.group_norm(x, 8, n[:32]),
            lambda c: c.group_norm(x, 8, n, act="relu"), lambda c: c.group_norm(x, 8, n, eps=-1.0), lambda c: c.group_norm(x.view(18, 64), 8),
            lambda c: c.linear(x, w[:, :32]), lambda c: c.linear(x, w.bfloat16()), lambda c: c.linear(x, w, n)]


@pytest.mark.parametrize("bits", [4, gact.GACT_BITS_UNCOMPRESSED])
@pytest.mark.parametrize("which", range(9))
def test_a_refused_call_leaves_the_scheme_as_it_was(which, bits):
    """The context tensors behind it keep their numbers, and with them their widths and seeds."""
    ctl = Controller(group_size=64, bits=bits, min_numel=64)
    ctl.begin_iteration()
    with ctl.hooks():
        with pytest.raises((ValueError, RuntimeError)):
            refused_calls()[which](ctl)
        assert ctl.numel == [] and ctl._handles == []
        x = torch.randn(2, 9, 64, device="cuda", requires_grad=True)
        y = ctl.group_norm(x, 8)
    assert ctl.numel == [x.numel()] and len(ctl._handles) == 1
    other = Controller(group_size=64, bits=bits, min_numel=64)
    other.begin_iteration()
    with other.hooks():
        z = other.group_norm(x, 8)
    g = torch.randn_like(y)
    assert torch.equal(*(torch.autograd.grad(t, x, g)[0] for t in (y, z)))


@pytest.mark.parametrize("group_size", [64, 96])
@pytest.mark.parametrize("bits", [8, gact.GACT_BITS_UNCOMPRESSED])
def test_pixels_of_any_spacing(bits, group_size):
    """A crop of a larger map, whose rows of pixels lie apart, is laid out first, as the linear layer lays out its input."""
    big = torch.randn(2, 9, 11, 64, device="cuda", requires_grad=True)
    n = torch.ones(64, device="cuda", requires_grad=True)
    g = torch.randn(2, 5, 6, 64, device="cuda")
    results = []
    for lay in (lambda t: t, lambda t: t.contiguous()):
        ctl = Controller([n], group_size=group_size, bits=bits, seed=3, min_numel=64)
        ctl.begin_iteration()
        with ctl.hooks():
            y = ctl.group_norm(lay(big[:, 2:7, 3:9]), 8, n, act="silu")
        assert ctl.numel == [2 * 5 * 6 * 64]
        results.append((y, *torch.autograd.grad(y, (big, n), g)))
    assert all(torch.equal(u, v) for u, v in zip(*results))
    with torch.no_grad():
        assert torch.equal(ctl.group_norm(big[:, 2:7, 3:9], 8, n, act="silu"), results[0][0])
    small = Controller(group_size=64, bits=4, min_numel=1 << 20)
    assert torch.equal(small.group_norm(big[:, 2:7, 3:9], 8, n, act="silu"), results[0][0]) and small.numel == []


def test_channels_that_the_norm_does_not_take():
    """No multiple of eight, or of the groups: refused by their name, by the controller too, whatever its group size."""
    for group_size in (64, 96):
        ctl = Controller(group_size=group_size, bits=4, min_numel=64)
        ctl.begin_iteration()
        for channels, groups in ((60, 4), (64, 7), (64, 0), (64, -8), (64, 128)):
            x = torch.randn(2, 9, channels, device="cuda", requires_grad=True)
            for call in (ctl.group_norm, layers.group_norm):
                with ctl.hooks(), pytest.raises(ValueError, match="multiple of eight and of the groups"):
                    call(x, groups)
                with torch.no_grad(), pytest.raises(ValueError, match="multiple of eight and of the groups"):
                    call(x, groups)
        assert ctl.numel == []


def test_parameters_are_left_alone():
    """A parameter that is a layer's input (learned queries) is no context tensor: the hooks do not compress it either."""
    query = torch.randn(2, 9, 64, device="cuda", requires_grad=True)
    w = torch.randn(16, 64, device="cuda", requires_grad=True)
    ctl = Controller([query, w], group_size=64, bits=1, min_numel=64)
    ctl.begin_iteration()
    with ctl.hooks():
        y, z = ctl.linear(query, w), ctl.group_norm(query, 8)
    assert ctl.numel == []
    g = torch.randn_like(y)
    assert torch.equal(torch.autograd.grad(y, w, g)[0], torch.autograd.grad(torch.nn.functional.linear(query, w), w, g)[0])
    g = torch.randn_like(z)
    assert torch.equal(torch.autograd.grad(z, query, g)[0], torch.autograd.grad(layers.group_norm(query, 8), query, g)[0])


@pytest.mark.parametrize("reentrant", [False, True])
def test_values_of_regions_that_are_computed_twice(reentrant):
    """A checkpointed region's input is a context tensor of the hooks', the first; a reentrant one's second run begins with what was
    compressed of it, and makes the contexts; else the first run makes them."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(2, 30, 64, generator=gen, device="cuda", requires_grad=True)
    w = torch.randn(96, 64, generator=gen, device="cuda", requires_grad=True)
    n = torch.randn(96, generator=gen, device="cuda", requires_grad=True)
    ctl = Controller([w, n], group_size=64, bits=4, seed=4, min_numel=64)
    ctl.begin_iteration()
    with ctl.hooks():
        y = checkpoint(lambda t: ctl.group_norm(ctl.linear(t, w), 12, n, act="silu"), x, use_reentrant=reentrant)
    g = torch.randn(y.shape, generator=gen, device="cuda")
    y.backward(g)
    assert ctl.numel == [x.numel(), x.numel(), y.numel()]
    with torch.no_grad():
        if reentrant:
            x.copy_(gact.gact_decompress(*gact.gact_compress(x, 64, 4, ctl.seed_of(0)), x.numel(), 64, 4).view_as(x))
        a = torch.nn.functional.linear(x, w)
        context = gact.make_group_norm_context(a, 12, 4, 64, ctl.seed_of(2))
        again = gact.gact_group_norm(a, 12, n, act="silu", context=context)
        assert reentrant or torch.equal(again, y)
        da, dn, _ = gact.gact_group_norm_backward(g, 12, n, act="silu", context=context)
        dw, _ = gact.gact_linear_weight_grad(da, *gact.gact_compress(x, 64, 4, ctl.seed_of(1)), 64, 64, 4)
        assert torch.equal(n.grad, dn) and torch.equal(w.grad, dw)
        assert torch.equal(x.grad, torch.mm(da.view(60, 96), w).view_as(x))
