"""The autograd form of the head norms: what it refuses, and what it keeps for how long."""
import pytest
import torch
from torch.autograd import forward_ad

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
