"""Norms of heads with the position rotation, their compressed context and their gradients, against the formulas in 64
bits.  u = 2^-24 is half a step of binary32.  The bounds count roundings; each is relative to the magnitudes that its
sum is made of:
  r     a row's sum of squares: 8 fused steps and at most 6 lane steps, the mean and eps 2; the root halves that, root and
        division add 2: 10 u
  y     r, two products, product and fused step of the rotation: 14 u of |n_a cos| + |n_b sin|; then half a step of the type
  dx    with G = (|dy_a cos| + |dy_b sin|) |w| and X = |x r|: g 4 u; its sum with x r (11 u) 8 + 6 + 1 steps; the last
        product and fused step 12 u and more: below 64 u of r (G + X mean(G X)); then half a step of the type
  dw    a term 16 u; at most `run` fused steps in a lane, 64 x 4 additions in the block, binary64 behind: below
        (run + 300) u of the sum of |dn| X
"""
import math

import numpy as np
import pytest
import torch

import oracle
import synthetic_inputs as syn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
EPS = 1e-6


def rng(seed):
    return torch.Generator("cuda").manual_seed(seed)


def randn(seed, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, device="cuda", generator=rng(seed)) * scale).to(dtype)


def tables(n, rot, seed=0):
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1))
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * f + 0.1 * seed
    return a.cos().float(), a.sin().float()


class Formula:
    """One tensor's forward and backward pass in 64 bits, and the magnitudes behind the bounds."""

    def __init__(self, x, w, cos, sin, positions, interleaved, eps=EPS):
        B, S, H, D = x.shape
        self.x, self.D = x.double(), D
        self.w = torch.ones(D, dtype=torch.float64, device="cuda") if w is None else w.double()
        R = 2 * cos.shape[1] if cos is not None else 0
        i = torch.arange(R // 2, device="cuda")
        self.a, self.b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        p = (torch.arange(S, device="cuda").expand(B, S) if positions is None else positions.view(B, S))
        if R:
            self.c, self.s = cos.double()[p][:, :, None], sin.double()[p][:, :, None]
        self.R = R
        self.r = ((self.x ** 2).mean(-1, keepdim=True) + eps) ** -0.5

    def turned(self, n, back=False, magnitude=False):
        if self.R == 0:
            return n.abs() if magnitude else n
        y = n.abs().clone() if magnitude else n.clone()
        na, nb, c, s = n[..., self.a], n[..., self.b], self.c, -self.s if back else self.s
        if magnitude:
            y[..., self.a] = (na * c).abs() + (nb * s).abs()
            y[..., self.b] = (nb * c).abs() + (na * s).abs()
        else:
            y[..., self.a], y[..., self.b] = na * c - nb * s, nb * c + na * s
        return y

    def check_forward(self, y):
        n = self.x * self.r * self.w
        want, size = self.turned(n), self.turned(n, magnitude=True)
        err = (y.double() - want).abs()
        assert (err <= 16 * U * size + HALF[y.dtype] * want.abs() * (1 + 1e-3) + 1e-38).all(), float((err / (size + 1e-30)).max())

    def check_backward(self, dy, dx, dw=None, x=None, run=1):
        x = self.x if x is None else x.double()
        dn, mag = self.turned(dy.double(), back=True), self.turned(dy.double(), back=True, magnitude=True)
        xr = x * self.r
        g, G, X = dn * self.w, mag * self.w.abs(), xr.abs()
        want = self.r * (g - xr * (g * xr).mean(-1, keepdim=True))
        size = self.r * (G + X * (G * X).mean(-1, keepdim=True))
        err = (dx.double() - want).abs()
        assert (err <= 64 * U * size + HALF[dx.dtype] * want.abs() * (1 + 1e-3) + 1e-38).all(), float((err / (size + 1e-30)).max())
        if dw is not None:
            want, size = (dn * xr).sum((0, 1, 2)), (mag * X).sum((0, 1, 2))
            err = (dw.double() - want).abs()
            assert (err <= (run + 300) * U * size + HALF[dw.dtype] * want.abs() * (1 + 1e-3) + 1e-38).all(), float((err / size).max())


CASES = [
    # B, S, Hq, Hk, D, rot, dtype, weights, interleaved
    (1, 1, 1, 1, 8, 0, "f32", "f32", False),
    (1, 1, 4, 2, 64, 64, "bf16", "bf16", False),
    (3, 7, 5, 3, 16, 16, "f32", None, True),
    (2, 33, 12, 1, 80, 32, "bf16", "bf16", False),
    (1, 129, 3, 1, 96, 96, "f32", "bf16", False),
    (2, 65, 8, 8, 128, 128, "bf16", "f32", False),
    (2, 65, 8, 2, 128, 64, "f32", "f32", True),
    (4, 5, 2, 1, 256, 256, "bf16", "f32", True),
    (1, 19, 3, 2, 512, 512, "f32", "f32", False),
    (1, 19, 3, 2, 504, 496, "bf16", None, False),
    (5, 3, 7, 7, 40, 32, "bf16", "bf16", True),
    (1, 2100, 6, 2, 64, 64, "bf16", "f32", False),
]
DT = {"f32": torch.float32, "bf16": torch.bfloat16, None: None}


def inputs(case, seed=1, layout="contiguous"):
    B, S, Hq, Hk, D, rot, dtype, weights, interleaved = case
    dt = DT[dtype]
    if layout == "contiguous":
        q, k = randn(seed, B, S, Hq, D, dtype=dt, scale=1.5), randn(seed + 1, B, S, Hk, D, dtype=dt, scale=0.7)
    elif layout == "fused":                           # slices of one projection's output, one element behind a line
        row = (Hq + 2 * Hk) * D + 3
        flat = randn(seed, B * S * row + 1, dtype=dt)[1:]
        x = flat.as_strided((B, S, Hq + 2 * Hk, D), (S * row, row, D, 1), flat.storage_offset())
        q, k = x[:, :, :Hq], x[:, :, Hq:Hq + Hk]
    else:                                             # head by head
        q, k = (randn(seed + j, B, H, S, D, dtype=dt).transpose(1, 2) for j, H in enumerate((Hq, Hk)))
    w = [None if weights is None else randn(seed + 5 + j, D, dtype=DT[weights], scale=0.3) + 1 for j in range(2)]
    cos, sin = tables(S + 3, rot) if rot else (None, None)
    positions = torch.randint(0, S + 3, (B, S), device="cuda", generator=rng(seed + 9)) if rot and seed % 2 else None
    return q, k, cos, sin, w[0], w[1], positions


@pytest.mark.parametrize("layout", ("contiguous", "fused", "by_head"))
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward_and_backward_against_the_formula(gact, case, layout):
    B, S, Hq, Hk, D, rot, dtype, weights, inter = case
    q, k, cos, sin, wq, wk, pos = args = inputs(case, 1 if layout != "by_head" else 2, layout)
    ctx = tuple(gact.make_head_context(x) for x in (q, k))
    by_head = tuple(torch.empty(B, x.shape[2], S, D, dtype=x.dtype, device="cuda").transpose(1, 2) for x in (q, k))
    out = by_head if layout == "by_head" else None
    yq, yk = gact.gact_head_norm_rotate(*args, eps=EPS, interleaved=inter, out=out, context=ctx)
    dyq, dyk = (randn(30 + j, *x.shape, dtype=x.dtype) for j, x in enumerate((q, k)))
    if layout == "by_head":
        dyq, dyk = (torch.empty_like(o).copy_(d) for o, d in zip(by_head, (dyq, dyk)))
    dq, dk, dwq, dwk = gact.gact_head_norm_rotate_backward(dyq, dyk, cos, sin, wq, wk, pos, context=ctx, x=(q, k),
                                                           interleaved=inter)
    for x, w, y, dy, dx, dw in ((q, wq, yq, dyq, dq, dwq), (k, wk, yk, dyk, dk, dwk)):
        f = Formula(x, w, cos, sin, pos, inter)
        f.check_forward(y)
        f.check_backward(dy, dx, dw)
    # without a context and without keys: the same values
    only, none = gact.gact_head_norm_rotate(q, None, cos, sin, wq, None, pos, eps=EPS, interleaved=inter)
    assert none is None and torch.equal(only, yq.contiguous())


CONTEXTS = [
    # D, G, Hq, Hk: groups that are parts of a head, heads, several heads
    (64, 32, 4, 1), (64, 64, 3, 1), (64, 256, 8, 4), (64, 512, 16, 8), (128, 128, 4, 2), (128, 256, 4, 2), (96, 32, 2, 1),
    (96, 96, 3, 1), (96, 192, 4, 2), (80, 320, 8, 4), (16, 32, 2, 4), (16, 512, 32, 32), (256, 64, 1, 1), (512, 512, 2, 1),
    (512, 256, 1, 1), (160, 160, 3, 1), (8, 512, 64, 64), (40, 160, 4, 8),
]


@pytest.mark.parametrize("bits", (1, 2, 4, 8))
@pytest.mark.parametrize("D,G,Hq,Hk", CONTEXTS)
def test_the_context_is_what_the_compressor_gives(gact, D, G, Hq, Hk, bits):
    """Codes, minima, steps and pad bytes equal gact_compress's (and the oracle's) of the same elements laid out
    contiguously; the gradients are those of the decompressed values."""
    assert gact.head_context_fits(G, D, Hq, Hk)
    dtype = torch.float32 if (D // 8 + bits) % 2 else torch.bfloat16
    B, S, rot = 2, 11, D // 16 * 16
    q, k, cos, sin, wq, wk, pos = inputs((B, S, Hq, Hk, D, rot, "f32" if dtype == torch.float32 else "bf16", "f32", bits == 2),
                                         3, "fused")
    q[0, 3] = 0.25                                     # constant groups
    if Hq > 1:
        q[1, 4, 1] = 0.0
    ctx = [gact.make_head_context(x, bits, G, seed) for x, seed in ((q, (1 << 63) + 5), (k, 77))]
    for c in ctx:
        for t in (c.packed, c.gmin, c.gscale):
            t.view(torch.uint8).fill_(0xA5)
    yq, yk = gact.gact_head_norm_rotate(q, k, cos, sin, wq, wk, pos, interleaved=bits == 2, context=ctx)
    dyq, dyk = (randn(40 + j, *x.shape, dtype=dtype) for j, x in enumerate((q, k)))
    grads = gact.gact_head_norm_rotate_backward(dyq, dyk, cos, sin, wq, wk, pos, context=ctx, interleaved=bits == 2)
    for x, c, y, w, dy, dx, dw in zip((q, k), ctx, (yq, yk), (wq, wk), (dyq, dyk), grads[:2], grads[2:]):
        flat = x.contiguous().view(-1)
        p, mn, sc = gact.gact_compress(flat, G, bits, c.seed)
        assert torch.equal(c.packed, p)
        assert torch.equal(c.gmin.view(torch.int32), mn.view(torch.int32))
        assert torch.equal(c.gscale.view(torch.int32), sc.view(torch.int32))
        x_np = flat.cpu().numpy() if dtype == torch.float32 else flat.cpu().view(torch.int16).numpy().view(np.uint16)
        p_ref, mn_ref, sc_ref = oracle.compress(x_np, G, bits, c.seed)
        assert np.array_equal(p.cpu().numpy(), p_ref) and np.array_equal(mn.cpu().numpy(), mn_ref)
        f = Formula(x, w, cos, sin, pos, bits == 2)
        f.check_forward(y)
        held = gact.gact_decompress(c.packed, c.gmin, c.gscale, flat.numel(), G, bits).view(x.shape)
        f.check_backward(dy, dx, dw, x=held)


def test_parts_of_different_widths_and_an_uncompressed_one(gact):
    case = (2, 40, 4, 2, 64, 64, "bf16", "f32", False)
    q, k, cos, sin, wq, wk, pos = inputs(case)
    dyq, dyk = (randn(50 + j, *x.shape, dtype=x.dtype) for j, x in enumerate((q, k)))
    for bq, bk in ((2, 4), (32, 8), (1, 32)):
        ctx = [gact.make_head_context(x, b, 64 if b != 32 else 0, 9) for x, b in ((q, bq), (k, bk))]
        yq, yk = gact.gact_head_norm_rotate(q, k, cos, sin, wq, wk, pos, context=ctx)
        grads = gact.gact_head_norm_rotate_backward(dyq, dyk, cos, sin, wq, wk, pos, context=ctx, x=(q, k))
        for x, c, b, y, w, dy, dx, dw in zip((q, k), ctx, (bq, bk), (yq, yk), (wq, wk), (dyq, dyk), grads[:2], grads[2:]):
            held = None
            if b != 32:
                p, mn, sc = gact.gact_compress(x.contiguous().view(-1), 64, b, 9)
                assert torch.equal(c.packed, p) and torch.equal(c.gmin, mn) and torch.equal(c.gscale, sc)
                held = gact.gact_decompress(p, mn, sc, x.numel(), 64, b).view(x.shape)
            f = Formula(x, w, cos, sin, pos, False)
            f.check_forward(y)
            f.check_backward(dy, dx, dw, x=held)
    # one part alone, and no weight gradients: the other results stay what they were
    dq, none, dwq, none_w = gact.gact_head_norm_rotate_backward(dyq, None, cos, sin, wq, wk, pos, context=ctx, x=(q, k),
                                                                weight_grads=(False, False))
    assert torch.equal(dq, grads[0]) and none is None and dwq is None and none_w is None


def test_gradients_against_difference_quotients(gact):
    """Central differences of the formula in 64 bits along random directions: the quotient is off by h^2 times a third
    derivative, about 1e-8, beside the kernels' bounds."""
    case = (1, 6, 2, 1, 32, 32, "f32", "f32", False)
    q, k, cos, sin, wq, wk, pos = inputs(case)
    ctx = tuple(gact.make_head_context(x) for x in (q, k))
    gact.gact_head_norm_rotate(q, k, cos, sin, wq, wk, pos, context=ctx)
    dyq, dyk = (randn(60 + j, *x.shape) for j, x in enumerate((q, k)))
    dq, dk, dwq, dwk = gact.gact_head_norm_rotate_backward(dyq, dyk, cos, sin, wq, wk, pos, context=ctx, x=(q, k))

    def loss(x, w, dy):
        f = Formula(x, w, cos, sin, pos, False)
        return float((f.turned(f.x * f.r * f.w) * dy.double()).sum())
    h = 1e-4
    for x, w, dy, dx, dw in ((q, wq, dyq, dq, dwq), (k, wk, dyk, dk, dwk)):
        for t in range(3):
            v, vw = randn(70 + t, *x.shape).double(), randn(80 + t, *w.shape).double()
            quotient = (loss(x.double() + h * v, w.double() + h * vw, dy) - loss(x.double() - h * v, w.double() - h * vw, dy)) / (2 * h)
            ours = float((dx.double() * v).sum() + (dw.double() * vw).sum())
            size = float((dx.double() * v).abs().sum() + (dw.double() * vw).abs().sum())
            assert abs(ours - quotient) <= 2e-5 * size, (ours, quotient)


def test_rows_that_hold_zeros_infinities_and_nan(gact):
    """A head's values reach no other head; a head of zeros is divided by sqrt(eps) and stays zero."""
    case = (1, 9, 4, 2, 64, 64, "f32", "f32", False)
    q, k, cos, sin, wq, wk, pos = inputs(case)
    clean, _ = gact.gact_head_norm_rotate(q, k, cos, sin, wq, wk, pos)
    q[0, 2, 1], q[0, 3, 2, 5], q[0, 4, 0, 7] = 0.0, math.inf, math.nan
    ctx = tuple(gact.make_head_context(x) for x in (q, k))
    y, _ = gact.gact_head_norm_rotate(q, k, cos, sin, wq, wk, pos, context=ctx)
    dy = randn(90, *q.shape)
    dq = gact.gact_head_norm_rotate_backward(dy, None, cos, sin, wq, wk, pos, context=ctx, x=(q, k))[0]
    assert (y[0, 2, 1] == 0).all()
    f = Formula(q, wq, cos, sin, pos, False)
    g = f.turned(dy.double(), back=True) * f.w
    assert torch.allclose(dq[0, 2, 1].double(), g[0, 2, 1] * 1e3, rtol=1e-5, atol=1e-3)
    assert y[0, 4, 0].isnan().all() and y[0, 3, 2].isnan().any()
    touched = torch.zeros(1, 9, 4, dtype=torch.bool, device="cuda")
    touched[0, 2, 1] = touched[0, 3, 2] = touched[0, 4, 0] = True
    assert torch.equal(y[~touched], clean[~touched]) and dq[~touched].isfinite().all()


def test_positions_outside_the_tables(gact):
    """NaN in that token's rotated elements, all else as it was."""
    q, k, cos, sin, wq, wk, _ = inputs((1, 8, 3, 1, 64, 32, "bf16", "f32", False), 2)
    pos = torch.arange(8, device="cuda")
    good, _ = gact.gact_head_norm_rotate(q, k, cos, sin, wq, wk, pos)
    pos[2], pos[5], pos[6] = -1, cos.shape[0], 2 ** 40
    y, _ = gact.gact_head_norm_rotate(q, k, cos, sin, wq, wk, pos)
    for t in range(8):
        if t in (2, 5, 6):
            assert y[0, t, :, :32].isnan().all() and torch.equal(y[0, t, :, 32:], good[0, t, :, 32:])
        else:
            assert torch.equal(y[0, t], good[0, t])


def test_in_place_empty_and_streams(gact):
    case = (2, 30, 4, 2, 128, 128, "bf16", "bf16", False)
    q, k, cos, sin, wq, wk, pos = args = inputs(case)
    yq, yk = gact.gact_head_norm_rotate(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    zq, zk = gact.gact_head_norm_rotate(*args, stream=side)
    hq, hk = gact.gact_head_norm_rotate(*args, stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in ((yq, zq), (yk, zk), (yq, hq), (yk, hk)))
    same = (q.clone(), k.clone())
    call = gact.prepare_head_norm_rotate(*same, *args[2:], out=same)
    call(torch.cuda.current_stream().cuda_stream)
    assert torch.equal(same[0], yq) and torch.equal(same[1], yk)
    ctx = tuple(gact.make_head_context(x[:0], 4, 128, 1) for x in (q, k))
    e = gact.gact_head_norm_rotate(q[:0], k[:0], cos, sin, wq, wk, None, context=ctx)
    assert e[0].shape == (0, 30, 4, 128)
    grads = gact.gact_head_norm_rotate_backward(*e, cos, sin, wq, wk, None, context=ctx)
    assert grads[0].numel() == 0 and (grads[2] == 0).all() and (grads[3] == 0).all()


def test_captured_and_replayed(gact):
    """Forward with a compressed context and backward in one graph: every replay equals the eager calls on the inputs
    of its time, with eager work between the replays."""
    case = (2, 50, 8, 2, 64, 64, "bf16", "f32", False)
    q, k, cos, sin, wq, wk, _ = inputs(case)
    pos = torch.randint(0, 53, (2, 50), device="cuda", generator=rng(4))
    dyq, dyk = (randn(50 + j, *x.shape, dtype=x.dtype) for j, x in enumerate((q, k)))
    ctx = [gact.make_head_context(x, 4, 128, 9 + j) for j, x in enumerate((q, k))]
    ws = torch.empty(gact.gact_head_norm_rotate_workspace_bytes(64), dtype=torch.uint8, device="cuda")

    def step(context, workspace):
        y = gact.gact_head_norm_rotate(q, k, cos, sin, wq, wk, pos, context=context)
        return list(y) + list(gact.gact_head_norm_rotate_backward(dyq, dyk, cos, sin, wq, wk, pos, context=context,
                                                                  workspace=workspace))
    step(ctx, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(ctx, ws)
    other = [gact.make_head_context(x, 4, 128, 9 + j) for j, x in enumerate((q, k))]
    for n in range(4):
        q.copy_(randn(200 + n, *q.shape, dtype=q.dtype))
        wq.copy_(randn(300 + n, *wq.shape))
        pos.copy_(torch.randint(0, 53, (2, 50), device="cuda", generator=rng(n)))
        graph.replay()
        torch.cuda.synchronize()
        want = step(other, None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), n
        assert all(torch.equal(a.packed, b.packed) for a, b in zip(ctx, other)), n


def test_results_do_not_change_from_call_to_call(gact):
    case = (4, 700, 16, 4, 64, 64, "bf16", "f32", False)
    q, k, cos, sin, wq, wk, pos = inputs(case)
    ctx = [gact.make_head_context(x, 2, 256, 9 + j) for j, x in enumerate((q, k))]
    gact.gact_head_norm_rotate(q, k, cos, sin, wq, wk, pos, context=ctx)
    dyq, dyk = (randn(50 + j, *x.shape, dtype=x.dtype) for j, x in enumerate((q, k)))
    ref = gact.gact_head_norm_rotate_backward(dyq, dyk, cos, sin, wq, wk, pos, context=ctx)
    for _ in range(3):
        torch.empty(1 << 22, dtype=torch.uint8, device="cuda").fill_(0xFF)       # what the next workspace holds
        again = gact.gact_head_norm_rotate_backward(dyq, dyk, cos, sin, wq, wk, pos, context=ctx)
        assert all(torch.equal(a, b) for a, b in zip(ref, again))


def test_nothing_is_written_outside_the_outputs(gact):
    """Outputs as slices of larger buffers: what lies around them stays."""
    case = (2, 21, 3, 1, 80, 80, "bf16", "f32", False)
    q, k, cos, sin, wq, wk, pos = args = inputs(case, 1, "fused")
    want = gact.gact_head_norm_rotate(*args)
    area = [torch.full((2, 23, x.shape[2] + 2, 80 + 8), 7.0, dtype=x.dtype, device="cuda") for x in (q, k)]
    out = tuple(a[:, 1:22, 1:-1, 3:83] for a in area)
    gact.gact_head_norm_rotate(*args, out=out)
    for a, o, w in zip(area, out, want):
        assert torch.equal(o, w)
        o.fill_(7.0)
        assert (a == 7.0).all()
    ctx = [gact.make_head_context(x) for x in (q, k)]
    gact.gact_head_norm_rotate(*args, context=ctx)
    dy = [randn(3 + j, *x.shape, dtype=x.dtype) for j, x in enumerate((q, k))]
    want = gact.gact_head_norm_rotate_backward(*dy, *args[2:], context=ctx, x=(q, k))
    gact.gact_head_norm_rotate_backward(*dy, *args[2:], context=ctx, x=(q, k), out=out)
    for a, o, w in zip(area, out, want):
        assert torch.equal(o, w)
        o.fill_(7.0)
        assert (a == 7.0).all()


@pytest.mark.parametrize("D,Hq,Hk", [(64, 8, 8), (80, 3, 1)])
def test_offsets_beyond_32_bits(gact, D, Hq, Hk):
    """Tokens so far apart that the last ones lie 6 GB behind the first, in the wavefront's addresses and in the lanes' own;
    heads too far apart for 32-bit offsets in a lane."""
    S = 24
    far = 134_217_728 + 8                              # elements between tokens: S of them reach 6.4 GB
    area = torch.empty(S * far, dtype=torch.bfloat16, device="cuda")
    q = area.as_strided((1, S, Hq, D), (0, far, D, 1))
    k = area.as_strided((1, S, Hk, D), (0, far, D, 1), Hq * D)
    q.copy_(randn(1, *q.shape)), k.copy_(randn(2, *k.shape))
    out = tuple(area.as_strided(x.shape, x.stride(), o) for x, o in ((q, 4096), (k, 8192)))
    cos, sin = tables(S, 64)
    w = randn(3, D) * 0.1 + 1
    args = (cos, sin, w, w)
    ctx, near_ctx = ([gact.make_head_context(x) for x in (q, k)] for _ in range(2))
    gact.gact_head_norm_rotate(q, k, *args, out=out, context=ctx)
    near = gact.gact_head_norm_rotate(q.contiguous(), k.contiguous(), *args, context=near_ctx)
    assert all(torch.equal(a, b) for a, b in zip(out, near))
    dy = tuple(randn(4 + j, *x.shape, dtype=x.dtype) for j, x in enumerate((q, k)))
    want = gact.gact_head_norm_rotate_backward(*dy, *args, context=near_ctx, x=(q.contiguous(), k.contiguous()))
    for a, b in zip(out, dy):
        a.copy_(b)
    got = gact.gact_head_norm_rotate_backward(*out, *args, context=ctx, x=(q, k), out=out)        # dx in place of dy
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # heads of one token 400 M elements apart
    wide = area.as_strided((1, 2, 8, D), (0, 4096, 400_000_008, 1))
    wide.copy_(randn(7, *wide.shape))
    y, _ = gact.gact_head_norm_rotate(wide, None, *args)
    assert torch.equal(y, gact.gact_head_norm_rotate(wide.contiguous(), None, *args)[0])


def test_calls_whose_tensors_do_not_belong_together(gact):
    q, k, cos, sin, wq, wk, pos = args = inputs((2, 8, 4, 2, 64, 64, "bf16", "f32", False))
    ctx = [gact.make_head_context(x, 4, 64, 1) for x in (q, k)]
    gact.gact_head_norm_rotate(*args, context=ctx)
    for bad in (k[:1], k[:, :4], k[..., :32], k.float(), k[0]):
        with pytest.raises(ValueError):
            gact.gact_head_norm_rotate(q, bad, *args[2:])
        with pytest.raises(ValueError):
            gact.gact_head_norm_rotate_backward(q, bad, *args[2:], context=ctx)
    other = gact.make_head_context(k, 4, 128, 1)
    for context in ((ctx[0], ctx[0]), (ctx[0], other)):
        with pytest.raises(ValueError):
            gact.gact_head_norm_rotate(*args, context=context)
        with pytest.raises(ValueError):
            gact.gact_head_norm_rotate_backward(q, k, *args[2:], context=context)
    with pytest.raises(ValueError):
        gact.gact_head_norm_rotate(*args, out=(q, q))
    with pytest.raises(ValueError):
        gact.gact_head_norm_rotate_backward(q, k, *args[2:], context=ctx, out=(q, q))
    with pytest.raises(ValueError):
        gact.gact_head_norm_rotate_backward(q, k, *args[2:], context=[gact.make_head_context(x) for x in (q, k)])      # no x
    with pytest.raises(ValueError):
        gact.gact_head_norm_rotate(q, k, cos.cpu(), sin, wq, wk, pos)
    with pytest.raises(gact.GactError):
        gact.gact_head_norm_rotate(*args, context=[gact.make_head_context(x, 4, 256, 1) for x in (q, k)])              # 2 * 64 < 256
    with pytest.raises(gact.GactError):
        gact.gact_head_norm_rotate(*args, eps=0.0)


@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("case", [(64, 0, "f32", 32), (64, 32, "bf16", 32), (64, 48, "f32", 4), (80, 16, "bf16", 2), (256, 64, "f32", 8),
                                  (96, 96, "bf16", 32)], ids=str)
def test_infinities_go_where_the_formula_has_them(gact, case, interleaved):
    """In elements that are not rotated an infinite gradient reaches its own weight's gradient and, through the mean, its row,
    not the element beside it; in rotated ones its pair.  The same for infinite inputs, of which the others' norm is 0."""
    D, rot, dtype, bits = case
    q, k, cos, sin, wq, wk, pos = inputs((1, 5, 2, 2, D, rot, dtype, "f32", interleaved), 1)
    cos, sin = (cos.abs() + 0.1, sin.abs() + 0.1) if rot else (None, None)      # no turn by 0: 0 times infinity is NaN there
    ctx = tuple(gact.make_head_context(x, bits, 0 if bits == 32 else 160 if D == 80 else 64, 3) for x in (q, k))
    gact.gact_head_norm_rotate(q, k, cos, sin, wq, wk, pos, interleaved=interleaved, context=ctx)
    f = Formula(q, wq, cos, sin, pos, interleaved)
    held = f.x
    if bits != 32:
        held = gact.gact_decompress(ctx[0].packed, ctx[0].gmin, ctx[0].gscale, q.numel(), ctx[0].group_size, bits).view(q.shape).double()
    for at in {0, rot // 2, max(rot - 1, 0), rot % D, D - 2, D - 1}:
        dy = randn(90, *q.shape, dtype=q.dtype)
        dy[0, 2, 1, at] = -math.inf
        dx, _, dw, _ = gact.gact_head_norm_rotate_backward(dy, None, cos, sin, wq, wk, pos, context=ctx, x=(q, k), interleaved=interleaved)
        dn, xr = f.turned(dy.double(), back=True), held * f.r
        g = dn * f.w
        want_w, want = (dn * xr).sum((0, 1, 2)), f.r * (g - xr * (g * xr).mean(-1, keepdim=True))
        for got, ref in ((dw, want_w), (dx, want)):
            assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.isinf(), ref.isinf()), at
            inf = ref.isinf()
            assert torch.equal(got[inf].double(), ref[inf]) and (~ref.isfinite()).any()
        rest = want_w.isfinite()
        assert rest.sum() == D - (1 if at >= rot else 2)
        size = (f.turned(dy.double(), back=True, magnitude=True) * xr.abs()).sum((0, 1, 2))
        assert ((dw.double() - want_w).abs() <= 301 * U * size)[rest].all()
        x = q.clone()
        x[0, 2, 1, at] = math.inf
        y, _ = gact.gact_head_norm_rotate(x, None, cos, sin, wq, None, pos, interleaved=interleaved)
        nan = torch.zeros(D, dtype=torch.bool, device="cuda")
        nan[at] = True
        if at < rot:
            nan[at ^ 1 if interleaved else (at + rot // 2) % rot] = True
        assert torch.equal(y[0, 2, 1].isnan(), nan) and (y[0, 2, 1][~nan] == 0).all()


@pytest.mark.parametrize("expand", ((3, -1, -1, -1), (-1, 16, -1, -1), (-1, -1, 8, -1)), ids=str)
@pytest.mark.parametrize("bits", (32, 4))
def test_inputs_whose_rows_share_memory(gact, expand, bits):
    """Queries, keys and gradients expanded over the batch, the tokens or the heads: read as if they were copies."""
    B, S, H, D = 3, 16, 8, 64
    cos, sin = tables(S, D)
    w = [randn(5 + j, D, scale=0.3) + 1 for j in range(2)]
    q, k = (randn(j, *(1 if e != -1 else n for e, n in zip(expand, (B, S, H, D))), dtype=torch.bfloat16).expand(B, S, H, D) for j in range(2))
    dy = [randn(7 + j, *(1 if e != -1 else n for e, n in zip(expand, (B, S, H, D))), dtype=torch.bfloat16).expand(B, S, H, D) for j in range(2)]
    got, want = [], []
    for results, x, d in ((got, (q, k), dy), (want, [t.contiguous() for t in (q, k)], [t.contiguous() for t in dy])):
        ctx = [gact.make_head_context(t, bits, 0 if bits == 32 else 64, 1 + j) for j, t in enumerate(x)]
        results += gact.gact_head_norm_rotate(*x, cos, sin, *w, context=ctx)
        results += gact.gact_head_norm_rotate_backward(*d, cos, sin, *w, context=ctx, x=x)
        results += [c.packed for c in ctx]
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    with pytest.raises((gact.GactError, ValueError)):
        gact.gact_head_norm_rotate(q, k, cos, sin, *w, out=(q, k))
    if bits == 32:
        leaf = q[tuple(slice(0, 1) if e != -1 else slice(None) for e in expand)].clone().requires_grad_(True)
        from paper_2206_11357_amd import heads
        y, _ = heads.head_norm_rotate(leaf.expand(B, S, H, D), k, cos, sin, *w)
        y.backward(dy[0])
        full = want[2].double().sum([i for i, e in enumerate(expand) if e != -1], keepdim=True)
        size = want[2].double().abs().sum([i for i, e in enumerate(expand) if e != -1], keepdim=True)
        # at most 16 rows added in binary32, rounded once
        assert ((leaf.grad.double() - full).abs() <= 2.0 ** -8 * full.abs() * 1.001 + 16 * U * size).all()
