"""Group norm with an activation over channels-last maps, its context and its gradients, against the formulas in binary64."""
import pytest
import torch

import paper_2206_11357_amd as gact

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a step, relative
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
RAW = gact.GACT_BITS_UNCOMPRESSED


def inputs(B, P, C, dtype, w_dtype, wide=0, seed=0, mean=0.5, spread=1.0):
    gen = torch.Generator().manual_seed(seed * 7919 + B + 3 * P + 17 * C)

    def normal(*shape):
        return torch.randn(*shape, generator=gen)
    x = (normal(B, P, C + wide) * spread + mean).to(dtype).cuda()[..., :C]
    dy = (normal(B, P, C + wide) * 0.1).to(dtype).cuda()[..., :C]
    w = b = None
    if w_dtype is not None:
        w, b = (1.0 + 0.2 * normal(C)).to(w_dtype).cuda(), (0.2 * normal(C)).to(w_dtype).cuda()
    return x, dy, w, b


def by_group(x, H):
    B, P, C = x.shape
    return x.view(B, P, H, C // H)


def statistics(x, H, eps):
    v = by_group(x.cpu().double(), H)
    m = v.mean((1, 3), keepdim=True)
    return m, ((v - m).square().mean((1, 3), keepdim=True) + eps).rsqrt()


def channels(v, H, like):
    return torch.full((1, 1, H, like // H), 0.0, dtype=torch.float64) + (v.cpu().double().view(1, 1, H, like // H))


def forward(x, H, w, b, eps, act):
    """y in binary64, and a bound on what binary32 arithmetic may be off by."""
    C = x.shape[-1]
    m, r = statistics(x, H, eps)
    v = by_group(x.cpu().double(), H)
    w = channels(w, H, C) if w is not None else torch.ones(1, 1, H, C // H, dtype=torch.float64)
    b = channels(b, H, C) if b is not None else torch.zeros(1, 1, H, C // H, dtype=torch.float64)
    z = (v - m) * r * w + b
    # m and x - m round by 2^-24 of the values, and m's sum is merged from parts, each merge a rounding or two: 2^-21 of the
    # largest value covers 8 of them; r's sum likewise; then three roundings of z; the activation's slope is at most 1.1, its own
    # arithmetic (exp, a sum, a quotient, a product) off by four steps of binary32, or in bf16's form |z| + 4 of them.
    far = v.abs().amax((1, 3), keepdim=True)
    off = 2.0 ** -21 * ((far * r + (v - m).abs() * r * (1 + (far * r).square() * 2.0 ** -10)) * w.abs() + z.abs() + b.abs())
    if act == "silu":
        y = z * torch.sigmoid(z)
        off = 1.1 * off + y.abs() * (4 + z.abs()) * 2.0 ** -22
    else:
        y = z
    return y.view(x.shape), off.view(x.shape), (m, r, w, b)


def within(got, want, off, what):
    got, want, off = got.cpu(), want, off
    assert torch.isfinite(got).all(), what
    bound = off + HALF[got.dtype] * (want.abs() + off) + 2.0 ** -126
    worst = ((got.double() - want).abs() / bound).max()
    assert worst <= 1, "%s: %g times the roundings" % (what, worst)


def check_forward(B, P, C, H, act="silu", dtype=torch.float32, w_dtype=torch.float32, wide=0, eps=1e-5, **how):
    x, _, w, b = inputs(B, P, C, dtype, w_dtype, wide, **how)
    y = gact.gact_group_norm(x, H, w, b, eps, act)
    want, off, _ = forward(x, H, w, b, eps, act)
    within(y, want, off, "y")
    return x, w, b, y


def check_step(B, P, C, H, bits, G=32, act="silu", dtype=torch.float32, w_dtype=torch.float32, wide=0, eps=1e-5, seed=5):
    x, dy, w, b = inputs(B, P, C, dtype, w_dtype, wide)
    context = gact.make_group_norm_context(x, H, bits, G if bits != RAW else 0, seed)
    y = gact.gact_group_norm(x, H, w, b, eps, act, context=context)
    want, off, (m, r, wc, bc) = forward(x, H, w, b, eps, act)
    within(y, want, off, "y")
    within(context.mean, m.view(B, H), 2.0 ** -21 * x.cpu().double().abs().amax() + 0 * m.view(B, H), "mean")
    xc = x.cpu().double()
    if bits != RAW:
        packed, gmin, gscale = gact.gact_compress(x.contiguous(), G, bits, seed)
        assert torch.equal(context.packed, packed) and torch.equal(context.gmin, gmin) and torch.equal(context.gscale, gscale)
        xc = gact.gact_decompress(packed, gmin, gscale, x.numel(), G, bits).view(B, P, C).cpu().double()
    dx, dw, db = gact.gact_group_norm_backward(dy, H, w, b, act, context=context, x=x if bits == RAW else None)
    # from the kernel's own m and r, which are inputs of the backward pass
    m, r = (t.cpu().double().view(B, 1, H, 1) for t in (context.mean, context.rstd))
    v = by_group(xc, H)
    n = (v - m) * r
    z = n * wc + bc
    d = by_group(dy.cpu().double(), H)
    # binary32: x - m and the product round; z by three more; act' moves by at most 0.5 a unit of z, and its own steps
    off_n = 2.0 ** -23 * (n.abs() + v.abs() * r)
    dz, off_z = d, 2.0 ** -24 * d.abs()
    if act == "silu":
        s = torch.sigmoid(z)
        dz = d * (s + z * s * (1 - s))
        off_z = d.abs() * (0.5 * (off_n * wc.abs() + 2.0 ** -22 * (z.abs() + bc.abs())) + (8 + 2 * z.abs()) * 2.0 ** -23)
    g, M = dz * wc, P * (C // H)
    m1, m2 = g.mean((1, 3), keepdim=True), (g * n).mean((1, 3), keepdim=True)
    # sums of k terms in binary32 (a thread's pixels, then rows): k roundings of the partial sums
    k = min(P, 4096) + 8
    off_g = off_z * wc.abs() + 2.0 ** -23 * g.abs()
    off1 = (off_g + k * 2.0 ** -24 * g.abs()).mean((1, 3), keepdim=True) + 2.0 ** -24 * m1.abs()
    off2 = (off_g * n.abs() + g.abs() * off_n + k * 2.0 ** -24 * (g * n).abs()).mean((1, 3), keepdim=True) + 2.0 ** -24 * m2.abs()
    ref = r * (g - m1 - n * m2)
    off = r * (off_g + off1 + n.abs() * off2 + off_n * m2.abs() + 2.0 ** -22 * (g.abs() + m1.abs() + (n * m2).abs()))
    within(dx, ref.view(B, P, C), off.view(B, P, C), "dx")
    if w is None:
        assert dw is None and db is None
        return
    total = (off_z * n.abs() + dz.abs() * off_n + (k + 2) * 2.0 ** -24 * (dz * n).abs()).sum((0, 1)).view(C)
    within(dw, (dz * n).sum((0, 1)).view(C), total, "dw")
    within(db, dz.sum((0, 1)).view(C), (off_z + (k + 2) * 2.0 ** -24 * dz.abs()).sum((0, 1)).view(C), "db")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("B,P,C,H", [(1, 1, 16, 2), (1, 1, 8, 1), (2, 3, 8, 4), (1, 64, 512, 32), (3, 17, 104, 13), (2, 50, 24, 8),
                                     (2, 7, 40, 40), (1, 300, 128, 32), (5, 1, 2048, 8), (2, 33, 2056, 257), (1, 5000, 8, 8), (1, 4099, 16, 1)])
def test_forward(B, P, C, H, act, dtype):
    check_forward(B, P, C, H, act, DTYPES[dtype], eps=1e-2 if P * (C // H) < 16 else 1e-5)


@pytest.mark.parametrize("w_dtype", [None, "f32", "bf16"])
@pytest.mark.parametrize("wide", [0, 8, 40, 3])
def test_weights_and_strides(wide, w_dtype):
    check_forward(3, 29, 72, 9, "silu", torch.bfloat16, None if w_dtype is None else DTYPES[w_dtype], wide)


@pytest.mark.parametrize("mean,spread", [(1000.0, 1.0), (-30.0, 0.01), (0.0, 1e-4), (0.0, 1e6)])
def test_far_means_and_small_spreads(mean, spread):
    check_forward(2, 700, 32, 4, "none", torch.float32, mean=mean, spread=spread)


def test_constant_groups():
    x = torch.full((2, 37, 16), 3.0, device="cuda")
    b = torch.randn(16, device="cuda")
    assert torch.equal(gact.gact_group_norm(x, 4, None, b), b.expand(2, 37, 16))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bits", [1, 2, 4, 8, RAW])
@pytest.mark.parametrize("B,P,C,H,G", [(2, 30, 64, 8, 64), (3, 221, 104, 13, 64), (2, 33, 24, 8, 128), (1, 40, 512, 32, 256),
                                       (4, 1, 256, 2, 512), (1, 3, 8, 1, 32)])
def test_step(B, P, C, H, G, bits, dtype):
    check_step(B, P, C, H, bits, G, "silu", DTYPES[dtype], eps=1e-2 if P * (C // H) < 32 else 1e-5)


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("w_dtype", [None, "f32", "bf16"])
@pytest.mark.parametrize("wide", [0, 16, 5])
def test_step_weights_and_strides(wide, w_dtype, act):
    check_step(2, 45, 80, 10, 4, 128, act, torch.bfloat16, None if w_dtype is None else DTYPES[w_dtype], wide)
    check_step(2, 45, 80, 10, RAW, 0, act, torch.bfloat16, None if w_dtype is None else DTYPES[w_dtype], wide)


# several chunks of pixels, more channels than a workgroup has columns, more samples than it has parts
@pytest.mark.parametrize("B,P,C,H", [(1, 20000, 32, 4), (2, 3000, 96, 32), (1, 40, 4104, 27), (70, 9, 48, 3)])
def test_step_larger(B, P, C, H):
    check_step(B, P, C, H, 2, 32)
    check_step(B, P, C, H, RAW, 0, "none", torch.bfloat16)


def test_axes_between_are_one_and_channels_last_memory():
    x = torch.randn(2, 24, 6, 7, device="cuda").to(memory_format=torch.channels_last)
    y = gact.gact_group_norm(x.permute(0, 2, 3, 1), 3)
    assert y.shape == (2, 6, 7, 24)
    assert torch.equal(y.view(2, 42, 24), gact.gact_group_norm(x.permute(0, 2, 3, 1).reshape(2, 42, 24), 3))


def test_in_place():
    x, dy, w, b = inputs(2, 50, 64, torch.bfloat16, torch.float32, wide=8)
    want = gact.gact_group_norm(x, 8, w, b, 1e-5, "silu")
    context = gact.make_group_norm_context(x, 8, 4, 64, 3)
    other = gact.make_group_norm_context(x, 8, 4, 64, 3)
    gact.gact_group_norm(x, 8, w, b, 1e-5, "silu", context=other)
    assert torch.equal(gact.gact_group_norm(x, 8, w, b, 1e-5, "silu", context=context, out=x), want) and torch.equal(x, want)
    assert torch.equal(context.blob[:context.off[3]], other.blob[:context.off[3]])
    grads = gact.gact_group_norm_backward(dy, 8, w, b, "silu", context=context)
    inside = gact.gact_group_norm_backward(dy, 8, w, b, "silu", context=context, out=dy)
    assert inside[0] is dy and all(torch.equal(p, q) for p, q in zip(grads, inside))


def test_empty_maps():
    w = torch.ones(16, device="cuda")
    for shape in ((0, 5, 16), (3, 0, 16)):
        x = torch.empty(shape, device="cuda")
        context = gact.make_group_norm_context(x, 4, 4, 32)
        assert gact.gact_group_norm(x, 4, w, w, context=context).shape == shape
        dx, dw, db = gact.gact_group_norm_backward(x, 4, w, w, context=context)
        assert dx.shape == shape and (dw == 0).all() and (db == 0).all()


def test_not_a_number_stays_in_its_group():
    x, dy, w, b = inputs(2, 40, 32, torch.float32, torch.float32)
    clean = gact.gact_group_norm(x, 4, w, b, 1e-5, "silu")
    x[1, 7, 9] = float("nan")
    y = gact.gact_group_norm(x, 4, w, b, 1e-5, "silu")
    assert torch.isnan(y[1, :, 8:16]).all()
    y[1, :, 8:16] = clean[1, :, 8:16]
    assert torch.equal(y, clean)


def test_what_lies_behind_the_buffers_stays():
    B, P, C, H = 3, 37, 40, 5
    x, dy, w, b = inputs(B, P, C, torch.bfloat16, torch.float32)
    room = torch.full((B * P * C + 256,), 7.0, dtype=torch.bfloat16, device="cuda")
    gapped = torch.full((B, P, C + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    need = max(gact.gact_group_norm_workspace_bytes(B, P, C, H, x.dtype, back) for back in (False, True))
    ws = torch.full((need + 256,), 77, dtype=torch.uint8, device="cuda")
    context = gact.make_group_norm_context(x, H, 2, 32, 1)
    size = context.blob.numel()
    blob = torch.full((size + 256,), 77, dtype=torch.uint8, device="cuda")
    context.blob = blob[:size]
    y = gact.gact_group_norm(x, H, w, b, context=context, out=room[:B * P * C].view(B, P, C), workspace=ws[:need])
    y2 = gact.gact_group_norm(x, H, w, b, out=gapped[..., :C], workspace=ws[:need])
    assert torch.equal(y, y2) and (gapped[..., C:] == 7).all()
    gact.gact_group_norm_backward(dy, H, w, b, context=context, out=room[:B * P * C].view(B, P, C), workspace=ws[:need])
    assert (room[B * P * C:] == 7).all() and (ws[need:] == 77).all() and (blob[size:] == 77).all()


def test_captured_repeated_and_on_another_stream():
    B, P, C, H = 2, 900, 64, 8
    x, dy, w, b = inputs(B, P, C, torch.bfloat16, torch.float32)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    context = gact.make_group_norm_context(x, H, 4, 64, 9)
    need = max(gact.gact_group_norm_workspace_bytes(B, P, C, H, x.dtype, back) for back in (False, True))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step():
        gact.gact_group_norm(x, H, w, b, 1e-5, "silu", context=context, out=y, workspace=ws)
        return gact.gact_group_norm_backward(dy, H, w, b, "silu", context=context, out=dx, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = step()
    prepared_out = torch.empty_like(x)
    call = gact.prepare_group_norm(x, H, w, b, 1e-5, "silu", out=prepared_out)
    for i in range(3):
        x.copy_(torch.randn(B, P, C, device="cuda"))
        dy.copy_(torch.randn(B, P, C, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        other = gact.make_group_norm_context(x, H, 4, 64, 9)
        eager = gact.gact_group_norm(x, H, w, b, 1e-5, "silu", context=other)
        assert torch.equal(eager, y) and torch.equal(other.blob, context.blob)
        call(torch.cuda.current_stream().cuda_stream)
        assert torch.equal(prepared_out, y)
        eager = gact.gact_group_norm_backward(dy, H, w, b, "silu", context=other)
        assert all(torch.equal(p, q) for p, q in zip(eager, grads))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    third = gact.make_group_norm_context(x, H, 4, 64, 9, stream=side)
    y3 = gact.gact_group_norm(x, H, w, b, 1e-5, "silu", context=third, stream=side)
    g3 = gact.gact_group_norm_backward(dy, H, w, b, "silu", context=third, stream=side)
    side.synchronize()
    assert torch.equal(y3, y) and all(torch.equal(p, q) for p, q in zip(g3, grads))


def test_gradients_against_differences():
    """Central differences of sum(y * dy) in binary64 arithmetic over fp32 outputs: the step h moves y by about h, whose rounding,
    2^-24 |y| a value, summed over the outputs that x reaches and divided by 2 h, bounds the difference beside the third
    derivative's h^2."""
    B, P, C, H = 1, 6, 16, 2
    x, dy, w, b = inputs(B, P, C, torch.float32, torch.float32)
    context = gact.make_group_norm_context(x, H)
    y = gact.gact_group_norm(x, H, w, b, 1e-5, "silu", context=context)
    dx, dw, db = gact.gact_group_norm_backward(dy, H, w, b, "silu", context=context, x=x)
    d = dy.double()
    h = 2.0 ** -7
    tol = 2.0 ** -22 * float((y.double().abs() + 2).mul(d.abs()).sum()) / h + 40 * h * h * float(d.abs().max())

    def loss(x_, w_, b_):
        return float((gact.gact_group_norm(x_, H, w_, b_, 1e-5, "silu").double() * d).sum())
    for grad, which, count in ((dx, 0, 24), (dw, 1, 16), (db, 2, 16)):
        args = [x, w, b]
        for i in range(0, args[which].numel(), max(1, args[which].numel() // count)):
            vals = []
            for sign in (1.0, -1.0):
                moved = args[which].clone()
                moved.view(-1)[i] += sign * h
                vals.append(loss(*(moved if j == which else t for j, t in enumerate(args))))
            assert abs((vals[0] - vals[1]) / (2 * h) - float(grad.view(-1)[i])) <= tol


# groups that are no whole columns of eight channels, in maps that a workgroup holds and in larger ones, part of a slab and several
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,P,C,H", [(3, 20, 120, 4), (2, 61, 72, 2), (2, 500, 72, 4), (1, 130, 504, 8), (2, 9, 1008, 16), (1, 40, 56, 1),
                                     (2, 33, 80, 5), (3, 100, 24, 12), (2, 17, 176, 16), (1, 700, 144, 8)])
def test_groups_of_any_size(B, P, C, H, dtype):
    check_step(B, P, C, H, 4, 64, "silu", DTYPES[dtype])
    check_step(B, P, C, H, RAW, 0, "none", DTYPES[dtype], None if H % 2 else torch.float32, wide=8)


# maps whose backward pass holds dy in the workgroups of the most registers: groups of one column and of two, a last slab of one, and
# outputs in place of dy
@pytest.mark.parametrize("B,P,C,H,bits,G,act,dtype", [(32, 2060, 264, 33, 2, 256, "none", "f32"), (64, 2111, 128, 8, 4, 64, "silu", "bf16")])
def test_step_of_many_large_maps(B, P, C, H, bits, G, act, dtype):
    check_step(B, P, C, H, bits, G, act, DTYPES[dtype])
    x, dy, w, b = inputs(B, P, C, DTYPES[dtype], torch.float32)
    context = gact.make_group_norm_context(x, H, bits, G, 3)
    gact.gact_group_norm(x, H, w, b, 1e-5, act, context=context)
    first = gact.gact_group_norm_backward(dy, H, w, b, act, context=context)
    again = gact.gact_group_norm_backward(dy, H, w, b, act, context=context, out=dy)
    assert again[0] is dy and all(torch.equal(u, v) for u, v in zip(first, again))
