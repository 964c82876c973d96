"""Gradient norm over many buffers and clipping, against 64 bits.  Bounds: squares are exact or rounded once in binary64
and added in at most 10^5 steps a thread and about 30 behind them, all terms positive: below 1e-11 relative for the sizes
here (the root halves it).  A clipped value is (double) g * c rounded to the type: half a step, and in bf16, which goes by
way of binary32, 2^-24 more; c itself is good to 1e-11."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def grads(sizes, kinds, seed=0, scale=0.01, odd=False):
    g = torch.Generator("cuda").manual_seed(seed)
    out = []
    for k, n in enumerate(sizes):
        dt = DT[kinds[k % len(kinds)]]
        t = (torch.randn(n + 1, device="cuda", generator=g) * scale * (1 + k % 5)).to(dt)
        out.append(t[1:] if odd else t[:n])
    return out


def norm_of(g, kind):
    if not any(t.numel() for t in g):
        return 0.0
    if kind == 2:
        return math.sqrt(sum(float((t.double() ** 2).sum()) for t in g))
    return max(float(t.double().abs().max()) for t in g if t.numel())


def check_clip(before, after, norm, max_norm):
    c = min(1.0, max_norm / (norm + 1e-6))
    for b, a in zip(before, after):
        want = b.double() * c
        assert ((a.double() - want).abs() <= want.abs() * (HALF[a.dtype] * (1 + 1e-3) + 1e-7 * (a.dtype == torch.bfloat16)) + 1e-38).all()


LISTS = [
    ((1,), ("f32",)), ((7,), ("bf16",)), ((4096,), ("f32",)), ((8192, 8193, 8191), ("bf16",)), ((0, 5, 0, 4097), ("f32",)),
    ((4096 * 3 + 1, 1, 2, 3, 100), ("f32", "bf16")), (tuple(1 + (k * 977) % 9000 for k in range(135)), ("bf16", "f32")),
    (tuple(1 + (k * 977) % 9000 for k in range(136)), ("f32",)), (tuple(1 + (k * 977) % 9000 for k in range(137)), ("f32", "bf16")),
    (tuple(k % 3 for k in range(700)), ("bf16",)), ((4096 * 1024,), ("f32",)), ((4096 * 1023 + 1, 4096), ("f32",)),
    ((8192 * 1025 + 5, 3, 8192 * 2), ("bf16",)), ((30_000_001, 5, 10_000_000), ("f32", "bf16")),
]


@pytest.mark.parametrize("odd", (False, True))
@pytest.mark.parametrize("kind", (2, math.inf))
@pytest.mark.parametrize("sizes,kinds", LISTS, ids=lambda v: "%d" % len(v) if isinstance(v, tuple) else None)
def test_norm_and_clip(gact, sizes, kinds, kind, odd):
    g = grads(sizes, kinds, 3, odd=odd)
    want = norm_of(g, kind)
    got = gact.gact_grad_norm(g, kind)
    assert got.dtype == torch.float64 and got.shape == (1,)
    assert abs(float(got) - want) <= (1e-11 if kind == 2 else 0.0) * want
    for share in (0.3, 1.7):
        max_norm = share * want + (1e-3 if want == 0 else 0)
        outs = [torch.full_like(t, 9.0) for t in g]
        norm = gact.gact_grad_clip(g, max_norm, kind, outs)
        assert torch.equal(norm, got)
        check_clip(g, outs, want, max_norm)
        by = [torch.full_like(t, 9.0) for t in g]
        gact.gact_grad_clip_by(g, max_norm, norm, by)
        assert all(torch.equal(a, b) for a, b in zip(outs, by))
        mine = [t.clone() for t in g]
        gact.gact_grad_clip(mine, max_norm, kind)
        assert all(torch.equal(a, b) for a, b in zip(outs, mine))


def test_no_buffers_and_empty_ones(gact):
    assert float(gact.gact_grad_norm([])) == 0.0
    g = [torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.bfloat16, device="cuda")]
    assert float(gact.gact_grad_norm(g)) == 0.0 and float(gact.gact_grad_clip(g, 1.0)) == 0.0
    gact.gact_grad_clip_by(g, 1.0, torch.ones(1, dtype=torch.float64, device="cuda"))


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
def test_infinities_and_nan(gact, dtype):
    base = grads((5000, 70, 9000), (dtype,), 5)
    for kind in (2, math.inf):
        g = [t.clone() for t in base]
        g[1][3] = -math.inf
        norm = gact.gact_grad_clip(g, 1.0, kind)
        assert float(norm) == math.inf
        assert g[1][3].isnan() and (g[0] == 0).all() and (g[2] == 0).all()
        for bad in (math.nan, -math.nan):
            g = [t.clone() for t in base]
            g[2][8999], g[0][0] = bad, math.inf
            norm = gact.gact_grad_clip(g, 1.0, kind)
            assert math.isnan(float(norm)) and all(t.isnan().all() for t in g)


def test_largest_values_do_not_overflow(gact):
    g = [torch.full((5000,), 3e38, device="cuda"), torch.full((10,), 1e-40, device="cuda")]
    got = float(gact.gact_grad_norm(g))
    want = math.sqrt(5000) * float(torch.tensor(3e38))
    assert abs(got - want) <= 1e-11 * want
    gact.gact_grad_clip(g, 1.0)
    assert torch.allclose(g[0].double(), torch.full((5000,), 1 / math.sqrt(5000), dtype=torch.float64, device="cuda"), rtol=1e-6)


def test_a_bound_of_zero_and_below_the_offset(gact):
    g = grads((100, 200), ("f32",), 7)
    z = [t.clone() for t in g]
    gact.gact_grad_clip(z, 0.0)
    assert all((t == 0).all() for t in z)
    zero = [torch.zeros(50, device="cuda")]
    assert float(gact.gact_grad_clip(zero, 1.0)) == 0.0 and (zero[0] == 0).all()


def test_nothing_around_the_buffers_changes(gact):
    for dtype in (torch.float32, torch.bfloat16):
        area = torch.full((60000,), 5.0, dtype=dtype, device="cuda")
        spans = [(1, 4098), (4099, 4100), (4103, 20000), (20001, 59999)]
        g = [area[a:b] for a, b in spans]
        gact.gact_grad_clip(g, 0.5)
        keep = torch.ones(60000, dtype=torch.bool, device="cuda")
        for a, b in spans:
            keep[a:b] = False
        assert (area[keep] == 5.0).all() and (area[~keep] != 5.0).all()


def test_channels_last_gradients(gact):
    g = torch.randn(8, 6, 5, 4, device="cuda").to(memory_format=torch.channels_last)
    want = g.double()
    norm = gact.gact_grad_clip([g], 0.25)
    assert abs(float(norm) - float(want.norm())) <= 1e-11 * float(norm)
    check_clip([want.float()], [g], float(norm), 0.25)


@pytest.mark.parametrize("K", (5, 300))
def test_captured_and_replayed(gact, K):
    """Short and long lists (whose table a graph carries in kernel arguments); the workspace is overwritten between the
    replays, and every replay equals the eager call."""
    g = grads([1 + (k * 7919) % 20000 for k in range(K)], ("f32", "bf16"), 2)
    src = [t.clone() for t in g]
    outs = [torch.empty_like(t) for t in g]
    ws = torch.empty(gact.gact_grad_norm_workspace_bytes(K), dtype=torch.uint8, device="cuda")
    norm = torch.empty(1, dtype=torch.float64, device="cuda")
    gact.gact_grad_clip(g, 0.5, outs=outs, norm=norm, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gact.gact_grad_clip(g, 0.5, outs=outs, norm=norm, workspace=ws)
    for n in range(4):
        for t, s in zip(g, src):
            t.copy_(s * (0.01 + n))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        ref = [torch.empty_like(t) for t in g]
        want = gact.gact_grad_clip(g, 0.5, outs=ref)
        assert torch.equal(norm, want) and all(torch.equal(a, b) for a, b in zip(outs, ref)), n


def test_streams_and_repeated_calls(gact):
    g = grads((100_000, 33, 1_000_000), ("f32", "bf16"), 8)
    want = gact.gact_grad_norm(g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = gact.gact_grad_norm(g, stream=side), gact.gact_grad_norm(g, stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, want) and torch.equal(b, want)
    for _ in range(3):
        assert torch.equal(gact.gact_grad_norm(g), want)


def test_a_buffer_of_more_than_2_31_elements(gact):
    n = 2 ** 31 + 12345
    area = torch.ones(n + 1, dtype=torch.bfloat16, device="cuda")
    g = [area[1:], torch.ones(5, device="cuda")]
    area[-1] = 3.0
    norm = gact.gact_grad_clip(g, 0.5 * math.sqrt(n + 13), 2.0)
    assert abs(float(norm) - math.sqrt(n + 13)) <= 1e-11 * math.sqrt(n)
    c = 0.5 * math.sqrt(n + 13) / (math.sqrt(n + 13) + 1e-6)
    want = torch.tensor(c).to(torch.bfloat16)
    assert area[0] == 1.0 and (area[1:-1] == want).all() and area[-1] == torch.tensor(3 * c).to(torch.bfloat16)
    assert float(gact.gact_grad_norm(g, math.inf)) == float(area[-1])


def test_bufs_of_other_gradients_are_noticed(gact):
    g = grads((100, 200), ("f32",), 7)
    bufs = gact.make_grad_bufs(g)
    with pytest.raises(ValueError):
        gact.gact_grad_norm([t.clone() for t in g], bufs=bufs)
    with pytest.raises(ValueError):
        gact.gact_grad_clip(g, 1.0, outs=[torch.empty_like(t) for t in g], bufs=bufs)
    with pytest.raises(ValueError):
        gact.gact_grad_norm(g + g, bufs=bufs)
    with pytest.raises(gact.GactError):
        gact.gact_grad_clip([g[0], g[0]], 1.0)                                   # the same buffer twice
    twice, once = float(gact.gact_grad_norm([g[0], g[0]])), float(gact.gact_grad_norm([g[0]]))
    assert abs(twice - math.sqrt(2) * once) <= 1e-11 * twice                     # counted as often as it is listed


def test_calls_whose_arguments_are_missing_or_strided(gact):
    g = grads((100, 200), ("f32",), 8)
    with pytest.raises(ValueError):
        gact.gact_grad_clip_by(g, 1.0, None)
    ws = torch.empty(2 * gact.gact_grad_norm_workspace_bytes(2), dtype=torch.uint8, device="cuda")
    for bad in (ws[::2], ws[:1].expand(ws.numel())):
        with pytest.raises(ValueError):
            gact.gact_grad_norm(g, workspace=bad)
    with pytest.raises(ValueError):
        gact.gact_grad_norm([g[0].view(10, 10)[:, :5]])


def test_gradients_in_another_order_of_axes(gact):
    g = [t.view(4, 5, -1).permute(2, 0, 1) for t in grads((100, 2000), ("f32", "bf16"), 9)]
    want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in g))
    before = [t.clone() for t in g]
    norm = float(gact.gact_grad_clip(g, 0.25 * want))
    assert abs(norm - want) <= 1e-11 * want
    c = 0.25 * want / (want + 1e-6)
    for t, b in zip(g, before):
        assert ((t.double() - c * b.double()).abs() <= c * b.double().abs() * torch.finfo(t.dtype).eps / 2 * 1.01).all()


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_every_offset_in_a_cache_line(gact, dtype):
    """Buffers that begin at every element of a line and end before, at and behind its end; what is between them stays."""
    lengths = (1, 5, 31, 32, 63, 64, 65, 8300)
    step = 8448                                        # whole lines
    area = torch.randn(64 * len(lengths) * step, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(dtype)
    before = area.clone()
    at = [(i * step + offset, n) for i, (offset, n) in enumerate((o, n) for o in range(64) for n in lengths)]
    g = [area[a:a + n] for a, n in at]
    inside = torch.zeros_like(area, dtype=torch.bool)
    for a, n in at:
        inside[a:a + n] = True
    want = math.sqrt(float((before[inside].double() ** 2).sum()))
    norm = float(gact.gact_grad_clip(g, 0.5 * want))
    assert abs(norm - want) <= 1e-11 * want
    assert torch.equal(area[~inside], before[~inside])
    c = 0.5 * want / (want + 1e-6)
    x, y = area[inside].double(), c * before[inside].double()
    # half a step of the type; binary32 on the way to bf16
    assert ((x - y).abs() <= (torch.finfo(dtype).eps / 2 * (1 + 2.0 ** -10)) * y.abs()).all()
    assert float(gact.gact_grad_norm(g, math.inf)) == float(area[inside].abs().max())


def test_a_table_is_looked_at_to_its_end(gact):
    """Whatever of the list has changed since the table was made, in its last buffer only: nothing is read or written by the old
    addresses, sizes or types."""
    g = grads((100, 200, 300), ("f32", "bf16"), 7)
    outs = [torch.zeros_like(t) for t in g]
    norm = gact.gact_grad_norm(g)
    in_place, copies = gact.make_grad_bufs(g), gact.make_grad_bufs(g, outs)
    flat = g[2].clone()
    wrong = [g[:2] + [g[2].clone()], g[:2] + [g[2][:299]], g[:2] + [g[2].view(torch.int16).view(torch.bfloat16)[:300]],
             g[:2] + [flat], [g[0], g[2], g[1]], g + [flat], g[:2] + [torch.as_strided(g[2], (300,), (0,))]]
    before = [t.clone() for t in g]
    for other in wrong:
        for call in (lambda: gact.gact_grad_norm(other, bufs=in_place), lambda: gact.gact_grad_clip(other, 1e-3, bufs=in_place),
                     lambda: gact.gact_grad_clip_by(other, 1e-3, norm, bufs=in_place),
                     lambda: gact.gact_grad_clip(other, 1e-3, outs=outs, bufs=copies)):
            with pytest.raises(ValueError):
                call()
    # outputs: others in the last place, too few, and none where the table has some
    for other in (outs[:2] + [flat], outs[:2], None, g):
        with pytest.raises(ValueError):
            gact.gact_grad_clip(g, 1e-3, outs=other, bufs=copies)
        with pytest.raises(ValueError):
            gact.gact_grad_clip_by(g, 1e-3, norm, outs=other, bufs=copies)
    with pytest.raises(ValueError):
        gact.gact_grad_clip(g, 1e-3, outs=outs, bufs=in_place)
    assert all(torch.equal(a, b) for a, b in zip(g, before)) and all((t == 0).all() for t in outs)
    # the same memory by other names, and the list's beginning
    same = [t.view(10, -1) for t in g]
    assert torch.equal(gact.gact_grad_norm(same, bufs=in_place), norm) and torch.equal(gact.gact_grad_norm(g, bufs=copies), norm)
    assert torch.equal(gact.gact_grad_norm(g[:2], bufs=in_place), gact.gact_grad_norm(g[:2]))
    assert torch.equal(gact.gact_grad_clip(g, 1e-3, outs=outs, bufs=copies), norm)
    # a tensor that has been given other memory
    g[2].data = g[2].clone()
    with pytest.raises(ValueError):
        gact.gact_grad_norm(g, bufs=in_place)


def test_a_table_keeps_its_buffers(gact):
    """Memory of gradients that are let go is not handed to others while a table that lists it can still be used."""
    g = grads((1 << 20,), ("f32",), 1)
    bufs = gact.make_grad_bufs(g)
    at = g[0].data_ptr()
    del g
    assert torch.zeros(1 << 20, device="cuda").data_ptr() != at
    assert bufs[0].g == at


@pytest.mark.parametrize("kinds", (("f32",), ("bf16",), ("f32", "bf16")), ids=str)
@pytest.mark.parametrize("mb", (250, 270, 300, 400, 450, 470))
def test_the_norm_is_the_same_in_every_call(gact, mb, kinds):
    """Bit for bit, below, between and above the sizes at which the launches change: its order depends on the list alone."""
    each = mb * 1_000_000 // sum(4 if t == "f32" else 2 for t in kinds)
    g = grads((each + 1,) * len(kinds), kinds, mb, scale=1.0, odd=True)
    norm = gact.gact_grad_norm(g)
    assert abs(float(norm) - norm_of(g, 2)) <= 1e-11 * float(norm)
    assert torch.equal(gact.gact_grad_clip(g, 1e9), norm)
    assert torch.equal(gact.gact_grad_clip(g, 1.0, outs=[torch.empty_like(t) for t in g]), norm)
