"""Argument checks of the gradient norm, clipping and head norm calls, on the host: nothing is launched.  The kernels' divisions
by variables, compiled for the host."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

import paper_2206_11357_amd as gact

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2206_11357_amd", "csrc")
BUF = (ctypes.c_char * (1 << 16))()
P = (ctypes.addressof(BUF) + 255) // 256 * 256



class Heads(ctypes.Structure):
    _fields_ = [(f, ctypes.c_void_p) for f in ("x", "y", "dy", "dx", "w", "dw", "rstd", "packed", "gmin", "gscale")] + \
        [(f, ctypes.c_int64 * 3) for f in ("x_stride", "y_stride", "dy_stride", "dx_stride")] + \
        [("seed", ctypes.c_uint64), ("heads", ctypes.c_int32), ("bits", ctypes.c_int32)]


class Rotation(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("tokens", ctypes.c_int64), ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p),
                ("positions", ctypes.c_void_p), ("n_positions", ctypes.c_int64)] + \
        [(f, ctypes.c_int32) for f in ("head_dim", "rot_dim", "interleaved", "dtype", "w_dtype", "group_size")] + \
        [("eps", ctypes.c_float), ("reserved", ctypes.c_int32)]


def test_the_binding_packs_the_records_of_the_interface():
    assert gact._HEADS.size == ctypes.sizeof(Heads) and gact._ROTATION.size == ctypes.sizeof(Rotation)
    h = Heads.from_buffer_copy(gact._HEADS.pack(*range(1, 11), *range(11, 23), 2**64 - 1, 5, 4))
    assert [getattr(h, f) for f in ("x", "y", "dy", "dx", "w", "dw", "rstd", "packed", "gmin", "gscale")] == list(range(1, 11))
    assert list(h.x_stride) + list(h.dx_stride) == [11, 12, 13, 20, 21, 22] and (h.seed, h.heads, h.bits) == (2**64 - 1, 5, 4)
    t = torch.zeros(9, 16)
    r = Rotation.from_buffer_copy(gact._rotation(2, 3, 64, torch.float32, t, t, torch.zeros(6, dtype=torch.int64), True,
                                                 torch.bfloat16, 64, 0.5))
    assert (r.batch, r.tokens, r.head_dim, r.rot_dim, r.n_positions, r.interleaved, r.dtype, r.w_dtype, r.group_size, r.eps,
            r.cos) == (2, 3, 64, 32, 9, 1, 0, 1, 64, 0.5, t.data_ptr())


def bufs(*entries):
    arr = (gact.GradBuf * max(len(entries), 1))()
    for b, (g, out, n, dtype) in zip(arr, entries):
        b.g, b.out, b.n, b.dtype = g, out, n, dtype
    return arr


def clip(arr, K, kind=0, max_norm=1.0, norm=P + 32768, ws=P + 49152, size=None):
    size = gact.gact_grad_norm_workspace_bytes(K) if size is None else size
    return gact.lib.gact_grad_clip(ctypes.addressof(arr) if arr is not None else None, K, kind, max_norm, norm, ws, size, None)


def test_norm_and_clip_refusals():
    E = gact.GACT_E_ARG
    ok = bufs((P, P, 64, 0), (P + 1024, P + 1024, 64, 1))
    assert clip(ok, -1) == E and clip(None, 2) == E
    assert clip(ok, 2, kind=2) == E and clip(ok, 2, kind=-1) == E
    for bad in (-1.0, math.nan, math.inf, -math.inf):
        assert clip(ok, 2, max_norm=bad) == E
    assert clip(ok, 2, norm=None) == E and clip(ok, 2, norm=P + 4) == E
    assert clip(ok, 2, ws=None) == E and clip(ok, 2, ws=P + 8) == E
    assert clip(ok, 2, size=gact.gact_grad_norm_workspace_bytes(2) - 1) == E
    for entry in ((None, P, 64, 0), (P, None, 64, 0), (P + 2, P + 2, 64, 0), (P, P + 1, 64, 1), (P, P, -1, 0), (P, P, 64, 2)):
        assert clip(bufs(entry), 1) == E, entry
    assert gact.lib.gact_grad_norm(ctypes.addressof(ok), 2, 5, P + 32768, P + 49152, 16000, None) == E
    assert gact.lib.gact_grad_norm(ctypes.addressof(ok), 2, 0, P + 32768, P + 49152, 8, None) == E
    assert gact.lib.gact_grad_clip_by(ctypes.addressof(ok), 2, -1.0, P + 32768, P + 49152, 16000, None) == E
    assert gact.gact_grad_norm_workspace_bytes(-1) == 0
    # more chunks than a launch takes
    assert clip(bufs((P, P, 1 << 62, 0)), 1) == E


def test_overlapping_outputs_are_refused():
    """A buffer listed twice, outputs that touch each other or an input that is not their own, also where a long one spans
    several short ones."""
    E = gact.GACT_E_ARG
    for entries in (((P, P, 64, 0), (P, P, 64, 0)),
                    ((P, P, 64, 0), (P + 252, P + 252, 64, 0)),
                    ((P, P + 4096, 64, 0), (P + 8192, P + 4096 + 255 // 4 * 4, 4, 0)),
                    ((P, P + 128, 64, 0),),
                    ((P, P + 1024, 64, 0), (P + 1024, P + 2048, 64, 0)),
                    ((P, P, 1000, 1), (P + 100, P + 8192, 10, 1)),
                    ((P, P + 8192, 10, 0), (P + 16384, P + 16384, 10, 0), (P + 20, P + 10, 300, 1))):
        assert clip(bufs(*entries), len(entries)) == E, entries


def record(**over):
    parts, r = (Heads * 2)(), Rotation()
    D = over.get("head_dim", 64)
    for k, h in enumerate(parts):
        h.heads, h.bits = 4, 4
        for f in ("x", "y", "dy", "dx", "w", "dw", "rstd", "packed", "gmin", "gscale"):
            setattr(h, f, P + 1024 * (k + 1))
        for f in ("x_stride", "y_stride", "dy_stride", "dx_stride"):
            setattr(h, f, (ctypes.c_int64 * 3)(8 * 4 * D, 4 * D, D))
    r.batch, r.tokens, r.head_dim, r.rot_dim, r.dtype, r.w_dtype, r.group_size, r.eps = 2, 8, D, D // 16 * 16, 1, 0, 64, 1e-6
    r.cos, r.sin, r.positions, r.n_positions = P, P, P, 8
    n_parts = over.pop("n_parts", 2)
    for key, v in over.items():
        if hasattr(r, key):
            setattr(r, key, v)
        else:
            setattr(parts[1 if n_parts == 2 else 0], key, v)
    return parts, n_parts, r


def forward(**over):
    parts, n, r = record(**over)
    return gact.lib.gact_head_norm_rotate(ctypes.addressof(parts), n, ctypes.addressof(r), None)


def backward(ws=P, size=1 << 30, **over):
    parts, n, r = record(**over)
    return gact.lib.gact_head_norm_rotate_backward(ctypes.addressof(parts), n, ctypes.addressof(r), ws, size, None)


BOTH = [dict(n_parts=0), dict(n_parts=3), dict(head_dim=0), dict(head_dim=12), dict(head_dim=520), dict(rot_dim=8),
        dict(rot_dim=80), dict(rot_dim=-16), dict(dtype=2), dict(w_dtype=7), dict(batch=-1), dict(tokens=-1),
        dict(batch=1 << 40), dict(batch=1 << 20, tokens=1 << 12), dict(batch=1 << 16, tokens=1 << 14, heads=4),
        dict(heads=0), dict(cos=None), dict(sin=P + 2), dict(positions=P + 4), dict(n_positions=-1), dict(rstd=None),
        dict(rstd=P + 2), dict(packed=None), dict(packed=P + 8), dict(gmin=None), dict(gscale=P + 1), dict(w=P + 2)]


@pytest.mark.parametrize("over", BOTH, ids=str)
def test_head_calls_refuse_what_neither_takes(over):
    assert forward(**dict(over)) == gact.GACT_E_ARG
    assert backward(**dict(over)) == gact.GACT_E_ARG


def test_head_calls_refuse_their_own():
    E = gact.GACT_E_ARG
    for over in (dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(x=None), dict(x=P + 1), dict(y=None)):
        assert forward(**over) == E, over
    for over in (dict(dy=None), dict(dx=None), dict(dx=P + 1), dict(dw=P + 2), dict(w=None), dict(bits=32, x=None),
                 dict(ws=None), dict(ws=P + 8), dict(size=gact.gact_head_norm_rotate_workspace_bytes(64) - 1)):
        assert backward(**over) == E, over
    assert gact.lib.gact_head_norm_rotate(None, 1, P, None) == E and gact.lib.gact_head_norm_rotate(P, 1, None, None) == E
    for bits in (0, 3, 16, -1):
        assert forward(bits=bits) == gact.GACT_E_BITS and backward(bits=bits) == gact.GACT_E_BITS
    assert [gact.gact_head_norm_rotate_workspace_bytes(d) for d in (0, 4, 12, 520, -8)] == [0] * 5


def apart(k, bits=4):
    """Part k of a call whose buffers are all different."""
    h = Heads()
    h.heads, h.bits = 4, bits
    for i, f in enumerate(("x", "y", "dy", "dx", "w", "dw", "rstd", "packed", "gmin", "gscale")):
        setattr(h, f, P + 8192 * (10 * k + i + 1))
    for f in ("x_stride", "y_stride", "dy_stride", "dx_stride"):
        setattr(h, f, (ctypes.c_int64 * 3)(8 * 4 * 64, 4 * 64, 64))
    return h


def refused(backward, change, bits=4):
    parts = (Heads * 2)(apart(0, bits), apart(1, bits))
    change(*parts)
    _, _, r = record()
    if backward:
        rc = gact.lib.gact_head_norm_rotate_backward(ctypes.addressof(parts), 2, ctypes.addressof(r), P, 1 << 30, None)
    else:
        rc = gact.lib.gact_head_norm_rotate(ctypes.addressof(parts), 2, ctypes.addressof(r), None)
    return rc == gact.GACT_E_ARG


def test_outputs_of_heads_that_overlap_are_refused():
    def to(field, value):
        return lambda a, b: setattr(b, field, value(a, b) if callable(value) else value)

    def strides(*s):
        return (ctypes.c_int64 * 3)(*s)
    for change in (to("y", lambda a, b: a.y), to("y", lambda a, b: a.x), to("rstd", lambda a, b: a.rstd),
                   to("packed", lambda a, b: a.packed), to("gmin", lambda a, b: a.gmin), to("gscale", lambda a, b: a.gscale),
                   to("y_stride", strides(2048, 256, 0)), to("y_stride", strides(0, 256, 64)),
                   to("y_stride", strides(2048, 255, 64)), to("y_stride", strides(2048, 64, 64)),
                   to("y_stride", strides(2048, 256, -63)), to("y_stride", strides(1 << 62, 256, 64)),
                   lambda a, b: (to("y", b.x)(a, b), to("y_stride", strides(2048, 64, 512))(a, b))):
        assert refused(False, change)
    for bits, change in ((4, to("dx", lambda a, b: a.dx)), (4, to("dx", lambda a, b: a.dy)), (4, to("dw", lambda a, b: a.dw)),
                         (32, to("dx", lambda a, b: b.x)), (32, to("dx", lambda a, b: a.x)),
                         (4, to("dx_stride", strides(2048, 256, 0))),
                         (4, lambda a, b: (to("dx", b.dy)(a, b), to("dx_stride", strides(2048, 64, 512))(a, b)))):
        assert refused(True, change, bits)


def test_groups_that_do_not_fit_heads():
    """The binding's rule and the library's are the same one."""
    for D in range(8, 520, 8):
        for G in (0, 16, 32, 64, 80, 96, 128, 160, 192, 256, 320, 384, 512, 640, 768, 1024):
            for heads in (1, 2, 3, 4, 8):
                fits = gact.head_context_fits(G, D, heads)
                # a call that is refused behind the group check where the group fits
                rc = forward(head_dim=D, group_size=G, heads=heads, n_parts=1, w=P + 2)
                assert rc == (gact.GACT_E_ARG if fits else gact.GACT_E_GROUP), (D, G, heads)
    assert gact.head_context_fits(256, 64, 16) and not gact.head_context_fits(1024, 64, 16)
    assert not gact.head_context_fits(256, 64, 2)


def test_empty_calls_need_no_tensors():
    parts, n, r = record(batch=0)
    for h in parts:
        for f in ("x", "y", "dy", "dx", "w", "dw", "rstd", "packed", "gmin", "gscale"):
            setattr(h, f, None)
    assert gact.lib.gact_head_norm_rotate(ctypes.addressof(parts), n, ctypes.addressof(r), None) == gact.GACT_OK
    assert gact.lib.gact_head_norm_rotate_backward(ctypes.addressof(parts), n, ctypes.addressof(r), None, 0, None) == gact.GACT_OK


def test_the_binding_refuses_tensors_the_kernels_cannot_take():
    x = torch.zeros(2, 3, 4, 64)
    with pytest.raises(ValueError):
        gact.gact_head_norm_rotate(x, None, None, None)                     # host memory
    with pytest.raises(ValueError):
        gact.make_grad_bufs([x])
    dense = [x, x.transpose(1, 3), x.permute(2, 0, 3, 1), x[:1, :1, :1], x[:0, ::2], torch.zeros(6, 5).t(), torch.zeros(())]
    assert all(gact._dense(t) for t in dense)
    assert not any(gact._dense(t) for t in (x[:, :2], x[:, :1, :1], x[..., ::2], x[:1].expand(2, 3, 4, 64), torch.zeros(6, 5).t()[1:]))
    with pytest.raises(ValueError):
        gact._norm_kind(1.0)
    for strided in (x.transpose(2, 3), x[0, 0], x[:, :, :, ::2]):
        with pytest.raises(ValueError):
            gact._head_strides(strided)
    t = torch.zeros(3, 32)
    for cos, sin, pos in ((t, None, None), (t.double(), t.double(), None), (t, t[:2], None), (t.t(), t.t(), None),
                          (t, t, torch.zeros(6, dtype=torch.int32)), (t, t, torch.zeros(5, dtype=torch.int64)), (t[:2], t[:2], None)):
        with pytest.raises(ValueError):
            gact._rotation(2, 3, 64, x.dtype, cos, sin, pos, False, None, 0, 1e-6)
    with pytest.raises(TypeError):
        gact._rotation(2, 3, 64, torch.float16, t, t, None, False, None, 0, 1e-6)
    for weights in ((torch.zeros(64), torch.zeros(64, dtype=torch.bfloat16)), (torch.zeros(63), None), (None, torch.zeros(128)[::2])):
        with pytest.raises(ValueError):
            gact._weights_dtype(*weights, 64)
    for bad in (x[0, 0], x[None]):
        with pytest.raises(ValueError):
            gact._head_shape(bad)


PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "gact_heads.h"
#include "gact_norm.h"
int main() {
    int failed = 0;
    uint64_t z = 88172645463325252ull;
    const auto next = [&]() { z ^= z << 13; z ^= z >> 7; z ^= z << 17; return z; };
    for (int i = 0; i < 400000; ++i) {
        const uint32_t d = i < 3000 ? (uint32_t)i + 1 : (uint32_t)(next() % 0x7FFFFFFF) >> (i % 31) | 1u;
        const gact::Divisor m = gact::divisor(d);
        const uint32_t top = 0x7FFFFFFFu / d * d;
        const uint32_t xs[] = {0u, 1u, d - 1, d, top - 1, top, 0x7FFFFFFFu, (uint32_t)next() >> 1};
        for (uint32_t x : xs) {
            if (x > 0x7FFFFFFFu) continue;
            const uint32_t q = m.magic == 0 ? x : (uint32_t)(((uint64_t)x * m.magic) >> 32) >> m.shift;
            if (q != x / d) { std::printf("%u / %u = %u\n", x, d, q); failed = 1; }
        }
    }
    // the launches' plans, whatever the parts' sizes
    for (uint32_t passes = 1; passes < 5000; ++passes) {
        for (const uint32_t most : {1u, 2u, 3u, 8u}) {
            const uint32_t run = gact::head_run(passes, most);
            if (run < 1 || run > most || passes % run != 0 || (passes <= most && run != passes)) { std::printf("run\n"); failed = 1; }
        }
    }
    for (const uint64_t passes : {0ull, 1ull, 2047ull, 2048ull, 4095ull, 4096ull, 6144ull, 16384ull, 1ull << 31}) {
        for (const uint32_t most : {3u, 8u}) {
            const uint32_t run = gact::head_most_run(passes, most);
            if (run < 1 || run > most || (run > 1 && passes / run < gact::kHeadFill)) { std::printf("most run\n"); failed = 1; }
        }
    }
    for (int i = 0; i < 100000; ++i) {
        gact::HeadArgs a{};
        for (auto& p : a.part) {
            p.run = 1 + (uint32_t)(next() % 8);
            p.units = (i < 3000 ? (uint32_t)(next() % 60000) : (uint32_t)(next() % 0x7FFFFFFF) >> (next() % 31)) / p.run;
        }
        for (const uint32_t all : {gact::head_backward_blocks(0), gact::head_backward_blocks(1), gact::kHeadForwardBlocks}) {
            gact::plan_heads(a.part, 2, all);
            if (a.part[0].blocks + a.part[1].blocks > all) { std::printf("blocks\n"); failed = 1; }
            for (auto& p : a.part) {
                if ((p.units != 0) != (p.blocks != 0) || p.waves != p.blocks * gact::kHeadWaves) { std::printf("waves\n"); failed = 1; }
                if (p.blocks != 0 && (uint64_t)(p.blocks - 1) * gact::kHeadWaves >= p.units) { std::printf("idle block\n"); failed = 1; }
            }
        }
    }
    // every row of a part is taken once, by a lane that has its token and its address, however the part is laid out
    for (int i = 0; i < 4000; ++i) {
        gact::HeadArgs a{};
        a.lanes_shift = (int)(next() % 7);
        a.dim = a.lanes_shift == 0 ? 8 : (4 << a.lanes_shift) + 8 + (int)(next() % (1 << a.lanes_shift)) / 2 * 8;
        if (i % 2) a.dim = 8 << a.lanes_shift;
        a.seq = 1 + (uint32_t)(next() % 9);
        a.by_seq = gact::divisor(a.seq);
        const uint32_t batch = 1 + (uint32_t)(next() % 5), in_pass = 64u >> a.lanes_shift;
        gact::HeadPart& p = a.part[0];
        p.heads = 1 + (uint32_t)(next() % (i % 3 ? 20 : 200));
        p.rows = batch * a.seq * p.heads;
        p.row_by_heads = gact::divisor(p.heads);
        gact::HeadTensor& t = p.t[gact::kIn];
        const int64_t far = i % 5 == 0 ? 1ll << 31 : 100000, offset = i % 7 == 0 ? far / 2 : 0;      // too far for 32 bits; negative
        t.batch = (int64_t)(next() % 100000) - 50000;
        t.token = (int64_t)(next() % far) - offset;
        t.head = (int64_t)(next() % far) - offset;
        const int size = i % 2 ? 2 : 4;
        const int mode = gact::lay_out_heads(a, &p, i % 4 == 3 ? 0 : 1 + (uint32_t)(next() % 8), size);
        if ((i % 4 == 3 || t.token < 0 || t.head < 0) && mode != gact::kAny) { std::printf("mode\n"); failed = 1; }
        gact::plan_heads(a.part, 1, 8);
        const bool steady = mode != gact::kAny;
        std::vector<int> taken(p.rows);
        for (uint32_t w = 0; w < p.waves; ++w)
            for (uint32_t unit = w; unit < p.units; unit += p.waves)
                for (uint32_t lane = 0; lane < in_pass; ++lane) {
                    const gact::UnitPlace u = gact::unit_place(a, p, steady, unit, lane, a.lanes_shift);
                    const uint32_t more = gact::lane_token(p, steady, lane);
                    const int64_t mine = gact::lane_first(p, t, steady, lane, more);
                    if (steady && (mine < 0 || (mine + a.dim) * size > 0xFFFFFFFFll)) { std::printf("offset\n"); failed = 1; }
                    int64_t at = gact::unit_first(t, steady, u) + mine;
                    for (uint32_t pass = 0; pass < p.run; ++pass, at += t.pass) {
                        const uint64_t row = ((uint64_t)unit * p.run + pass) * in_pass + lane;
                        if (row >= p.rows) { if (steady) { std::printf("row\n"); failed = 1; } continue; }
                        const uint32_t token = (uint32_t)(row / p.heads), head = (uint32_t)(row % p.heads);
                        const int64_t want = (int64_t)(token / a.seq) * t.batch + (int64_t)(token % a.seq) * t.token + (int64_t)head * t.head;
                        if (at != want || u.token + more != token || u.at + more != token % a.seq) { std::printf("place\n"); failed = 1; }
                        ++taken[row];
                    }
                }
        for (int n : taken) if (n != 1) { std::printf("taken\n"); failed = 1; break; }
    }
    return failed;
}
"""


def test_divisions_and_launch_plans(tmp_path):
    src = tmp_path / "plans.cpp"
    src.write_text(PROGRAM)
    exe = tmp_path / "plans"
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout[:500]
