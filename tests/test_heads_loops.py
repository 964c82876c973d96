"""Norms of heads where a wavefront has more than one unit and, where heads allow it, a unit more than one pass: long calls in
every layout, against the formulas in 64 bits and the compressor.  That the sizes reach these loops is asserted on the host, from
the launch plans themselves."""
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2206_11357_amd", "csrc")

ANY, STEADY = 0, 1
# B, S, Hq, Hk (0: no keys), D, rot, dtype, interleaved, positions given, bits of q and k, G; mode of a head's lanes (3, 4, 5: heads of
# 64, 128, 256), passes of a unit of q forward and backward, units of q a token (or 0: tokens of a unit's pass)
CASES = [
    # one token a unit, several passes; the keys' units have one
    (1, 25003, 12, 4, 128, 128, "bf16", False, False, (4, 4), 128, 4, 3, 3, 1),
    (3, 8335, 12, 4, 128, 64, "f32", True, True, (32, 32), 0, 4, 3, 3, 1),
    (1, 25003, 12, 4, 128, 128, "bf16", True, True, (32, 32), 0, 4, 3, 3, 1),
    (1, 25003, 12, 4, 128, 96, "f32", False, True, (8, 8), 512, 4, 3, 3, 1),
    (1, 23003, 16, 8, 64, 64, "f32", True, False, (2, 2), 32, 3, 2, 2, 1),
    (2, 11503, 16, 8, 64, 64, "bf16", False, True, (8, 8), 256, 3, 2, 2, 1),
    (1, 25003, 6, 2, 256, 256, "bf16", False, True, (1, 1), 256, 5, 3, 3, 1),
    (5, 5003, 6, 2, 256, 128, "f32", True, False, (4, 4), 512, 5, 3, 3, 1),
    (1, 25003, 6, 2, 256, 256, "f32", False, True, (32, 32), 0, 5, 3, 3, 1),
    (1, 25003, 6, 2, 256, 256, "bf16", True, False, (32, 32), 0, 5, 3, 3, 1),
    # several units a token
    (1, 11003, 36, 0, 128, 128, "bf16", False, True, (2, 2), 64, 4, 3, 3, 3),
    (1, 11003, 36, 0, 128, 128, "f32", False, False, (32, 32), 0, 4, 3, 3, 3),
    # lanes that are idle in every pass
    (1, 25003, 12, 4, 80, 32, "bf16", False, True, (2, 2), 320, STEADY, 3, 3, 1),
    (1, 25003, 12, 4, 80, 80, "f32", True, False, (32, 32), 0, STEADY, 3, 3, 1),
    (1, 25003, 3, 1, 512, 512, "f32", False, True, (8, 8), 512, STEADY, 3, 3, 1),
    (1, 33003, 64, 0, 8, 0, "bf16", False, False, (1, 1), 512, STEADY, 1, 1, 1),
    # several tokens a pass
    (3, 14800, 4, 2, 64, 64, "bf16", False, True, (4, 4), 64, 3, 1, 1, 0),
    (3, 14800, 4, 2, 64, 64, "f32", True, False, (32, 32), 0, 3, 1, 1, 0),
    (1, 66004, 4, 4, 40, 32, "f32", False, True, (8, 8), 160, STEADY, 1, 1, 0),
    # passes that begin in the middle of a token
    (1, 17001, 5, 3, 96, 96, "f32", False, False, (8, 8), 96, ANY, 1, 1, None),
    (1, 35003, 5, 3, 64, 64, "bf16", True, True, (32, 32), 0, ANY, 1, 1, None),
    (1, 35003, 5, 3, 64, 48, "bf16", False, True, (4, 4), 64, ANY, 1, 1, None),
    # queries would be steady, the one key head is not
    (1, 10501, 12, 1, 80, 32, "bf16", False, False, (32, 32), 0, ANY, 1, 1, None),
    # launches of their own: a compressed context and none, two widths
    (1, 33003, 16, 8, 128, 128, "bf16", False, True, (4, 32), 128, 4, 4, 2, None),
    (1, 66004, 8, 4, 64, 64, "f32", False, False, (2, 8), 64, 3, 1, 1, None),
]

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "gact_heads.h"
int main(int, char** v) {
    const int64_t B = std::atoll(v[1]), S = std::atoll(v[2]);
    const int heads[2] = {std::atoi(v[3]), std::atoi(v[4])}, dim = std::atoi(v[5]), f32 = std::atoi(v[6]);
    const int bits[2] = {std::atoi(v[7]), std::atoi(v[8])}, n = heads[1] ? 2 : 1;
    for (int backward = 0; backward < 2; ++backward) {
        gact::HeadArgs a{};
        while ((8 << a.lanes_shift) < dim) ++a.lanes_shift;
        a.dim = dim;
        a.seq = (uint32_t)S;
        a.by_seq = gact::divisor(a.seq);
        for (int k = 0; k < n; ++k) {
            gact::HeadPart& p = a.part[k];
            p.heads = (uint32_t)heads[k];
            p.rows = (uint32_t)(B * S * heads[k]);
            p.row_by_heads = gact::divisor(p.heads);
            for (auto& t : p.t) t = gact::HeadTensor{nullptr, S * heads[k] * dim, (int64_t)heads[k] * dim, dim, 0, 0};
        }
        const gact::HeadLaunches l = gact::arrange_heads(&a, n, bits, f32 ? GACT_DT_F32 : GACT_DT_BF16, backward != 0);
        for (int k = 0; k < n; ++k) {
            const gact::HeadPart& p = a.part[k];
            std::printf("%d %u %u %u %u %u\n", l.mode[k], p.run, p.units, p.waves, p.units_per_token, p.tokens_per_pass);
        }
    }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("plans")
    (d / "plans.cpp").write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", CSRC, str(d / "plans.cpp"), "-o", str(d / "plans")])
    return str(d / "plans")


@pytest.mark.parametrize("case", CASES, ids=str)
def test_the_sizes_reach_the_loops(plans, case):
    B, S, Hq, Hk, D, rot, dtype, inter, pos, bits, G, mode, forward, backward, units = case
    held = [0 if b == 32 else b for b in bits]
    out = subprocess.check_output([plans] + [str(v) for v in (B, S, Hq, Hk, D, int(dtype == "f32"), *held)], text=True)
    rows = [tuple(map(int, line.split())) for line in out.splitlines()]
    parts = 2 if Hk else 1
    assert len(rows) == 2 * parts
    for mode_, run, in_all, waves, units_per_token, tokens_per_pass in rows:
        assert mode_ == mode and in_all > waves
    assert rows[0][1] == forward and rows[parts][1] == backward
    if units is not None:
        assert all((r[4] == units and r[5] == 1) if units else r[5] > 1 for r in (rows[0], rows[parts]))


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_long_calls_against_the_formula(gact, case):
    """Bounds: those of the module that has the formula.  A lane adds the weight gradients of no more passes than the call has
    for each of 4,000 wavefronts, and some more at its ends."""
    from test_gpu_heads import DT, Formula, randn, rng, tables
    B, S, Hq, Hk, D, rot, dtype, inter, given, bits, G, *_ = case
    dt = DT[dtype]
    cos, sin = tables(S if not given else 5000, rot) if rot else (None, None)
    pos = torch.randint(0, 5000, (B, S), device="cuda", generator=rng(3)) if given else None
    x = [randn(1 + j, B, S, H, D, dtype=dt, scale=1.5) for j, H in enumerate((Hq, Hk)) if H]
    w = [randn(5 + j, D, scale=0.3) + 1 for j in range(2)]
    ctx = [gact.make_head_context(t, b, G if b != 32 else 0, 11 + j) for j, (t, b) in enumerate(zip(x, bits))]
    dy = [randn(7 + j, *t.shape, dtype=dt) for j, t in enumerate(x)]
    lone = len(x) == 1
    pair = (lambda t: (t[0], None) if lone else tuple(t))
    y = gact.gact_head_norm_rotate(*pair(x), cos, sin, w[0], None if lone else w[1], pos, interleaved=inter, context=pair(ctx))
    grads = gact.gact_head_norm_rotate_backward(*pair(dy), cos, sin, w[0], None if lone else w[1], pos, context=pair(ctx), x=pair(x),
                                                interleaved=inter)
    run = B * S * (Hq + Hk) * D // 512 // 4000 * 2 + 10
    for j, t in enumerate(x):
        held = None
        if bits[j] != 32:
            p, mn, sc = gact.gact_compress(t.view(-1), G, bits[j], 11 + j)
            assert torch.equal(ctx[j].packed, p)
            assert torch.equal(ctx[j].gmin, mn) and torch.equal(ctx[j].gscale, sc)
            held = gact.gact_decompress(p, mn, sc, t.numel(), G, bits[j]).view(t.shape)
        f = Formula(t, w[j], cos, sin, pos, inter)
        f.check_forward(y[j])
        f.check_backward(dy[j], grads[j], grads[2 + j], x=held, run=run)


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_no_row_is_left_out_of_the_weight_gradients(gact, case):
    """Whole numbers: x of -1 and 1, eps 3 and so r = 1/2, no turn, |dy| of 1 to 4.  Every term is a multiple of 1/2 and every sum
    below 2^23, so binary32 adds them without rounding and dw has to be exact (one bit, if a context is kept: its values are
    -1 and 1 again)."""
    from test_gpu_heads import DT, rng
    B, S, Hq, Hk, D, rot, dtype, inter, given, bits, G, *_ = case
    bits = [b if b == 32 else 1 for b in bits]
    n = S if not given else 5000
    cos, sin = (torch.ones(n, rot // 2, device="cuda"), torch.zeros(n, rot // 2, device="cuda")) if rot else (None, None)
    pos = torch.randint(0, n, (B, S), device="cuda", generator=rng(3)) if given else None
    x, dy = ([torch.randint(lo, hi, (B, S, H, D), device="cuda", generator=rng(20 + j + hi)) for j, H in enumerate((Hq, Hk)) if H]
             for lo, hi in ((0, 2), (1, 5)))
    x = [(2 * t - 1).to(DT[dtype]) for t in x]
    dy = [t.to(DT[dtype]) * s for t, s in zip(dy, x)]              # all of one sign: none hides another
    for t in x if G else ():                                       # every group has both
        t = t.view(-1, G)
        t[:, 0], t[:, 1] = -1, 1
    lone = len(x) == 1
    pair = (lambda t: (t[0], None) if lone else tuple(t))
    w = [torch.ones(D, device="cuda")] * 2
    ctx = [gact.make_head_context(t, b, G if b != 32 else 0, 11 + j) for j, (t, b) in enumerate(zip(x, bits))]
    gact.gact_head_norm_rotate(*pair(x), cos, sin, w[0], None if lone else w[1], pos, eps=3.0, interleaved=inter, context=pair(ctx))
    grads = gact.gact_head_norm_rotate_backward(*pair(dy), cos, sin, w[0], None if lone else w[1], pos, context=pair(ctx), x=pair(x),
                                                interleaved=inter)
    for j, t in enumerate(x):
        assert (ctx[j].rstd == 0.5).all()
        want = (dy[j].long() * t.long()).sum((0, 1, 2))
        assert int(want.abs().max()) < 1 << 23
        assert torch.equal(grads[2 + j].double(), want.double() / 2)
