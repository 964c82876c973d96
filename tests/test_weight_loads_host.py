"""Where the weight gradient's large forms load, on the host: a wavefront's offset into dy, codes, minima and steps lies
inside the buffer for every chunk that a block fetches, those that its loop asks for behind its split's end too."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2206_11357_amd", "csrc")

PROGRAM = r"""
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include "gact_weight.h"
#ifndef FETCHED
#define FETCHED gact::weight_fetched
#endif
static long checked = 0;
static int failed = 0;
static void check(uint64_t T, uint64_t N, uint64_t K, int dtype, int bits, uint32_t group, uint64_t stride) {
    const gact::WeightPlan p = gact::weight_splits(T, N, K, dtype, gact::kWeightLarge);
    const uint64_t BT = (uint64_t)gact::weight_tile(dtype, p.form).tokens, size = dtype == GACT_DT_F32 ? 4 : 2;
    gact::WeightArgs a{};
    a.dy_stride = (int64_t)stride;
    a.T = (uint32_t)T; a.N = (uint32_t)N; a.K = (uint32_t)K;
    a.group = group;
    a.chunks = p.chunks;
    const uint32_t dy_chunk = (uint32_t)(BT * stride * size), code_chunk = (uint32_t)(BT * K / 8 * bits), group_chunk = (uint32_t)(BT * K / group * 4);
    const bool buffer = gact::weight_buffer(a, dtype, p.form), even = gact::weight_even(a, dtype, p.form);
    const uint64_t all = (T + BT - 1) / BT, last_group = (T * K - 1) / group;
    for (uint64_t split = 0; split < p.splits; ++split) {
        const uint32_t c0 = (uint32_t)split * p.chunks, c1 = c0 + p.chunks < all ? c0 + p.chunks : (uint32_t)all;
        if (c0 >= c1) continue;
        const uint64_t t0 = c0 * BT;
        const uint64_t of_dy = ((T - t0 - 1) * stride + N) * size, of_codes = (T - t0) * K / 8 * bits, of_groups = (last_group + 1 - t0 * K / group) * 4;
        for (uint32_t c = c0; c < c1 + 3; ++c) {       // the loop reaches three chunks behind the present one
            const uint32_t f = FETCHED(c, c1), i = f - c0;
            if (f < c0 || f >= c1 || (c < c1 && f != c)) failed = 1;
            if (buffer && !((uint64_t)i * dy_chunk < of_dy && (uint64_t)i * dy_chunk < gact::kWeightReach)) failed = 1;
            if (even && K && !((uint64_t)i * code_chunk < of_codes && (uint64_t)i * group_chunk < of_groups)) failed = 1;
            ++checked;
        }
        if (failed) {
            std::printf("T %llu N %llu K %llu type %d bits %d group %u stride %llu split %llu\n", (unsigned long long)T, (unsigned long long)N,
                        (unsigned long long)K, dtype, bits, group, (unsigned long long)stride, (unsigned long long)split);
            return;
        }
    }
}
int main() {
    for (int dtype : {GACT_DT_F32, GACT_DT_BF16})
        for (int bits : {1, 2, 4, 8})
            for (uint32_t group : {32u, 96u, 256u, 1024u})
                for (uint64_t T : {1, 31, 32, 33, 64, 65, 127, 700, 9001, 19000, 19001, 33333, 169343})
                    for (uint64_t N : {33, 256, 510, 4100})
                        for (uint64_t K : {40, 256, 264, 520, 1024})
                            for (uint64_t wide : {0, 6, 4096}) {
                                check(T, N, K, dtype, bits, group, N + wide);
                                if (failed) return 1;
                            }
    return checked > 1000000 ? 0 : 2;
}
"""


def test_wavefronts_offsets_lie_inside_the_buffers(tmp_path):
    src, exe = tmp_path / "loads.cpp", tmp_path / "loads"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)])
    done = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stdout
