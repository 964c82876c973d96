// Records of the group norm's kernels (gact_group_norm.hip), filled by their entry points.
#ifndef GACT_GROUP_NORM_H
#define GACT_GROUP_NORM_H

#include <stdint.h>

#include "gact_device.h"
#include "gact_heads.h"

namespace gact {

constexpr int kGnThreads = 256;

// [sample, pixel, channel], channels consecutive, the strides of the others in elements.
struct GnTensor {
    void*   p;
    int64_t sample, pixel;
};

// Work goes by blocks of eight channels.  Kernels that add over pixels: a thread stays in its column, one such block, a
// workgroup takes `rows` pixels of `cols` columns at a time, of one sample and one chunk of its pixels.
struct GnArgs {
    GnTensor x, y, dy, dx;
    const void* w;                      // null: ones
    const void* b;                      // null: zeros
    void*       dw;                     // null: not wanted
    void*       db;
    float*      mean;                   // [samples][H]
    float*      rstd;
    uint8_t*    packed;
    float*      gmin;
    float*      gscale;
    float*      partial;                // of each sample, chunk and channel (or column): two floats
    float*      sums;                   // backward: of each sample and channel: sum of dz, sum of dz n
    float*      means;                  // backward: of each sample, group and slice of 64 channels: its part of mean g, mean g n
    uint32_t    B, P, C, H, D;
    uint32_t    slices;                 // of a group
    uint32_t    C8, cols, rows, slabs;  // columns of a workgroup; cols * slabs >= C8
    uint32_t    chunks, batch, batches; // pixels of a batch; a sample's
    uint32_t    blocks8;                // B P C / 8
    uint32_t    period, passes;         // a pass is 64 blocks; lanes come back to their channels after `period` passes
    uint32_t    stride_passes;
    uint32_t    dx_blocks;
    Divisor     by_c8, by_p, by_d, by_cols;
    uint32_t    seed_lo, seed_hi;
    uint32_t    block_shift;            // log2 of a context group's blocks of eight
    float       eps;
    int32_t     w_f32;
    double      inv;                    // 1 / (P D)
    // Kernels that hold their maps in registers: a workgroup takes the whole of a sample's next few units, a unit being a group of
    // the norm, or as many groups as are whole columns.  A unit's columns are lanes 0 .. unit_cols - 1 of 2^unit_shift.
    uint32_t    units, unit_cols, unit_shift, slab_shift, col_shift;       // slab_shift: log2 of a slab's units; col_shift: of its lanes
    uint32_t    unit_slabs, norm_blocks;
};

inline uint32_t gn_up(uint64_t a, uint64_t b) { return (uint32_t)((a + b - 1) / b); }

// Whether a block of eight channels lies in one group of the norm.
inline bool gn_uniform(const GnArgs& a) { return a.D % 8 == 0; }

// Of a launch that adds over pixels, about.  More leave more sums to add up behind them.  Us, sums and their addition, 2048 | 1024 | 768:
// 9 x 1023 x 1136 bf16 in 8 groups, 8 bits 28.7 | 26.0 | 27.3, statistics 23.3 | 19.9 | 15.9; 1 x 262144 x 128 42.4 | 36.3 | 38.6.
constexpr uint32_t kGnBlocks = 1024;
// Pixels that a thread of these takes at a time; a workgroup's are a batch.  Chunks take batches in turn, so that what all workgroups read
// at a time is one region of a sample.
constexpr uint32_t gn_batch(int dtype) { return dtype == GACT_DT_F32 ? 4 : 8; }

inline void plan_group_norm(GnArgs* a, int dtype) {
    a->C8 = a->C / 8;
    a->slices = gn_up(a->D, 64);
    a->slabs = gn_up(a->C8, kGnThreads);
    a->cols = gn_up(a->C8, a->slabs);
    a->rows = (uint32_t)kGnThreads / a->cols;
    a->by_c8 = divisor(a->C8);
    a->by_p = divisor(a->P);
    a->by_d = divisor(a->D);
    a->by_cols = divisor(a->cols);
    a->inv = 1.0 / ((double)a->P * a->D);
    a->blocks8 = a->B * a->P * a->C8;
    const uint64_t want = kGnBlocks / ((uint64_t)a->B * a->slabs) ? kGnBlocks / ((uint64_t)a->B * a->slabs) : 1;
    a->batch = a->rows * gn_batch(dtype);
    a->batches = gn_up(a->P, a->batch);
    a->chunks = want < a->batches ? (uint32_t)want : a->batches;
    uint32_t g = a->C8, h = 64;
    while (h) { const uint32_t t = g % h; g = h; h = t; }            // greatest common divisor
    a->period = a->C8 / g;
    a->passes = gn_up(a->blocks8, 64);
    uint32_t waves = a->passes / 4 ? a->passes / 4 : 1;
    if (waves > 16384) waves = 16384;
    a->stride_passes = gn_up(waves, a->period) * a->period;
}
// Workgroups that hold `threads` x `blocks` blocks of eight.
struct GnWhole {
    uint32_t threads, blocks;
};
constexpr int kGnWholes = 4;
constexpr GnWhole kGnWhole[kGnWholes] = {{256, 4}, {512, 8}, {1024, 8}, {512, 25}};
// The last, of wavefronts with all the registers that two to a SIMD have: backward, from codes; fp32 without an activation, whose slope
// would take more than there are.  Us by the others (64 bytes of a pixel, bf16 32) | by it (128, 64): 64 x 3136 x 256 fp32 131 | 113, with SiLU
// 143 | 184, from x 188 | 192; 16 x 2304 x 512 bf16 36.1 | 25.6, 64 x 3136 x 256 bf16, SiLU 104 | 101.
constexpr bool gn_held(int dtype, int bits, bool silu) { return bits != 0 && (dtype != GACT_DT_F32 || !silu); }
// Whether a sample's group fits the registers of a workgroup: which of them it is (0: of none, 1 ..), and how it is laid out.  held:
// the last may be it (which is never the one where there would be none without).
inline int plan_whole(GnArgs* a, int dtype, bool backward, bool held) {
    uint32_t g = a->D, h = 8;                          // their greatest common divisor
    while (h) { const uint32_t t = g % h; g = h; h = t; }
    const uint32_t cols = a->D / g;                     // whole groups in whole columns
    a->unit_cols = cols;
    a->units = a->C8 / cols;
    a->unit_shift = 0;
    while ((1u << a->unit_shift) < cols) ++a->unit_shift;
    if (a->unit_shift > 6) return 0;
    // 64 bytes of a pixel at least, if they fit.  Us, step of 32 x 1024 x 512 bf16, 4 bits, forward + backward, by bytes: 32 29.1 + 27.8,
    // 64 26.2 + 22.6, 128 (twice the threads) 29.7 + 21.9; of 64 x 3136 x 256 fp32, 2 bits 32 162 + 170, 64 136 + 131.
    const uint32_t size = dtype == GACT_DT_F32 ? 4 : 2;
    uint32_t shift = 0;
    // (and where there are few pixels, columns enough for the threads)
    while (((cols << shift) * 8 * size < 64 || (uint64_t)a->P << (a->unit_shift + shift) < kGnWhole[0].threads) &&
           (1u << shift) < a->units && a->unit_shift + shift < 6)
        ++shift;
    const auto fits = [&](const GnWhole& w) { return (uint64_t)a->P << (a->unit_shift + shift) <= (uint64_t)w.threads * w.blocks; };
    // (Groups that are no whole columns take more registers than the largest has: 16 x 500 x 72 bf16 in 4 groups, 4 bits, 18.5 us
    // forward, 24.1 backward; in passes over memory 15.3 and 20.4.)
    const int most = g == 8 ? 3 : 2;
    while (!fits(kGnWhole[most - 1]) && shift > 0) --shift;
    if (!fits(kGnWhole[most - 1])) return 0;
    // A cache line of a pixel, where the workgroups still fill the GPU.  Us, 64 bytes | 128 | 256: backward, 2 and 4 bits, 64 x 1024 x 256 fp32
    // 39.0 | 29.6 | 27.2, 256 x 784 x 256 fp32 130 | 102 | 101, 64 x 1024 x 512 bf16 SiLU 48.8 | 39.7, 128 x 784 x 256 bf16 29.0 | 30.2 | 31.4;
    // forward 256 x 784 x 256 fp32 131 | 123, 64 x 1024 x 256 fp32 38.5 | 35.1, 128 x 256 x 640 bf16 in groups of 20 84 | 63, 64 x 196 x
    // 1024 bf16 19.3 | 24.6, in workgroups of twice the threads 128 x 1568 x 256 fp32 131 | 145.
    const int largest = !backward ? 2 : held && g == 8 ? kGnWholes : most;
    if (backward || dtype == GACT_DT_F32 || g != 8) {
        while ((cols << shift) * 8 * size < 128 && (1u << shift) < a->units && a->unit_shift + shift < 6 &&
               (uint64_t)a->B * gn_up(a->units, 2u << shift) >= 256) {
            ++shift;
            if (fits(kGnWhole[largest - 1])) continue;
            --shift;
            break;
        }
    }
    a->slab_shift = shift;
    a->col_shift = a->unit_shift + shift;
    a->unit_slabs = gn_up(a->units, 1u << shift);
    a->norm_blocks = a->B * a->unit_slabs;
    for (int k = 0; k < (largest > most ? largest : most); ++k) if (fits(kGnWhole[k])) return k + 1;
    return 0;
}
inline size_t gn_align(size_t v) { return (v + 15) & ~(size_t)15; }
// Workspace: partial sums; forward: mean and rstd where the caller keeps none; backward: sums, means.  Maps held in registers:
// sums alone.
inline size_t gn_partial_bytes(const GnArgs& a) {
    return gn_align((size_t)a.B * a.chunks * a.C * 2 * sizeof(float));
}
inline size_t gn_sums_bytes(const GnArgs& a) { return gn_align((size_t)a.B * a.C * 2 * sizeof(float)); }
inline size_t gn_forward_bytes(const GnArgs& a, int whole) {
    return whole ? 0 : gn_partial_bytes(a) + 2 * gn_align((size_t)a.B * a.H * sizeof(float));
}
inline size_t gn_backward_bytes(const GnArgs& a, int whole) {
    if (whole) return a.B > 1 ? gn_sums_bytes(a) : 0;
    return gn_partial_bytes(a) + gn_sums_bytes(a) + gn_align((size_t)a.B * a.H * a.slices * 2 * sizeof(float));
}

}  // namespace gact

// bits: 0 without a context; act: 0 none, 1 silu
// whole: what plan_whole gave
extern "C" int gact_launch_group_norm(const gact::GnArgs* a, int dtype, int bits, int act, int whole, void* stream);
extern "C" int gact_launch_group_norm_backward(const gact::GnArgs* a, int dtype, int bits, int act, int whole, void* stream);
extern "C" int gact_launch_group_norm_zero(const gact::GnArgs* a, void* stream);       // dw and db of nothing

#endif
