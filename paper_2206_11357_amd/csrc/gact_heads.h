// Records of the per-head norm and rotation kernels (gact_heads.hip), filled by their entry points.
#ifndef GACT_HEADS_H
#define GACT_HEADS_H

#include <stdint.h>

#include "gact_device.h"

namespace gact {

constexpr int kHeadParts = 2;           // queries and keys
constexpr int kHeadWaves = 4;           // wavefronts of a block
constexpr int kMaxHeadDim = 512;        // a head lies in one wavefront, eight elements a lane
// Blocks of a backward launch over all parts: each leaves one sum of weight gradients per element of a head.
constexpr uint32_t kHeadBackwardBlocks = 1024;

// x / d for x < 2^31, as a product: floor(2^(32+s) / d) + 1 with 2^(s+1) >= d (Granlund, Montgomery 1994, Thm. 4.2,
// as group_divisor); magic 0 stands for d = 1.
struct Divisor {
    uint32_t magic;
    int32_t  shift;
};
inline Divisor divisor(uint32_t d) {
    if (d <= 1) return Divisor{0, 0};
    int32_t s = 0;
    while (((uint64_t)2 << s) < d) ++s;
    return Divisor{(uint32_t)(((uint64_t)1 << (32 + s)) / d + ((d & (d - 1)) != 0 ? 1 : 0)), s};
}

// [batch, token, head, element], elements consecutive, the strides of the others in elements
struct HeadTensor {
    void*   p;
    int64_t batch, token, head;
};

struct HeadPart {
    HeadTensor in, out;                 // forward: x and y; backward: dy and dx
    HeadTensor x;                       // backward without a context
    const void* w;                      // null: none
    void*       dw;
    float*      rstd;
    uint8_t*    packed;
    float*      gmin;
    float*      gscale;
    float*      partial;                // backward: [blocks][dim]
    uint32_t    rows, heads;            // a row is one head of one token; heads of a token follow each other
    uint32_t    passes, run, blocks;    // of 64 >> lanes_shift rows; of one wavefront; of this part
    uint32_t    seed_lo, seed_hi;
    Divisor     by_heads;
};

struct HeadArgs {
    HeadPart part[kHeadParts];
    const float*   cos;                 // [n_positions][rot / 2]
    const float*   sin;
    const int64_t* positions;           // of each token; null: its place in its sequence
    int64_t        n_positions;
    Divisor        by_seq;
    uint32_t       seq;
    float          eps, inv_dim;
    int32_t        dim;
    int32_t        lanes_shift;         // log2 of a head's lanes
    int32_t        rot_lanes;           // rot / 8
    // context: lanes of a group; rows >> row_shift where a group is one head or several, else groups a row and
    // log2 of a group's elements
    int32_t        group_lanes, row_shift, groups_per_row, group_shift;
    int32_t        w_f32;
};

// Blocks and passes of each part.  Forward: a wavefront takes up to eight neighbouring passes, fewer where that would leave
// wavefronts out.
constexpr uint32_t kHeadRun = 8, kHeadForwardWaves = 8192;
inline void plan_heads(HeadArgs* a, int parts) {
    uint64_t passes = 0;
    for (int k = 0; k < parts; ++k) passes += a->part[k].passes;
    const uint64_t even = passes / kHeadForwardWaves;
    uint32_t run = even < 1 ? 1 : even > kHeadRun ? kHeadRun : (uint32_t)even;
    // more only where a launch would have too many threads: beyond what fits the memory
    while (!launchable(passes / ((uint64_t)run * kHeadWaves) + kHeadParts, 64 * kHeadWaves)) run *= 2;
    for (int k = 0; k < parts; ++k) {
        HeadPart& p = a->part[k];
        p.run = run;
        p.blocks = (uint32_t)(((uint64_t)p.passes + run * kHeadWaves - 1) / (run * kHeadWaves));
    }
}
// Backward: kHeadBackwardBlocks blocks at most, dealt to the parts by their passes.
inline void plan_heads_backward(HeadArgs* a, int parts) {
    uint64_t passes = 0;
    for (int k = 0; k < parts; ++k) passes += a->part[k].passes;
    // every part of all but kHeadParts blocks rounds down
    const uint64_t slots = (uint64_t)(kHeadBackwardBlocks - kHeadParts) * kHeadWaves;
    const uint32_t run = (uint32_t)((passes + slots - 1) / slots);
    for (int k = 0; k < parts; ++k) {
        HeadPart& p = a->part[k];
        p.run = run;
        p.blocks = run == 0 ? 0 : (uint32_t)(((uint64_t)p.passes + (uint64_t)run * kHeadWaves - 1) / ((uint64_t)run * kHeadWaves));
    }
}

}  // namespace gact

// bits: 0 without a context
extern "C" int gact_launch_heads(const gact::HeadArgs* a, int dtype, int bits, int halves, int backward, void* stream);
extern "C" int gact_launch_heads_dw(const gact::HeadArgs* a, int parts, void* stream);

#endif
