// Records of the per-head norm and rotation kernels (gact_heads.hip), filled by their entry points.
#ifndef GACT_HEADS_H
#define GACT_HEADS_H

#include <stdint.h>

#include "gact_device.h"

namespace gact {

constexpr int kHeadParts = 2;           // queries and keys
constexpr int kHeadWaves = 4;           // wavefronts of a block
constexpr int kMaxHeadDim = 512;        // a head lies in one wavefront, eight elements a lane
// Blocks of a backward launch, each of which leaves one sum of weight gradients per element of a head: as many as the 256 compute
// units hold at a time, a wavefront of each on every SIMD.  The kernels' registers are bounded to that, 96 for five and 128 for
// four: in fp32 five spill where heads of other sizes than 64, 128, 256 are turned by halves.  More blocks than fit take a second,
// short round.  Us, blocks and wavefronts a SIMD 1024, 4 | 1280, 5 | 1280, 4: 8192 tokens of 64 + 16 heads of 160, bf16 152 | 139 |
// 209; 65536 of 12 + 1 of 80 118 | 106 | 149; 13107 of 32 + 8 of 128, 4 bits 68 | 65 | 65; fp32, 65536 of 8 + 4 of 192 364 | 383 |
// 407, of 4 + 4 of 256 328 | 336 | 338.  With six a SIMD all spill.
constexpr int head_backward_waves(int dtype) { return dtype == GACT_DT_F32 ? 4 : 5; }
constexpr uint32_t head_backward_blocks(int dtype) { return 256u * (uint32_t)head_backward_waves(dtype); }
constexpr uint32_t kHeadBackwardBlocks = 1280;          // the most
static_assert(head_backward_blocks(GACT_DT_F32) <= kHeadBackwardBlocks && head_backward_blocks(GACT_DT_BF16) <= kHeadBackwardBlocks,
              "room in the workspace");

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

__host__ __device__ inline uint32_t divided(uint32_t x, const Divisor& d) {
    return d.magic == 0 ? x : (uint32_t)(((uint64_t)x * d.magic) >> 32) >> d.shift;
}

// [batch, token, head, element], elements consecutive, the strides of the others in elements; and, unless kAny, how much
// further on the next pass and the next unit of the same token are.
struct HeadTensor {
    void*   p;
    int64_t batch, token, head;
    int64_t pass, unit;
};
// How the parts of a launch lie (gact_heads.hip).
enum { kAny = 0, kSteady = 1, kFullModes = 3, kLastFullMode = 5 };

// forward: x and y; backward: dy, dx and, without a context, x
enum { kIn, kOut, kX, kHeadTensors };

struct HeadPart {
    HeadTensor t[kHeadTensors];
    const void* w;                      // null: none
    void*       dw;
    float*      rstd;
    uint8_t*    packed;
    float*      gmin;
    float*      gscale;
    float*      partial;                // backward: [blocks][dim]
    uint32_t    rows, heads;            // a row is one head of one token; heads of a token follow each other
    // A pass is 64 >> lanes_shift rows, what a wavefront works on at a time; a unit is `run` passes that it takes one after
    // the other, of the same token (kAny: one pass).  Unit i goes to wavefront i modulo `waves`, four to a block.
    uint32_t    run, units, waves, blocks;
    uint32_t    seed_lo, seed_hi;
    uint32_t    units_per_token, tokens_per_pass;       // one of them 1; both 0: kAny
    Divisor     by_units;               // of a unit's number by units_per_token; kAny: of a row's by heads
    Divisor     row_by_heads;           // of a row's number in a pass by heads
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

// Forward: more blocks than fit, which even out the end.  Us, queries and keys in bf16, 8192 tokens of 32 + 8 heads of 128 |
// the same with 4-bit contexts, 32768 tokens | fp32, 12608 of 16 + 16 of 64, 2 bits, by blocks:
//    1024  30.8 | 192 | 46.4     1536  30.8 | 208 | 48.1     4096  29.7 | 174 | 47.2     8192  29.7 | 173 | 47.0     16384  29.5 | 171 | 47.0
// Longer units share a token's angles and what a unit costs, shorter ones keep what all wavefronts work on at a time closer
// together in memory.  By the passes of a unit:
//    forward   2  28.5 | 184 | 47.1     4  30.6 | 177 | 46.8     8  29.7 | 172 | 46.9     16  29.6 | 170 | 47.2
//    backward of the second  1  176     2  148     4  154     8  165; one of three passes (12 heads of 80)  1  13.0     3  9.0
constexpr uint32_t kHeadForwardBlocks = 8192;
constexpr uint32_t kHeadForwardRun = 8, kHeadBackwardRun = 3;
// Shorter ones in calls that would not fill the GPU otherwise, until this many wavefronts have a unit.  Us, units of 8 | as said: 8
// tokens of 32 + 8 heads of 128 5.2 | 3.0, with 4-bit contexts 7.9 | 3.7, of 64 + 16 of 160 10.4 | 4.4; 128 tokens of the last 11.0
// | 6.9, 1024 of the first 6.5 | 5.5 and 10.1 | 8.5.  (1024 wavefronts: 128 tokens 8.2, 4096: 1024 tokens 8.9, 8192: 10.5.)
constexpr uint32_t kHeadFill = 2048;
inline uint32_t head_most_run(uint64_t passes, uint32_t most) {
    const uint64_t fill = passes / kHeadFill;
    return fill >= most ? most : fill > 1 ? (uint32_t)fill : 1;
}
// Passes of a unit where a token has `passes` of them: all up to `most`, else the most of these that divide them evenly.
inline uint32_t head_run(uint32_t passes, uint32_t most) {
    uint32_t run = passes < most ? passes : most;
    while (passes % run != 0) --run;
    return run;
}
// Whether what lanes add to their unit's addresses, up to `rows` heads and `tokens` tokens, fits 32 bits of bytes.
inline bool lane_offsets_fit(const HeadArgs& a, const HeadPart& p, uint32_t rows, uint32_t tokens, int size) {
    for (const HeadTensor& t : p.t) {
        if (t.head < 0 || t.token < 0 || t.head > 0x7FFFFFFF || t.token > 0x7FFFFFFF) return false;
        if (((rows - 1) * (uint64_t)t.head + (tokens - 1) * (uint64_t)t.token + (uint64_t)a.dim) * (uint64_t)size > 0xFFFFFFFFull) return false;
    }
    return true;
}
// Divides a part into units, from its rows, heads and strides of elements of `size` bytes; returns its mode.  run: most passes of a
// unit; 0: as kAny, so that it can go into a launch with one that is.
inline int lay_out_heads(const HeadArgs& a, HeadPart* p, uint32_t run, int size) {
    const uint32_t rows = 64u >> a.lanes_shift;          // of a pass
    p->run = 1;
    p->units = (p->rows + rows - 1) / rows;
    p->units_per_token = p->tokens_per_pass = 0;
    if (run != 0 && p->heads % rows == 0 && lane_offsets_fit(a, *p, rows, 1, size)) {
        p->run = head_run(p->heads / rows, run);
        p->units_per_token = p->heads / rows / p->run;
        p->tokens_per_pass = 1;
        p->units /= p->run;
    } else if (run != 0 && rows % p->heads == 0 && a.seq % (rows / p->heads) == 0 &&
               lane_offsets_fit(a, *p, p->heads, rows / p->heads, size)) {
        p->units_per_token = 1;
        p->tokens_per_pass = rows / p->heads;
    }
    p->by_units = divisor(p->units_per_token ? p->units_per_token : p->heads);
    for (HeadTensor& t : p->t) {
        t.pass = t.head * rows;
        t.unit = t.pass * p->run;
    }
    if (p->units_per_token == 0) return kAny;
    return a.dim == 8 << a.lanes_shift && a.lanes_shift >= kFullModes && a.lanes_shift <= kLastFullMode ? a.lanes_shift : kSteady;
}
inline uint64_t head_passes(const HeadPart& p) { return (uint64_t)p.units * p.run; }
// Blocks of the parts of a launch, at most `all`, dealt by their passes.
inline void plan_heads(HeadPart* part, int parts, uint32_t all) {
    uint64_t passes = 0;
    for (int k = 0; k < parts; ++k) passes += head_passes(part[k]);
    for (int k = 0; k < parts; ++k) {
        HeadPart& p = part[k];
        // rounded up, for every part of all but kHeadParts blocks
        const uint64_t most = passes == 0 ? 0 : ((uint64_t)(all - kHeadParts) * head_passes(p) + passes - 1) / passes;
        const uint64_t need = ((uint64_t)p.units + kHeadWaves - 1) / kHeadWaves;
        p.blocks = (uint32_t)(need < most ? need : most);
        p.waves = p.blocks * kHeadWaves;
    }
}

// The launches of a staged call: one where the parts have the same kind of context, in a mode that both have, else one for
// each.  (Parts that lie differently in launches of their own, with all the blocks of one each, are no faster: 12 query
// heads of 80 and one key head, 1021 tokens, forward 8.8 us, together 4.8; 28 and 7 of 128, 30001 tokens 112.6, 112.4.)
struct HeadLaunches {
    bool together;
    int mode[kHeadParts];
};
inline HeadLaunches arrange_heads(HeadArgs* a, int n_parts, const int* part_bits, int dtype, bool backward) {
    HeadLaunches l{};
    const int size = dtype == GACT_DT_F32 ? 4 : 2;
    uint64_t rows = 0;
    for (int k = 0; k < n_parts; ++k) rows += a->part[k].rows;
    const uint32_t run = head_most_run(rows >> (6 - a->lanes_shift), backward ? kHeadBackwardRun : kHeadForwardRun);
    for (int k = 0; k < n_parts; ++k) l.mode[k] = lay_out_heads(*a, &a->part[k], run, size);
    l.together = n_parts == 1 || part_bits[0] == part_bits[1];
    if (l.together && n_parts > 1 && l.mode[0] != l.mode[1])
        for (int k = 0; k < n_parts; ++k) l.mode[k] = lay_out_heads(*a, &a->part[k], 0, size);
    const uint32_t blocks = backward ? head_backward_blocks(dtype) : kHeadForwardBlocks;
    if (l.together) plan_heads(a->part, n_parts, blocks);
    else for (int k = 0; k < n_parts; ++k) plan_heads(&a->part[k], 1, blocks);
    return l;
}

// Where a unit begins.  steady (a part whose mode is not kAny): for all lanes of the wavefront; kAny: a unit is one pass, and
// this is the place of its row `lane_row`, or of the part's last row.
struct UnitPlace {
    uint32_t token, at, batch, head;    // at: the token's place in its sequence; head: steady: in units
};
__host__ __device__ inline UnitPlace unit_place(const HeadArgs& a, const HeadPart& p, bool steady, uint32_t unit,
                                                uint32_t lane_row, int lanes_shift) {
    UnitPlace u;
    if (steady) {
        u.token = divided(unit, p.by_units);
        u.head = unit - u.token * p.units_per_token;
        u.token *= p.tokens_per_pass;
    } else {
        uint32_t row = (unit << (6 - lanes_shift)) + lane_row;
        row = row < p.rows ? row : p.rows - 1;
        u.token = divided(row, p.by_units);
        u.head = row - u.token * p.heads;
    }
    u.batch = divided(u.token, a.by_seq);
    u.at = u.token - u.batch * a.seq;
    return u;
}
// Elements of a tensor in front of it; what a lane adds to its token, and to the elements in front of its row.
__host__ __device__ inline int64_t unit_first(const HeadTensor& t, bool steady, const UnitPlace& u) {
    return (int64_t)u.batch * t.batch + (int64_t)u.at * t.token + (int64_t)u.head * (steady ? t.unit : t.head);
}
__host__ __device__ inline uint32_t lane_token(const HeadPart& p, bool steady, uint32_t lane_row) {
    return steady && p.tokens_per_pass > 1 ? divided(lane_row, p.row_by_heads) : 0;
}
__host__ __device__ inline int64_t lane_first(const HeadPart& p, const HeadTensor& t, bool steady, uint32_t lane_row, uint32_t token) {
    return steady ? (int64_t)(lane_row - token * p.heads) * t.head + (int64_t)token * t.token : 0;
}

}  // namespace gact

// bits: 0 without a context
extern "C" int gact_launch_heads(const gact::HeadArgs* a, int mode, int dtype, int bits, int halves, int backward, void* stream);
extern "C" int gact_launch_heads_dw(const gact::HeadArgs* a, int parts, void* stream);

#endif
