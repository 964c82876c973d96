// Records of the weight gradient's kernels (gact_weight.hip), filled by its entry point.
#ifndef GACT_WEIGHT_H
#define GACT_WEIGHT_H

#include <stdint.h>

#include "gact_device.h"
#include "gact_heads.h"

namespace gact {

// A block's tile of dW, n x k, the tokens that it takes from memory at a time, and its threads.  Four wavefronts share a tile; where
// there are more, each team of four takes its part of the tokens, and the teams' sums are added in shared memory.
enum { kWeightLarge, kWeightSmall, kWeightLong, kWeightForms };
struct WeightTile {
    int n, k, tokens, threads;
};
constexpr WeightTile weight_tile(int dtype, int which) {
    const int team = dtype == GACT_DT_F32 ? 16 : 32;                // tokens of a team
    return which == kWeightLarge ? WeightTile{256, 128, 2 * team, 512}
         : which == kWeightSmall ? WeightTile{64, 64, team, 256} : WeightTile{64, 64, 4 * team, 1024};
}

struct WeightArgs {
    const uint8_t* dy;
    const uint8_t* packed;
    const float*   gmin;
    const float*   gscale;
    void*          dw;
    void*          db;                  // null: not wanted
    float*         partial;             // [splits][N][K]; null with one split
    float*         db_partial;          // [splits * db_every][N]; null: one block a tile of rows writes db
    int64_t        dy_stride;           // elements from token to token
    uint32_t       T, N, K;
    uint64_t       last_word;           // of the packed string
    uint32_t       last_group;
    uint32_t       group;
    Divisor        by_group;            // of an element's number / 32 by group / 32
    uint32_t       tiles_n, tiles_k, splits;
    uint32_t       chunks;              // of a split
    uint32_t       db_every;            // a block adds every so many-th chunk to db
    uint32_t       dy_chunk, code_chunk, group_chunk;   // bytes from chunk to chunk (kEven)
    int32_t        w_f32;
};

// How a launch loads.
//   kOdd    anything: elements of x in blocks of eight whose codes begin inside bytes and may pass from group to group
//   kWhole  in_features a multiple of eight: whole bytes, one group a block
//   kEven   and out_features of what a lane loads, a chunk's tokens of whole groups, and a split within 2^31 bytes of each of its
//           tensors: offsets are counted on by the wavefront, and what lies behind the end reads as zero
enum { kOdd, kWhole, kEven };
inline int weight_mode(const WeightArgs& a, int dtype, int bits, int which) {
    if (a.K % 8 != 0) return kOdd;
    const uint64_t size = dtype == GACT_DT_F32 ? 4 : 2, BT = (uint64_t)weight_tile(dtype, which).tokens;
    if (a.N % (16 / size) != 0 || BT * a.K % a.group != 0 || a.dy_stride < (int64_t)a.N || a.T == 0) return kWhole;
    const uint64_t tokens = ((uint64_t)a.chunks + 4) * BT, most = 1ull << 31;       // and what is fetched behind the last
    if ((uint64_t)a.dy_stride >= most || tokens * (uint64_t)a.dy_stride * size >= most || tokens * a.K * 4 >= most) return kWhole;
    return kEven;
}

inline uint64_t weight_up(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

struct WeightPlan {
    int which;
    uint32_t tiles_n, tiles_k, chunks, splits, db_every;
    bool db_apart;
};
inline WeightPlan plan_weight(uint64_t T, uint64_t N, uint64_t K, int dtype) {
    WeightPlan p{};
    const uint64_t small = weight_up(N, 64) * (K ? weight_up(K, 64) : 1);
    p.which = N > 128 && K > 64 && T * N * K >= (uint64_t)1 << 28 ? kWeightLarge : small >= 256 || T <= 64 ? kWeightSmall : kWeightLong;
    const WeightTile tile = weight_tile(dtype, p.which);
    p.tiles_n = (uint32_t)weight_up(N, (uint64_t)tile.n);
    p.tiles_k = K ? (uint32_t)weight_up(K, (uint64_t)tile.k) : 1;      // (K = 0: db alone)
    const uint64_t tiles = (uint64_t)p.tiles_n * p.tiles_k, chunks = weight_up(T, (uint64_t)tile.tokens);
    const uint64_t fill = p.which == kWeightSmall ? 512 : 256;
    uint64_t splits = tiles >= fill ? 1 : fill / tiles;
    // a second launch costs as much as a few chunks
    const uint64_t most = chunks <= 12 ? 1 : chunks / 4;
    if (splits > most) splits = most;
    p.chunks = (uint32_t)weight_up(chunks, splits);
    p.splits = p.chunks ? (uint32_t)weight_up(chunks, p.chunks) : 1;
    if (p.splits == 0) p.splits = 1;
    p.db_apart = p.splits > 1;
    p.db_every = p.db_apart ? p.tiles_k : 1;
    return p;
}
inline size_t weight_partial_bytes(const WeightPlan& p, uint64_t N, uint64_t K) {
    return p.splits > 1 ? (size_t)((p.splits * N * K * sizeof(float) + 15) & ~(uint64_t)15) : 0;
}
inline size_t weight_workspace_bytes(const WeightPlan& p, uint64_t N, uint64_t K) {
    return weight_partial_bytes(p, N, K) + (p.db_apart ? (size_t)p.splits * p.db_every * N * sizeof(float) : 0);
}

// Parts that a workgroup of the second launch divides the splits into.
inline int join_parts(uint32_t splits) { return splits >= 64 ? 16 : splits >= 4 ? 4 : 1; }

}  // namespace gact

extern "C" int gact_launch_weight(const gact::WeightArgs* a, int which, int dtype, int bits, void* stream);

#endif
