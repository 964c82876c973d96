// Records of the weight gradient's kernels (gact_weight.hip), filled by its entry point.
#ifndef GACT_WEIGHT_H
#define GACT_WEIGHT_H

#include <stdint.h>

#include <initializer_list>

#include "gact_device.h"
#include "gact_heads.h"

namespace gact {

// A block's tile of dW, n x k, the tokens that it takes from memory at a time, and its threads.  Four wavefronts share a tile; where
// there are more, each team of four takes its part of the tokens, and the teams' sums are added in shared memory.
enum { kWeightLarge, kWeightSmall, kWeightLong, kWeightWide, kWeightTall };
struct WeightTile {
    int n, k, tokens, threads;
};
constexpr WeightTile weight_tile(int dtype, int form) {
    const int team = dtype == GACT_DT_F32 ? 16 : 32;                // tokens of a team
    return form == kWeightLarge ? WeightTile{256, 128, 2 * team, 512}
         : form == kWeightSmall ? WeightTile{64, 64, team, 256}
         : form == kWeightLong ? WeightTile{64, 64, 4 * team, 1024}
         : form == kWeightWide ? WeightTile{32, 128, 4 * team, 1024} : WeightTile{128, 32, 4 * team, 1024};
}
// The chunk that a block of the large forms fetches for chunk `chunk` of a split that ends in front of chunk `end`: behind the last one
// the last again.  Loads take the chunk's distance as the wavefront's offset; what a buffer's end does to one that is itself behind it
// is not asked for.
__host__ __device__ constexpr uint32_t weight_fetched(uint32_t chunk, uint32_t end) { return chunk < end ? chunk : end - 1; }
// Chunks that a block of the small forms has on their way.
constexpr uint32_t weight_depth(int form, bool even) { return even || form == kWeightSmall || form == kWeightLong ? 4 : 2; }

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
    uint32_t       dy_chunk, code_chunk, group_chunk;   // bytes from chunk to chunk, where they are the same
    int32_t        w_f32;
};

// How a launch loads.
//   buffer  dy's rows as words of a buffer: their elements pair up to words, and a split's lie within 2^31 bytes
//   even    blocks of eight elements of x are whole bytes of one group, and a chunk's tokens are whole groups
constexpr uint64_t kWeightReach = 1ull << 31;
inline uint64_t weight_span(const WeightArgs& a, int dtype, int form) {      // tokens of a split, and room for what its last rows' loads pass
    return ((uint64_t)a.chunks + 4) * (uint64_t)weight_tile(dtype, form).tokens;
}
inline bool weight_buffer(const WeightArgs& a, int dtype, int form) {
    if (a.T == 0 || a.dy_stride < (int64_t)a.N || (uint64_t)a.dy_stride >= kWeightReach) return false;
    if (dtype != GACT_DT_F32 && (a.N % 2 != 0 || a.dy_stride % 2 != 0 || (reinterpret_cast<uintptr_t>(a.dy) & 3u) != 0)) return false;
    return weight_span(a, dtype, form) * (uint64_t)a.dy_stride * (dtype == GACT_DT_F32 ? 4u : 2u) < kWeightReach;
}
inline bool weight_even(const WeightArgs& a, int dtype, int form) {
    return a.K % 8 == 0 && (uint64_t)weight_tile(dtype, form).tokens * a.K % a.group == 0;
}

inline uint64_t weight_up(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

struct WeightPlan {
    int form;
    uint32_t tiles_n, tiles_k, chunks, splits, db_every;
};
// A form's tiles and splits.
inline WeightPlan weight_splits(uint64_t T, uint64_t N, uint64_t K, int dtype, int form) {
    WeightPlan p{};
    p.form = form;
    const WeightTile tile = weight_tile(dtype, form);
    p.tiles_n = (uint32_t)weight_up(N, (uint64_t)tile.n);
    p.tiles_k = K ? (uint32_t)weight_up(K, (uint64_t)tile.k) : 1;      // (K = 0: db alone)
    const uint64_t tiles = (uint64_t)p.tiles_n * p.tiles_k, chunks = weight_up(T, (uint64_t)tile.tokens);
    const uint64_t fill = form == kWeightSmall ? 512 : 256;
    uint64_t splits = tiles >= fill ? 1 : fill / tiles;
    // A second launch costs as much as a few chunks, of which those whose blocks of eight are no whole bytes take longer.  Us, 4 bits,
    // one split | splits of two chunks: 1024 x 512 x 512 bf16 9.1 | 11.3 (8 chunks), 1044 x 22 x 3632 bf16 10.6 | 12.3 (9), 1500 x 20 x
    // 500 bf16 18.6 | 11.1 (12), 300 x 256 x 256 fp32 8.6 | 9.9 (5); 3063 x 48 x 200 bf16, of four | two 11.0 | 10.2
    const uint64_t few = dtype == GACT_DT_F32 ? 6 : K % 8 == 0 ? 12 : 8, most = chunks <= few ? 1 : chunks / 2;
    if (splits > most) splits = most;
    // a split's codes lie within kWeightReach
    const uint64_t least = weight_up(T * K, 1ull << 30);
    if (splits < least) splits = least;
    p.chunks = (uint32_t)weight_up(chunks, splits);
    p.splits = p.chunks ? (uint32_t)weight_up(chunks, p.chunks) : 1;
    if (p.splits == 0) p.splits = 1;
    p.db_every = p.splits > 1 ? p.tiles_k : 1;
    return p;
}
// About the us that it takes: products of whole tiles at the rate that the form reaches with the GPU full, rounds of blocks, a second
// launch.  What it goes by, us, large | small | long tiles, 4 bits, by tokens x out x in features:
//   bf16   1024 x 1024 x 1024 25.3 | 16.0 | 8.8    4096 x 1024 x 1024 32.7 | 28.6 | 19.9    8192 x 1024 x 1024 36.6 | 45.5 | 35.9
//          512 x 4096 x 1024 18.7 | 12.9 | 22.5    2048 x 4096 x 1024 39.8 | 35.4 | 43.6    12608 x 1024 x 1024 44.6 | 65.2 | 52.9
//   fp32   1024 x 1024 x 1024 36.1 | 31.1 | 18.7   4096 x 1024 x 1024 58.3 | 90.8 | 63.5    8192 x 1024 x 1024 92.6 | 164 | 121
//          512 x 4096 x 1024 43.7 | 34.9 | 41.5    14645 x 4711 x 104 109 | 239 | 184       128 x 4096 x 1024 20.3 | 13.7 | 22.6
inline double weight_us(const WeightPlan& p, uint64_t T, int dtype) {
    const WeightTile tile = weight_tile(dtype, p.form);
    const double blocks = (double)p.tiles_n * p.tiles_k * p.splits, rounds = (double)weight_up((uint64_t)blocks, 256);
    const double flops = 2.0 * (double)weight_up(T, (uint64_t)tile.tokens) * tile.tokens * p.tiles_n * tile.n * p.tiles_k * tile.k;
    const bool f32 = dtype == GACT_DT_F32;
    const double rate = p.form == kWeightLarge ? (f32 ? 230e6 : 1000e6) : p.form == kWeightLong ? (f32 ? 150e6 : 600e6) : (f32 ? 115e6 : 550e6);
    // blocks of one to a compute unit, in rounds, or of several
    const double full = p.form == kWeightSmall ? (blocks < 600 ? blocks / 600 : 1.0) : blocks / (256 * rounds);
    const double start = p.form == kWeightLarge ? 14 + 4 * rounds : p.form == kWeightLong ? 2 + 3.5 * rounds : 5;
    return start + flops / (rate * full) + (p.splits == 1 ? 0.0 : p.form == kWeightSmall ? 6.0 : 4.0);
}
inline WeightPlan plan_weight(uint64_t T, uint64_t N, uint64_t K, int dtype) {
    if (N <= 32) return weight_splits(T, N, K, dtype, kWeightWide);
    if (K <= 32) return weight_splits(T, N, K, dtype, kWeightTall);
    WeightPlan best = weight_splits(T, N, K, dtype, kWeightSmall);
    if (T <= 64) return best;                          // few tokens: one team has them all
    double us = weight_us(best, T, dtype);
    for (const int form : {kWeightLong, kWeightLarge}) {
        const WeightPlan p = weight_splits(T, N, K, dtype, form);
        const double t = weight_us(p, T, dtype);
        if (t >= us) continue;
        best = p;
        us = t;
    }
    return best;
}
inline size_t weight_partial_bytes(const WeightPlan& p, uint64_t N, uint64_t K) {
    return p.splits > 1 ? (size_t)((p.splits * N * K * sizeof(float) + 15) & ~(uint64_t)15) : 0;
}
inline size_t weight_workspace_bytes(const WeightPlan& p, uint64_t N, uint64_t K) {
    return weight_partial_bytes(p, N, K) + (p.splits > 1 ? (size_t)p.splits * p.db_every * N * sizeof(float) : 0);
}

// Parts that a workgroup of the second launch divides the splits into.
inline int join_parts(uint32_t splits) { return splits >= 64 ? 16 : splits >= 4 ? 4 : 1; }

}  // namespace gact

extern "C" int gact_launch_weight(const gact::WeightArgs* a, int form, int dtype, int bits, void* stream);
extern "C" int gact_launch_weight_f32(const gact::WeightArgs* a, int form, int bits, void* stream);
extern "C" int gact_launch_weight_bf16(const gact::WeightArgs* a, int form, int bits, void* stream);

#endif
