// Weight gradient of a linear layer from the compressed context of its input, for MI355X (gfx950).
//
//   dW[n, k] = sum over t of dy[t, n] x^[t, k],   db[n] = sum over t of dy[t, n],   x^ = code * step + minimum
//
// A matrix product whose right operand is decoded on its way into shared memory: codes are read from HBM, never x^.
// Both operands have the summed axis outermost.  bf16: rows of tokens in shared memory as they come, read transposed
// (ds_read_b64_tr_b16: four tokens of a column a lane), 32x32x16 products; fp32: 32x32x2 products, whose operands are a
// row's elements as they lie.  A wavefront holds its part of dW in registers; the next tokens are on their way from
// HBM meanwhile, and are decoded behind the products of the present ones.
// The tokens are split over blocks where the tiles of dW are too few for the GPU; the splits' sums are added in a fixed
// order by a second launch.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "gact_codec.h"
#include "gact_device.h"
#include "gact_weight.h"

namespace gact {

typedef uint32_t w4 __attribute__((ext_vector_type(4)));
typedef uint32_t w2 __attribute__((ext_vector_type(2)));
typedef w4 w4_any2 __attribute__((aligned(2)));
typedef w4 w4_any4 __attribute__((aligned(4)));
typedef float wf4 __attribute__((ext_vector_type(4)));
typedef float wf2 __attribute__((ext_vector_type(2)));
typedef float wf16 __attribute__((ext_vector_type(16)));
typedef short ws4 __attribute__((ext_vector_type(4)));
typedef __bf16 wb8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------- codes of x
// Eight codes from element e on, and what they stand for.
template <int BITS>
struct Codes {
    uint32_t lo, hi;
    float mn[2], step[2];
    uint32_t turn;                                     // the first of the eight that is of the next group; 8: none
};
template <int BITS, bool WHOLE>
__device__ __forceinline__ Codes<BITS> load_x(const WeightArgs& a, uint64_t e) {
    Codes<BITS> c;
    const uint32_t g = divided((uint32_t)(e >> 5), a.by_group);
    c.mn[0] = a.gmin[g];
    c.step[0] = a.gscale[g];
    c.hi = 0;
    if (WHOLE) {                                       // e is a multiple of eight: whole bytes, one group
        const uint8_t* p = a.packed + (e >> 3) * BITS;
        if (BITS == 1) c.lo = *p;
        if (BITS == 2) c.lo = *(const uint16_t*)p;
        if (BITS == 4) c.lo = *(const uint32_t*)p;
        if (BITS == 8) { const w2 w = *(const w2*)p; c.lo = w.x; c.hi = w.y; }
        c.turn = 8;
        c.mn[1] = c.mn[0];
        c.step[1] = c.step[0];
    } else {
        const uint64_t end = (uint64_t)(g + 1) * a.group - e;
        c.turn = end < 8 ? (uint32_t)end : 8u;
        const uint32_t g1 = g < a.last_group ? g + 1 : g;
        c.mn[1] = a.gmin[g1];
        c.step[1] = a.gscale[g1];
        const uint32_t* words = (const uint32_t*)a.packed;
        const uint64_t bit = e * BITS;
        const uint64_t i = bit >> 5, j = i < a.last_word ? i + 1 : i, l = j < a.last_word ? j + 1 : j;
        const uint32_t s = (uint32_t)bit & 31u;
        const uint32_t b = words[j];
        c.lo = __builtin_amdgcn_alignbit(b, words[i], s);
        if (BITS == 8) c.hi = __builtin_amdgcn_alignbit(words[l], b, s);
    }
    return c;
}
// 4 bits: every other nibble of a word, so that its bytes convert in place (an empty statement keeps the compiler from
// taking each nibble out by itself).
template <int BITS>
__device__ __forceinline__ void part_codes(Codes<BITS>& c) {
    if (BITS != 4) return;
    c.hi = c.lo >> 4 & 0x0F0F0F0Fu;
    c.lo &= 0x0F0F0F0Fu;
    asm("" : "+v"(c.lo), "+v"(c.hi));
}
// Value j of them in binary32, as gact_decompress has it: the product is rounded before the sum.  (In one instruction, a few bf16
// values in a million come out a step apart: 1.5e-5 of a dW of 12608 tokens, 8 bits, where 1.8e-7 is its own sums'.)
template <int BITS, bool WHOLE>
__device__ __forceinline__ float value_of(const Codes<BITS>& c, int j) {
    const uint32_t word = BITS == 8 ? (j >= 4 ? c.hi : c.lo) : BITS == 4 && (j & 1) != 0 ? c.hi : c.lo;
    const uint32_t q = BITS == 8 ? word >> (8 * (j & 3)) & 0xFFu
                     : BITS == 4 ? word >> (8 * (j >> 1)) & 0xFFu
                     : word >> (j * BITS) & ((1u << BITS) - 1u);
    const bool next = !WHOLE && (uint32_t)j >= c.turn;
    const float step = next ? c.step[1] : c.step[0], mn = next ? c.mn[1] : c.mn[0];
    const float t = (float)q * step;
    return t + mn;
}

// ---------------------------------------------------------------- buffer loads
// From a buffer of so many bytes, at an offset of the lane's and one of the wavefront's; zeros behind the end.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const void* p, uint64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(uint32_t)bytes, 0x00027000);
}
__device__ __forceinline__ uint32_t buffer_word(Buffer b, uint32_t lane, uint32_t wave) {
    return __builtin_amdgcn_raw_buffer_load_b32(b, lane, wave, 0);
}
template <int BITS>
__device__ __forceinline__ void buffer_codes(Buffer b, uint32_t lane, uint32_t wave, Codes<BITS>& c) {
    c.hi = 0;
    if (BITS == 1) c.lo = __builtin_amdgcn_raw_buffer_load_b8(b, lane, wave, 0);
    if (BITS == 2) c.lo = __builtin_amdgcn_raw_buffer_load_b16(b, lane, wave, 0);
    if (BITS == 4) c.lo = buffer_word(b, lane, wave);
    if (BITS == 8) {
        const w2 w = __builtin_bit_cast(w2, __builtin_amdgcn_raw_buffer_load_b64(b, lane, wave, 0));
        c.lo = w.x;
        c.hi = w.y;
    }
}

// ------------------------------------------------------------------ the tiles
template <int DT>
struct Operand {
    typedef wb8 type;
};
template <>
struct Operand<GACT_DT_F32> {
    typedef float type;
};
template <int DT, int WHICH>
struct Tiling {
    static constexpr WeightTile tile = weight_tile(DT, WHICH);
    static constexpr int BN = tile.n, BK = tile.k, BT = tile.tokens, kThreads = tile.threads, kTeams = kThreads / 256;
    static constexpr int kSize = DT == GACT_DT_F32 ? 4 : 2;
    static constexpr int kPiece = 16 / kSize;                       // elements of dy that a lane loads at a time
    static constexpr int kRowPieces = BN / kPiece;
    static constexpr int kPieces = BT * kRowPieces / kThreads;
    static constexpr int kRowBlocks = BK / 8;                       // blocks of eight elements of x
    static constexpr int kBlocks = BT * kRowBlocks >= kThreads ? BT * kRowBlocks / kThreads : 1;
    // Bytes from row to row in shared memory.  bf16: 64 more than a multiple of 256, so that the four rows of a
    // transposed read lie in different banks.
    static constexpr int kPad = DT == GACT_DT_F32 ? 0 : 64;
    static constexpr int kRowN = BN * kSize + kPad, kRowK = BK * kSize + kPad;
    static constexpr int kBufN = BT * kRowN, kBuf = kBufN + BT * kRowK;
    static constexpr int TN = BN / 64, TK = BK / 64;                // 32 x 32 products of a wavefront, 2 x 2 of which share a tile
    static_assert(kThreads % kRowPieces == 0 && BT * kRowPieces % kThreads == 0, "a thread stays in its column");
};

// bytes of a buffer: all that a split reaches lies below 2^31 (weight_mode)
__device__ __forceinline__ uint64_t within(uint64_t bytes) { return bytes < 0x80000000ull ? bytes : 0x80000000ull; }

template <int DT, int BITS, int WHICH, int MODE>
__global__ __launch_bounds__(weight_tile(DT, WHICH).threads, weight_tile(DT, WHICH).threads == 1024 ? 4 : 2) void weight_kernel(WeightArgs a) {
    typedef Tiling<DT, WHICH> L;
    constexpr bool WHOLE = MODE != kOdd;
    constexpr int BN = L::BN, BK = L::BK, BT = L::BT, TN = L::TN, TK = L::TK;
    __shared__ __align__(16) uint8_t lds[2][L::kBuf];
    const uint32_t tid = threadIdx.x;
    const int lane = (int)tid & 63, wave = (int)__builtin_amdgcn_readfirstlane((int)(tid >> 6));

    // Blocks of one XCD (every eighth) are neighbours in the order split, rows, columns: they share tokens in its L2.
    const uint32_t total = gridDim.x, per = total >> 3, rest = total & 7u, xcd = blockIdx.x & 7u;
    uint32_t b = xcd * per + (xcd < rest ? xcd : rest) + (blockIdx.x >> 3);
    const uint32_t tiles = a.tiles_n * a.tiles_k;
    const uint32_t split = b / tiles;
    b -= split * tiles;
    const uint32_t tile_n = b / a.tiles_k, tile_k = b - tile_n * a.tiles_k;
    const uint32_t n0 = tile_n * BN, k0 = tile_k * BK;
    const uint32_t all = (a.T + BT - 1) / BT;
    const uint32_t c0 = split * a.chunks, c1 = c0 + a.chunks < all ? c0 + a.chunks : all;

    // ---- what a thread loads
    const uint32_t pn = tid % L::kRowPieces, pt = tid / L::kRowPieces;
    constexpr uint32_t kRows = L::kThreads / L::kRowPieces;      // rows from piece to piece of a thread
    const uint32_t n = n0 + pn * L::kPiece;
    const uint32_t valid = n < a.N ? (a.N - n < (uint32_t)L::kPiece ? a.N - n : (uint32_t)L::kPiece) : 0;
    const uint32_t bk = tid % L::kRowBlocks, bt = tid / L::kRowBlocks;
    constexpr uint32_t kXRows = L::kThreads / L::kRowBlocks;
    const uint32_t k = k0 + bk * 8;
    const bool x_thread = BT * L::kRowBlocks >= L::kThreads || bt < (uint32_t)BT;

    w4 dy[L::kPieces];
    Codes<BITS> codes[L::kBlocks];
    // kEven: a split's rows, codes, minima and steps as buffers from its first token on; a lane's offsets in them stay, the
    // wavefront's go on from chunk to chunk.  What lies behind the last token reads as zero.
    Buffer in_dy, in_codes, in_mn, in_step;
    uint32_t dy_at[L::kPieces], code_at[L::kBlocks], group_at[L::kBlocks];
    if constexpr (MODE == kEven) {
        const uint64_t t0 = (uint64_t)c0 * BT, tokens = a.T - t0;
        in_dy = buffer_of(a.dy + t0 * a.dy_stride * L::kSize, within(((tokens - 1) * a.dy_stride + a.N) * L::kSize));
        in_codes = buffer_of(a.packed + t0 * a.K / 8 * BITS, within(tokens * a.K / 8 * BITS));
        const uint64_t g0 = t0 * a.K / a.group, groups = (uint64_t)a.last_group + 1 - g0;
        in_mn = buffer_of(a.gmin + g0, within(groups * 4));
        in_step = buffer_of(a.gscale + g0, within(groups * 4));
#pragma unroll
        for (int q = 0; q < L::kPieces; ++q) dy_at[q] = ((pt + q * kRows) * (uint32_t)a.dy_stride + n) * L::kSize;
#pragma unroll
        for (int q = 0; q < L::kBlocks; ++q) {
            const uint32_t e = (bt + q * kXRows) * a.K + k;
            code_at[q] = e / 8 * BITS;
            group_at[q] = divided(e >> 5, a.by_group) * 4;
        }
    }
    const auto fetch_dy = [&](uint32_t chunk, int q) {
        dy[q] = __builtin_bit_cast(w4, __builtin_amdgcn_raw_buffer_load_b128(in_dy, dy_at[q], (chunk - c0) * a.dy_chunk, 0));
    };
    const auto fetch_x = [&](uint32_t chunk, int q) {
        const uint32_t i = chunk - c0;
        buffer_codes<BITS>(in_codes, code_at[q], i * a.code_chunk, codes[q]);
        codes[q].mn[0] = __builtin_bit_cast(float, buffer_word(in_mn, group_at[q], i * a.group_chunk));
        codes[q].step[0] = __builtin_bit_cast(float, buffer_word(in_step, group_at[q], i * a.group_chunk));
    };
    const auto fetch = [&](uint32_t chunk) {
        if constexpr (MODE == kEven) {
#pragma unroll
            for (int q = 0; q < L::kPieces; ++q) fetch_dy(chunk, q);
#pragma unroll
            for (int q = 0; q < L::kBlocks; ++q) fetch_x(chunk, q);
            return;
        }
        const uint32_t t0 = chunk * BT;
#pragma unroll
        for (int q = 0; q < L::kPieces; ++q) {
            const uint32_t t = t0 + pt + q * kRows;
            w4 v = {0u, 0u, 0u, 0u};
            if (t < a.T && valid != 0) {
                const uint8_t* p = a.dy + ((int64_t)t * a.dy_stride + n) * L::kSize;
                if (valid == (uint32_t)L::kPiece) {
                    if (DT == GACT_DT_F32) v = *(const w4_any4*)p;
                    else v = *(const w4_any2*)p;
                } else {
                    uint32_t h[8];
#pragma unroll
                    for (int j = 0; j < L::kPiece; ++j)
                        h[j] = (uint32_t)j < valid ? (DT == GACT_DT_F32 ? ((const uint32_t*)p)[j] : ((const uint16_t*)p)[j]) : 0u;
                    if (DT == GACT_DT_F32) v = w4{h[0], h[1], h[2], h[3]};
                    else v = w4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4 % L::kPiece] | h[5 % L::kPiece] << 16,
                                h[6 % L::kPiece] | h[7 % L::kPiece] << 16};
                }
            }
            dy[q] = v;
        }
#pragma unroll
        for (int q = 0; q < L::kBlocks; ++q) {
            const uint32_t t = t0 + bt + q * kXRows;
            codes[q] = Codes<BITS>{};
            if (x_thread && t < a.T && k < a.K) codes[q] = load_x<BITS, WHOLE>(a, (uint64_t)t * a.K + k);
        }
    };
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
    const auto add_db = [&] {
#pragma unroll
        for (int q = 0; q < L::kPieces; ++q)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t v = dy[q][j];
                if (DT == GACT_DT_F32) sum[j] += __builtin_bit_cast(float, v);
                else {
                    sum[2 * j] += __builtin_bit_cast(float, v << 16);
                    sum[2 * j + 1] += __builtin_bit_cast(float, v & 0xFFFF0000u);
                }
            }
    };
    const auto place_dy = [&](uint8_t* buf, int q) { *(w4*)(buf + (pt + q * kRows) * L::kRowN + pn * 16) = dy[q]; };
    const auto place_x = [&](uint8_t* buf, int q, const float (&x)[8]) {
        uint8_t* p = buf + L::kBufN + (bt + q * kXRows) * L::kRowK + bk * (8 * L::kSize);
        if (DT == GACT_DT_F32) {
            *(wf4*)p = wf4{x[0], x[1], x[2], x[3]};
            *(wf4*)(p + 16) = wf4{x[4], x[5], x[6], x[7]};
        } else {
            *(w4*)p = w4{bf16_pair_rne(x[0], x[1]), bf16_pair_rne(x[2], x[3]), bf16_pair_rne(x[4], x[5]), bf16_pair_rne(x[6], x[7])};
        }
    };
    const auto place = [&](uint8_t* buf) {
#pragma unroll
        for (int q = 0; q < L::kPieces; ++q) place_dy(buf, q);
        if (!x_thread) return;
#pragma unroll
        for (int q = 0; q < L::kBlocks; ++q) {
            float x[8];
            part_codes<BITS>(codes[q]);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = value_of<BITS, WHOLE>(codes[q], j);
            place_x(buf, q, x);
        }
    };

    // ---- what a wavefront multiplies
    const int team = wave >> 2, wn = wave >> 1 & 1, wk = wave & 1;
    wf16 acc[TN][TK];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TK; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    // Operands of step s of a chunk in registers: part i of the rows, part j of the columns, of a 32 x 32 product each.
    //   bf16  a step is 16 tokens; 16 lanes read 4 rows of 16 elements, of which each gets a column
    //   fp32  a step is two tokens; a lane's operands are TN (TK) neighbouring elements of row 2 s + lane / 32
    typedef typename Operand<DT>::type Op;
    constexpr int kSteps = BT / L::kTeams / (DT == GACT_DT_F32 ? 2 : 16);      // of a team
    const uint32_t op_row = (uint32_t)(team * (BT / L::kTeams) + (DT == GACT_DT_F32 ? lane >> 5 : 8 * (lane >> 5) + ((lane & 15) >> 2)));
    const int col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const uint32_t op_n = op_row * L::kRowN + (DT == GACT_DT_F32 ? (wn * 32 * TN + (lane & 31) * TN) * 4 : (wn * 32 * TN + col) * 2);
    const uint32_t op_k = L::kBufN + op_row * L::kRowK + (DT == GACT_DT_F32 ? (wk * 32 * TK + (lane & 31) * TK) * 4 : (wk * 32 * TK + col) * 2);
    const auto columns = [](const uint8_t* p, int stride) {
        typedef __attribute__((address_space(3))) ws4* lds_ptr;
        union { ws4 h[2]; Op v; } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * stride));
        return u.v;
    };
    const auto read_n = [&](const uint8_t* buf, int s, int i, Op (&x)[TN]) {
        if constexpr (DT == GACT_DT_F32) {
            if (i == 0) __builtin_memcpy(x, __builtin_assume_aligned(buf + op_n + 2 * s * L::kRowN, 4 * TN), 4 * TN);
        } else {
            x[i] = columns(buf + op_n + 16 * s * L::kRowN + 64 * i, L::kRowN);
        }
    };
    const auto read_k = [&](const uint8_t* buf, int s, Op (&y)[TK]) {
        if constexpr (DT == GACT_DT_F32) {
            __builtin_memcpy(y, __builtin_assume_aligned(buf + op_k + 2 * s * L::kRowK, 4 * TK), 4 * TK);
        } else {
#pragma unroll
            for (int j = 0; j < TK; ++j) y[j] = columns(buf + op_k + 16 * s * L::kRowK + 64 * j, L::kRowK);
        }
    };
    const auto product = [&](int i, const Op (&x)[TN], const Op (&y)[TK]) {
#pragma unroll
        for (int j = 0; j < TK; ++j) {
            if constexpr (DT == GACT_DT_F32) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[j], acc[i][j], 0, 0, 0);
            else acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], y[j], acc[i][j], 0, 0, 0);
        }
    };
    const auto multiply = [&](const uint8_t* buf) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            Op x[TN], y[TK];
            read_k(buf, s, y);
#pragma unroll
            for (int i = 0; i < TN; ++i) read_n(buf, s, i, x);
#pragma unroll
            for (int i = 0; i < TN; ++i) product(i, x, y);
        }
    };
    // Large tiles: chunk c is multiplied while chunk c + 1 is placed, the first of its blocks decoded a step ahead, and c + 2
    // fetched, a little of each behind every row of products, in this order: two wavefronts of a SIMD that do one after the other
    // fall into step and leave the matrix unit idle together.  A step's operands are read during the step before it, so that
    // all of a chunk's have been read by the beginning of its last step; there the one barrier of a chunk stands: behind it chunk
    // c + 1 is whole, and the place of chunk c is free.
    // Without a question, also behind the split's last chunk, where nothing is read outside the buffers and nothing uses what is
    // placed.
    constexpr int kEarly = kSteps == 2 ? L::kBlocks / 2 : 0;
    Op x[2][TN], y[2][TK];
    float v[L::kBlocks][8];
    const auto decode = [&](uint32_t next, int e) {
        const int q = e / 8;
        if (e % 8 == 0) part_codes<BITS>(codes[q]);
        v[q][e % 8] = value_of<BITS, WHOLE>(codes[q], e % 8);
        if (e % 8 == 7) fetch_x(next, q);
    };
    const auto read_all = [&](const uint8_t* buf) {
        read_k(buf, 0, y[0]);
#pragma unroll
        for (int i = 0; i < TN; ++i) read_n(buf, 0, i, x[0]);
    };
    const auto flow = [&](const uint8_t* buf, uint8_t* other, uint32_t c) {
        constexpr int kSlots = (kSteps - 1) * TN, kValues = 8 * (L::kBlocks - kEarly);
#pragma unroll
        for (int s = 0; s + 1 < kSteps; ++s)
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                const int slot = s * TN + i;
                product(i, x[s & 1], y[s & 1]);
                if (i == 0) read_k(buf, s + 1, y[(s + 1) & 1]);
                read_n(buf, s + 1, i, x[(s + 1) & 1]);
#pragma unroll
                for (int q = 0; q < kEarly; ++q)
                    if (slot == q) place_x(other, q, v[q]);
#pragma unroll
                for (int e = slot * kValues / kSlots; e < (slot + 1) * kValues / kSlots; ++e) {
                    decode(c + 2, 8 * kEarly + e);
                    if (e % 8 == 7) place_x(other, kEarly + e / 8, v[kEarly + e / 8]);
                }
#pragma unroll
                for (int q = 0; q < L::kPieces; ++q)
                    if (slot == q * kSlots / L::kPieces) {
                        place_dy(other, q);
                        fetch_dy(c + 2, q);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            product(i, x[(kSteps - 1) & 1], y[(kSteps - 1) & 1]);
            if (i == 0) read_k(other, 0, y[0]);
            read_n(other, 0, i, x[0]);
#pragma unroll
            for (int e = i * 8 * kEarly / TN; e < (i + 1) * 8 * kEarly / TN; ++e) decode(c + 3, e);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    const bool with_db = a.db != nullptr && (a.db_partial || tile_k == 0);
    // the next chunk that this block adds to db
    uint32_t db_next = with_db && a.db_partial ? c0 + (tile_k + a.db_every - c0 % a.db_every) % a.db_every : with_db ? c0 : ~0u;
    const auto adds = [&](uint32_t chunk) {
        if (chunk != db_next) return false;
        db_next += a.db_every;
        return true;
    };
    if (c0 < c1) {
        fetch(c0);
        if (adds(c0)) add_db();
        place(lds[0]);
        if constexpr (MODE == kEven && WHICH == kWeightLarge) {
            fetch(c0 + 1);
            __syncthreads();
            read_all(lds[0]);
#pragma unroll
            for (int e = 0; e < 8 * kEarly; ++e) decode(c0 + 2, e);
            for (uint32_t c = c0; c < c1; ++c) {
                const uint32_t now = (c - c0) & 1u;
                if (c + 1 < c1 && adds(c + 1)) add_db();
                flow(lds[now], lds[now ^ 1u], c);
            }
            __syncthreads();
        } else {
            if (c0 + 1 < c1) fetch(c0 + 1);
            __syncthreads();
            for (uint32_t c = c0; c < c1; ++c) {
                const uint32_t now = (c - c0) & 1u;
                if (c + 1 < c1) {
                    if (adds(c + 1)) add_db();
                    place(lds[now ^ 1u]);
                    if (c + 2 < c1) fetch(c + 2);
                }
                multiply(lds[now]);
                __syncthreads();
            }
        }
    }

    // ---- the teams' sums, through shared memory.  Two teams: each hands half of its products to the other, a row of products at a
    // time, and is left with the other half's sums; more: the first adds them all.
    constexpr int kMine = L::kTeams == 2 ? TN / 2 : TN;             // rows of products that a wavefront writes
    const int first = L::kTeams == 2 ? team * kMine : 0;
    float* room = (float*)lds[0] + (tid & 255u);
    constexpr int kRow = TK * 16 * 256;
    if constexpr (L::kTeams == 2) {
        static_assert(TN % 2 == 0 && 2 * kRow * 4 <= 2 * L::kBuf, "room");
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < TK; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    if (team == 0) room[(j * 16 + r) * 256] = acc[kMine + i][j][r];
                    else room[kRow + (j * 16 + r) * 256] = acc[i][j][r];
                }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < TK; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    // the first team's first, for both
                    if (team == 0) acc[i][j][r] = acc[i][j][r] + room[kRow + (j * 16 + r) * 256];
                    else acc[i][j][r] = room[(j * 16 + r) * 256] + acc[kMine + i][j][r];
                }
        }
    } else if constexpr (L::kTeams > 2) {
        static_assert(TN == 1 && (L::kTeams - 1) * kRow * 4 <= 2 * L::kBuf, "room");
        if (team > 0) {
#pragma unroll
            for (int j = 0; j < TK; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) room[(team - 1) * kRow + (j * 16 + r) * 256] = acc[0][j][r];
        }
        __syncthreads();
        if (team == 0) {
#pragma unroll
            for (int t = 0; t < L::kTeams - 1; ++t)
#pragma unroll
                for (int j = 0; j < TK; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[0][j][r] += room[t * kRow + (j * 16 + r) * 256];
        }
    }

    // ---- out: element r of a product is row (r & 3) + 8 (r >> 2) + 4 (lane / 32), column lane % 32
    const bool whole = a.partial == nullptr, inside = n0 + BN <= a.N && k0 + BK <= a.K;
    const int low = lane >> 5, at_k = lane & 31;
    // of a lane: row, column, and their elements; of row r of products i: what all lanes add to them
    const uint32_t lane_n = n0 + (uint32_t)(wn * 32 * TN + (DT == GACT_DT_F32 ? 4 * low * TN + first : first * 32 + 4 * low));
    const uint32_t lane_k = k0 + (uint32_t)(wk * 32 * TK + (DT == GACT_DT_F32 ? at_k * TK : at_k));
    const auto put = [&](auto* to) {
        typedef typename std::remove_pointer<decltype(to)>::type Out;
        to += (size_t)lane_n * a.K + lane_k;
#pragma unroll
        for (int i = 0; i < kMine; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t row = (uint32_t)((r & 3) + 8 * (r >> 2)), n = DT == GACT_DT_F32 ? row * TN + i : i * 32 + row;
                if (!inside && lane_n + n >= a.N) continue;
                Out* p = to + (size_t)n * a.K;
#pragma unroll
                for (int j = 0; j < TK; ++j) {
                    const uint32_t k = DT == GACT_DT_F32 ? j : j * 32;
                    if (!inside && lane_k + k >= a.K) continue;
                    if constexpr (sizeof(Out) == 4) p[k] = acc[i][j][r];
                    else p[k] = (Out)bf16_pair_rne(acc[i][j][r], 0.0f);
                }
            }
    };
    if (L::kTeams <= 2 || team == 0) {
        if (!whole) put(a.partial + (size_t)split * a.N * a.K);
        else if (a.w_f32) put((float*)a.dw);
        else put((uint16_t*)a.dw);
    }

    if (L::kTeams > 1) __syncthreads();
    if (!with_db) return;
    // db of the tile's rows: over the threads of a column, in their order
    float* sums = (float*)lds[0];
#pragma unroll
    for (int j = 0; j < L::kPiece; ++j) sums[pt * BN + pn * L::kPiece + j] = sum[j];
    __syncthreads();
    for (uint32_t i = tid; i < (uint32_t)BN; i += L::kThreads) {
        if (n0 + i >= a.N) continue;
        float s = 0.0f;
        for (uint32_t r = 0; r < kRows; ++r) s += sums[r * BN + i];
        if (a.db_partial) a.db_partial[((size_t)split * a.db_every + tile_k) * a.N + n0 + i] = s;
        else if (a.w_f32) ((float*)a.db)[n0 + i] = s;
        else ((uint16_t*)a.db)[n0 + i] = (uint16_t)bf16_pair_rne(s, 0.0f);
    }
}

// dW and db from the splits' sums.  A workgroup takes 1024 / PARTS neighbouring elements of dW, four a thread, and each
// PARTS-th of the splits goes to one of its PARTS parts, whose sums are added in their order; the workgroups behind them add db
// likewise, a thread an element.  Many splits are those of a small dW, whose elements alone would not fill the GPU.
constexpr int kJoinThreads = 256;
__device__ __forceinline__ void put_weight(void* p, int f32, size_t i, float v) {
    if (f32) ((float*)p)[i] = v;
    else ((uint16_t*)p)[i] = (uint16_t)bf16_pair_rne(v, 0.0f);
}
template <int PARTS>
__global__ __launch_bounds__(kJoinThreads) void weight_join_kernel(WeightArgs a, uint32_t dw_blocks) {
    constexpr uint32_t kEach = kJoinThreads / PARTS;
    __shared__ wf4 lds[PARTS][kEach];
    const uint32_t part = threadIdx.x / kEach, j = threadIdx.x % kEach;
    const bool of_db = blockIdx.x >= dw_blocks;
    const size_t n = of_db ? a.N : (size_t)a.N * a.K;
    const size_t i = ((size_t)(of_db ? blockIdx.x - dw_blocks : blockIdx.x) * kEach + j) * 4;
    const float* from = of_db ? a.db_partial : a.partial;
    const uint32_t terms = of_db ? a.splits * a.db_every : a.splits;
    wf4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (i < n) {
        if (n % 4 == 0) {
#pragma unroll 8
            for (uint32_t k = part; k < terms; k += PARTS) {
                const wf4 v = *(const wf4*)(from + k * n + i);
#pragma unroll
                for (int c = 0; c < 4; ++c) s[c] += v[c];
            }
        } else {
            for (uint32_t k = part; k < terms; k += PARTS)
#pragma unroll
                for (int c = 0; c < 4; ++c) s[c] += i + c < n ? from[k * n + i + c] : 0.0f;
        }
    }
    if (PARTS > 1) {
        lds[part][j] = s;
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int k = 1; k < PARTS; ++k)
#pragma unroll
            for (int c = 0; c < 4; ++c) s[c] += lds[k][j][c];
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (i + c < n) put_weight(of_db ? a.db : a.dw, a.w_f32, i + c, s[c]);
}

// ------------------------------------------------------------- host launchers
template <int DT, int BITS, int WHICH>
static void launch_tile(const WeightArgs& a, hipStream_t s) {
    const dim3 grid(a.tiles_n * a.tiles_k * a.splits), block(weight_tile(DT, WHICH).threads);
    switch (weight_mode(a, DT, BITS, WHICH)) {
        case kEven: hipLaunchKernelGGL((weight_kernel<DT, BITS, WHICH, kEven>), grid, block, 0, s, a); break;
        case kWhole: hipLaunchKernelGGL((weight_kernel<DT, BITS, WHICH, kWhole>), grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL((weight_kernel<DT, BITS, WHICH, kOdd>), grid, block, 0, s, a); break;
    }
}
template <int DT, int BITS>
static void launch_bits(const WeightArgs& a, int which, hipStream_t s) {
    switch (which) {
        case kWeightLarge: launch_tile<DT, BITS, kWeightLarge>(a, s); break;
        case kWeightSmall: launch_tile<DT, BITS, kWeightSmall>(a, s); break;
        default: launch_tile<DT, BITS, kWeightLong>(a, s); break;
    }
}
template <int DT>
static void launch_type(const WeightArgs& a, int which, int bits, hipStream_t s) {
    switch (bits) {
        case 1: launch_bits<DT, 1>(a, which, s); break;
        case 2: launch_bits<DT, 2>(a, which, s); break;
        case 4: launch_bits<DT, 4>(a, which, s); break;
        default: launch_bits<DT, 8>(a, which, s); break;
    }
}

}  // namespace gact

extern "C" int gact_launch_weight(const gact::WeightArgs* a, int which, int dtype, int bits, void* stream) {
    const hipStream_t s = (hipStream_t)stream;
    if (dtype == GACT_DT_F32) gact::launch_type<GACT_DT_F32>(*a, which, bits, s);
    else gact::launch_type<GACT_DT_BF16>(*a, which, bits, s);
    if (hipGetLastError() != hipSuccess) return -1;
    if (a->splits > 1) {
        const int parts = gact::join_parts(a->splits);
        const uint64_t n = (uint64_t)a->N * a->K, each = 4 * gact::kJoinThreads / parts;
        const uint32_t dw_blocks = (uint32_t)((n + each - 1) / each);
        const uint32_t db_blocks = a->db ? (uint32_t)((a->N + each - 1) / each) : 0;
        const dim3 grid(dw_blocks + db_blocks), block(gact::kJoinThreads);
        switch (parts) {
            case 1: hipLaunchKernelGGL(gact::weight_join_kernel<1>, grid, block, 0, s, *a, dw_blocks); break;
            case 4: hipLaunchKernelGGL(gact::weight_join_kernel<4>, grid, block, 0, s, *a, dw_blocks); break;
            default: hipLaunchKernelGGL(gact::weight_join_kernel<16>, grid, block, 0, s, *a, dw_blocks); break;
        }
        if (hipGetLastError() != hipSuccess) return -1;
    }
    return 0;
}
