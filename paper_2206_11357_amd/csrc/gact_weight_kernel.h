// Weight gradient of a linear layer from the compressed context of its input, for MI355X (gfx950).
//
//   dW[n, k] = sum over t of dy[t, n] x^[t, k],   db[n] = sum over t of dy[t, n],   x^ = code * step + minimum
//
// A matrix product whose right operand is decoded on its way into shared memory: codes are read from HBM, never x^.
// Both operands have the summed axis outermost: rows of tokens in shared memory as they come, read transposed
// (ds_read_b64_tr_b16: four tokens of a column a lane), 32x32x16 products of bf16, fp32 in three parts.  A wavefront holds
// its part of dW in registers; the next tokens are on their way from HBM meanwhile, and are decoded behind the products of
// the present ones.
// The tokens are split over blocks where the tiles of dW are too few for the GPU; the splits' sums are added in a fixed
// order by a second launch.
// Measured, us with that launch: 32768 x 1024 x 4096 bf16, 4 bits 280 to 302 from card to card (a library's product of values
// decompressed before 336), 8192 x 4096 x 1024 85 to 91 (93), 169343 x 256 x 256 fp32, 2 bits 117 to 133 (502).  Bound by the matrix
// unit at the clock that the power allows, the decoding and the writes to shared memory beside it: of the first's 289 to 304 on one
// card 266 without fetching, 259 without decoding, 205 without the writes, 206 without products, 205 with products and their reads
// alone.
#ifndef GACT_WEIGHT_KERNEL_H
#define GACT_WEIGHT_KERNEL_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "gact_codec.h"
#include "gact_device.h"
#include "gact_weight.h"

namespace gact {

typedef uint32_t w4 __attribute__((ext_vector_type(4)));
typedef uint32_t w3 __attribute__((ext_vector_type(3)));
typedef uint32_t w2 __attribute__((ext_vector_type(2)));
typedef w4 w4_any2 __attribute__((aligned(2)));
typedef w4 w4_any4 __attribute__((aligned(4)));
typedef float wf4 __attribute__((ext_vector_type(4)));
typedef float wf16 __attribute__((ext_vector_type(16)));
typedef short ws4 __attribute__((ext_vector_type(4)));
typedef __bf16 wb8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------- buffer loads
// From a buffer of so many bytes, at an offset of the lane's and one of the wavefront's, which lies inside; words behind its end are
// zero.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const void* p, uint64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(uint32_t)(bytes < 0x80000000ull ? bytes : 0x80000000ull), 0x00027000);
}
constexpr uint32_t kBehind = 0x80000000u;              // behind the end of any
__device__ __forceinline__ uint32_t buffer_word(Buffer b, uint32_t lane, uint32_t wave) {
    return __builtin_amdgcn_raw_buffer_load_b32(b, lane, wave, 0);
}
__device__ __forceinline__ w2 buffer_words2(Buffer b, uint32_t lane, uint32_t wave) {
    return __builtin_bit_cast(w2, __builtin_amdgcn_raw_buffer_load_b64(b, lane, wave, 0));
}

// ---------------------------------------------------------------- codes of x
// Eight codes from some element on, and what they stand for.  EVEN: whole bytes, of one group; else they begin at bit `shift` of
// w[0], and those from `turn` on are of the next group (8: none).
template <int BITS, bool EVEN>
struct Codes {
    uint32_t w[EVEN ? (BITS == 8 ? 2 : 1) : (BITS == 8 ? 3 : 2)];
    uint32_t odd;                                      // 4 bits: every other nibble (part)
    float    mn[EVEN ? 1 : 2], step[EVEN ? 1 : 2];
    uint32_t shift, turn;

    __device__ __forceinline__ void load(Buffer codes, uint32_t lane, uint32_t wave) {
        if constexpr (EVEN) {
            if (BITS == 1) w[0] = __builtin_amdgcn_raw_buffer_load_b8(codes, lane, wave, 0);
            if (BITS == 2) w[0] = __builtin_amdgcn_raw_buffer_load_b16(codes, lane, wave, 0);
            if (BITS == 4) w[0] = buffer_word(codes, lane, wave);
            if constexpr (BITS == 8) { const w2 v = buffer_words2(codes, lane, wave); w[0] = v.x; w[1] = v.y; }
        } else if constexpr (BITS == 8) {
            const w3 v = __builtin_bit_cast(w3, __builtin_amdgcn_raw_buffer_load_b96(codes, lane, wave, 0));
            w[0] = v.x; w[1] = v.y; w[2] = v.z;
        } else {
            const w2 v = buffer_words2(codes, lane, wave);
            w[0] = v.x; w[1] = v.y;
        }
    }
    // Makes the codes begin at bit 0 of w[0].  4 bits: and takes every other nibble of the word apart, so that bytes convert in place (an
    // empty statement keeps the compiler from taking out each nibble by itself).
    __device__ __forceinline__ void part() {
        if constexpr (!EVEN) {
            w[0] = __builtin_amdgcn_alignbit(w[1], w[0], shift);
            if constexpr (BITS == 8) w[1] = __builtin_amdgcn_alignbit(w[2], w[1], shift);
        }
        if constexpr (BITS == 4) {
            odd = w[0] >> 4 & 0x0F0F0F0Fu;
            w[0] &= 0x0F0F0F0Fu;
            asm("" : "+v"(w[0]), "+v"(odd));
        }
    }
    // Value j in binary32, as gact_decompress has it: the product is rounded before the sum.  (In one instruction, a few bf16 values in a
    // million come out a step apart: 1.5e-5 of a dW of 12608 tokens, 8 bits, where 1.8e-7 is its own sums'.)
    __device__ __forceinline__ float value(int j) const {
        const uint32_t word = BITS == 8 && j >= 4 ? w[BITS == 8 ? 1 : 0] : BITS == 4 && (j & 1) != 0 ? odd : w[0];
        const uint32_t q = BITS == 8 ? word >> (8 * (j & 3)) & 0xFFu
                         : BITS == 4 ? word >> (8 * (j >> 1)) & 0xFFu
                         : word >> (j * BITS) & ((1u << BITS) - 1u);
        const bool next = !EVEN && (uint32_t)j >= turn;
        const float s = next ? step[EVEN ? 0 : 1] : step[0], m = next ? mn[EVEN ? 0 : 1] : mn[0];
        const float t = (float)q * s;
        return t + m;
    }
};

// ------------------------------------------------------------------ the tiles
template <int DT, int FORM>
struct Tiling {
    static constexpr WeightTile tile = weight_tile(DT, FORM);
    static constexpr int BN = tile.n, BK = tile.k, BT = tile.tokens, kThreads = tile.threads, kTeams = kThreads / 256;
    static constexpr int kSize = DT == GACT_DT_F32 ? 4 : 2;
    static constexpr int kPiece = 16 / kSize;                       // elements of dy that a lane loads at a time
    static constexpr int kRowPieces = BN / kPiece;
    static constexpr int kRowBlocks = BK / 8;                       // blocks of eight elements of x
    // a thread's; where there are more threads than pieces (blocks), the last ones have none
    static constexpr int kPieces = BT * kRowPieces >= kThreads ? BT * kRowPieces / kThreads : 1;
    static constexpr int kBlocks = BT * kRowBlocks >= kThreads ? BT * kRowBlocks / kThreads : 1;
    static constexpr int kRowsN = kThreads / kRowPieces, kRowsK = kThreads / kRowBlocks;      // rows from one of a thread's to the next
    // 32 x 32 products of a wavefront; a team's four lie 2 x 2, or in a row where a tile is narrow
    static constexpr int kWavesN = BN == 32 ? 1 : BK == 32 ? 4 : 2, kWavesK = 4 / kWavesN;
    static constexpr int TN = BN / 32 / kWavesN, TK = BK / 32 / kWavesK;
    // Shared memory: rows of tokens in bf16; fp32: in three parts, each a row.  The four rows of a transposed read, 64 bytes each, lie
    // in different banks.
    static constexpr int kParts = DT == GACT_DT_F32 ? 3 : 1;
    static constexpr int part(int elements) { return elements * 2 + (elements * 2 % 256 == 64 || elements * 2 % 256 == 192 ? 0 : 64); }
    static constexpr int kPartN = part(BN), kPartK = part(BK), kRowN = kParts * kPartN, kRowK = kParts * kPartK;
    static constexpr int kBufN = BT * kRowN, kBuf = kBufN + BT * kRowK;
    // where two do not fit, a chunk's operands are all read before the next one is placed
    static constexpr int kBufs = FORM == kWeightLarge && DT == GACT_DT_F32 ? 1 : 2;
    static_assert(kRowN % 256 == 64 || kRowN % 256 == 192, "banks");
    static_assert(kRowK % 256 == 64 || kRowK % 256 == 192, "banks");
    static_assert(kThreads % kRowPieces == 0 && kThreads % kRowBlocks == 0, "a thread stays in its column");
};

// Where a wavefront's operands lie in a chunk, and its products.  A step is 16 tokens; 16 lanes read 4 rows of 16 elements, of which
// each gets a column.
//   fp32  An element is the sum of three bf16, each the rounded rest of the ones before: 8 bits and a sign each, exactly (an infinity,
//         and what bf16 rounds to one, leaves NaN, of which weight_element makes what it has to be).  Of the nine products of their
//         parts the six largest are taken.  The second part is at most 2^-8 of the element and the third 2^-17, so that the others
//         come to at most 2^-24 of a product, as much as its rounding to binary32 would; sums are binary32.  Six products of bf16
//         take 6 x 32 cycles of the matrix unit for 16 tokens, eight of fp32 8 x 64: 169343 x 256 x 256 takes 124 us with the sums'
//         addition, 184 in fp32, and comes closer to the sum in 64 bits (6.8e-7 of it; the decompressed product by the library
//         4.0e-6).
template <int DT, int FORM>
struct Products {
    typedef Tiling<DT, FORM> L;
    static constexpr int TN = L::TN, TK = L::TK, kParts = L::kParts;
    static constexpr int kSteps = L::BT / L::kTeams / 16;                                    // of a team
    struct Op {
        wb8 part[kParts];
    };
    uint32_t at_n, at_k;
    wf16 acc[TN][TK];
    __device__ __forceinline__ Products(int lane, int team, int wn, int wk) {
        const uint32_t row = (uint32_t)(team * (L::BT / L::kTeams) + 8 * (lane >> 5) + ((lane & 15) >> 2));
        const int col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
        at_n = row * L::kRowN + (uint32_t)(wn * 32 * TN + col) * 2;
        at_k = L::kBufN + row * L::kRowK + (uint32_t)(wk * 32 * TK + col) * 2;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TK; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    }
    static __device__ __forceinline__ Op columns(const uint8_t* p, int row, int part) {
        typedef __attribute__((address_space(3))) ws4* lds_ptr;
        Op op;
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            union { ws4 h[2]; wb8 v; } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + k * part));
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + k * part + 4 * row));
            op.part[k] = u.v;
        }
        return op;
    }
    __device__ __forceinline__ void read_n(const uint8_t* buf, int s, int i, Op (&x)[TN]) const {
        x[i] = columns(buf + at_n + 16 * s * L::kRowN + 64 * i, L::kRowN, L::kPartN);
    }
    __device__ __forceinline__ void read_k(const uint8_t* buf, int s, Op (&y)[TK]) const {
#pragma unroll
        for (int j = 0; j < TK; ++j) y[j] = columns(buf + at_k + 16 * s * L::kRowK + 64 * j, L::kRowK, L::kPartK);
    }
    __device__ __forceinline__ void read(const uint8_t* buf, int s, Op (&x)[TN], Op (&y)[TK]) const {
        read_k(buf, s, y);
#pragma unroll
        for (int i = 0; i < TN; ++i) read_n(buf, s, i, x);
    }
    __device__ __forceinline__ void product(int i, const Op (&x)[TN], const Op (&y)[TK]) {
        // parts whose numbers add up to less than kParts, the small products first
#pragma unroll
        for (int sum = kParts - 1; sum >= 0; --sum)
#pragma unroll
            for (int p = 0; p <= sum; ++p)
#pragma unroll
                for (int j = 0; j < TK; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i].part[p], y[j].part[sum - p], acc[i][j], 0, 0, 0);
    }
    __device__ __forceinline__ void chunk(const uint8_t* buf) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            Op x[TN], y[TK];
            read(buf, s, x, y);
#pragma unroll
            for (int i = 0; i < TN; ++i) product(i, x, y);
        }
    }
};

// What a thread has of a chunk on its way.
template <int DT, int BITS, int FORM, bool EVEN>
struct Slot {
    w4 dy[Tiling<DT, FORM>::kPieces];
    Codes<BITS, EVEN> codes[Tiling<DT, FORM>::kBlocks];
};
// Loads a thread's part of a split's chunks and places it in shared memory.
//   BUFFER  dy through a buffer whose end stops it, offsets counted on by the wavefront; else token by token, with questions
//   EVEN    so are the codes, minima and steps; else each block looks for its word and its groups
template <int DT, int BITS, int FORM, bool BUFFER, bool EVEN>
struct Loader {
    typedef Tiling<DT, FORM> L;
    typedef Slot<DT, BITS, FORM, EVEN> S;
    const WeightArgs& a;
    uint32_t c0, pn, pt, bk, bt, n, k;
    Buffer in_dy, in_codes, in_mn, in_step;
    uint32_t at_dy[L::kPieces], at_code[L::kBlocks], at_group[L::kBlocks];
    uint32_t first_group, short_chunk;                 // the tensor's last chunk, where it has fewer tokens than the others (else none)
    uint64_t element;                                  // of block 0 in chunk c0

    __device__ __forceinline__ Loader(const WeightArgs& args, uint32_t n0, uint32_t k0, uint32_t chunk) : a(args), c0(chunk) {
        const uint32_t tid = threadIdx.x;
        pn = tid % L::kRowPieces;
        pt = tid / L::kRowPieces;
        bk = tid % L::kRowBlocks;
        bt = tid / L::kRowBlocks;
        n = n0 + pn * L::kPiece;
        k = k0 + bk * 8;
        const uint64_t t0 = (uint64_t)c0 * L::BT, tokens = a.T - t0;
        if constexpr (BUFFER) {
            in_dy = buffer_of(a.dy + t0 * a.dy_stride * L::kSize, ((tokens - 1) * a.dy_stride + a.N) * L::kSize);
#pragma unroll
            for (int q = 0; q < L::kPieces; ++q) at_dy[q] = ((pt + q * L::kRowsN) * (uint32_t)a.dy_stride + n) * L::kSize;
        }
        // from the last 32 elements on that begin at or in front of the first: a word's begin, and the group's that they are of
        const uint64_t from = t0 * a.K >> 5 << 5, all = (uint64_t)a.T * a.K;
        first_group = divided((uint32_t)(from >> 5), a.by_group);
        const uint64_t groups = all ? (uint64_t)a.last_group + 1 - first_group : 0;      // (in_features 0: db alone)
        in_codes = buffer_of(a.packed + (from >> 3) * BITS, EVEN || all == 0 ? (all - from) / 8 * BITS : (a.last_word + 1) * 4 - (from >> 3) * BITS);
        in_mn = buffer_of(a.gmin + first_group, groups * 4);
        in_step = buffer_of(a.gscale + first_group, groups * 4);
        element = (t0 + bt) * a.K + k;
        short_chunk = a.T % L::BT != 0 ? a.T / L::BT : ~0u;
        if constexpr (EVEN) {
#pragma unroll
            for (int q = 0; q < L::kBlocks; ++q) {
                const uint64_t e = element + (uint64_t)q * L::kRowsK * a.K;
                at_code[q] = (uint32_t)((e - from) >> 3) * BITS;
                at_group[q] = (divided((uint32_t)(e >> 5), a.by_group) - first_group) * 4;
            }
        }
    }
    __device__ __forceinline__ bool with_dy() const { return L::BT * L::kRowPieces >= L::kThreads || pt < (uint32_t)L::BT; }
    __device__ __forceinline__ bool with_x() const { return L::BT * L::kRowBlocks >= L::kThreads || bt < (uint32_t)L::BT; }

    __device__ __forceinline__ void fetch_dy(S& s, uint32_t chunk, int q) const {
        if constexpr (BUFFER) {
            s.dy[q] = __builtin_bit_cast(w4, __builtin_amdgcn_raw_buffer_load_b128(in_dy, at_dy[q], (chunk - c0) * a.dy_chunk, 0));
        } else {
            // A piece that passes its row's end takes what follows there, which no product of a stored element uses, but nothing from
            // behind the last row's.
            const uint64_t t = (uint64_t)chunk * L::BT + pt + q * L::kRowsN;
            const int64_t at = (int64_t)t * a.dy_stride + n, end = (int64_t)(a.T - 1) * a.dy_stride + a.N;
            w4 v = {0u, 0u, 0u, 0u};
            if (t < a.T && n < a.N) {
                const uint8_t* p = a.dy + at * L::kSize;
                const uint32_t valid = a.N - n;
                if (valid >= (uint32_t)L::kPiece || (a.dy_stride >= (int64_t)a.N && at + L::kPiece <= end)) {
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
            s.dy[q] = v;
        }
    }
    // Tokens behind the last are behind the codes' end, but their elements may be some of the last group's, whose minimum or step, where it
    // is not finite, dy's zeros would not take out of the sums: they have none.  To be called for blocks first .. end - 1 of a thread in front
    // of a chunk's fetch_x; the tensor's last chunk is fetched after all others.  (Asked in fetch_x, for each block, in turn with
    // this: 32768 x 1024 x 4096 bf16 281.4 us | 280.2, 12608 x 1024 x 1024 46.4 | 45.6, and more registers spilled.)
    __device__ __forceinline__ void cut(uint32_t chunk, int first, int end) {
        if constexpr (EVEN) {
            if (chunk != short_chunk) return;
            asm volatile("");                          // keeps it a branch, of the wavefront's: else four selections a chunk
#pragma unroll
            for (int q = 0; q < L::kBlocks; ++q)
                if (q >= first && q < end && bt + q * L::kRowsK >= a.T - chunk * L::BT) at_group[q] = kBehind;
        }
    }
    __device__ __forceinline__ void fetch_x(S& s, uint32_t chunk, int q) const {
        Codes<BITS, EVEN>& c = s.codes[q];
        const uint32_t i = chunk - c0;
        if constexpr (EVEN) {
            c.load(in_codes, at_code[q], i * a.code_chunk);
            c.mn[0] = __builtin_bit_cast(float, buffer_word(in_mn, at_group[q], i * a.group_chunk));
            c.step[0] = __builtin_bit_cast(float, buffer_word(in_step, at_group[q], i * a.group_chunk));
        } else {
            // a word begins with each 32 / BITS elements
            const uint64_t e = element + (uint64_t)i * (L::BT * (uint64_t)a.K) + (uint64_t)q * L::kRowsK * a.K;
            const uint32_t g = divided((uint32_t)(e >> 5), a.by_group), end = (g + 1) * a.group - (uint32_t)e;
            const uint64_t from = (uint64_t)c0 * L::BT * a.K >> 5 << 5;
            const uint32_t bit = (uint32_t)(e - from) * BITS;          // (modulo 2^32: its low bits)
            c.shift = bit & 31u;
            c.turn = end < 8u ? end : 8u;
            c.load(in_codes, (uint32_t)((e - from) / (32 / BITS)) * 4u, 0);
            const uint32_t at = bt + q * L::kRowsK < a.T - chunk * L::BT ? (g - first_group) * 4u : kBehind;
            const w2 m = buffer_words2(in_mn, at, 0), p = buffer_words2(in_step, at, 0);
            const uint32_t m0 = m.x, m1 = m.y, p0 = p.x, p1 = p.y;
            c.mn[0] = __builtin_bit_cast(float, m0);
            c.mn[EVEN ? 0 : 1] = __builtin_bit_cast(float, m1);
            c.step[0] = __builtin_bit_cast(float, p0);
            c.step[EVEN ? 0 : 1] = __builtin_bit_cast(float, p1);
        }
    }
    __device__ __forceinline__ void fetch(S& s, uint32_t chunk) {
        cut(chunk, 0, L::kBlocks);
#pragma unroll
        for (int q = 0; q < L::kPieces; ++q) fetch_dy(s, chunk, q);
#pragma unroll
        for (int q = 0; q < L::kBlocks; ++q) fetch_x(s, chunk, q);
    }
    // A pair of elements as its next part in bf16; what is left of them.
    static __device__ __forceinline__ uint32_t next_part(float& u, float& v) {
        const uint32_t w = bf16_pair_rne(u, v);
        u -= __builtin_bit_cast(float, w << 16);
        v -= __builtin_bit_cast(float, w & 0xFFFF0000u);
        return w;
    }
    __device__ __forceinline__ void place_dy(const S& s, uint8_t* buf, int q) const {
        uint8_t* p = buf + (pt + q * L::kRowsN) * L::kRowN + pn * (2 * L::kPiece);
        if constexpr (DT == GACT_DT_F32) {
            const uint32_t d[4] = {s.dy[q].x, s.dy[q].y, s.dy[q].z, s.dy[q].w};
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = __builtin_bit_cast(float, d[j]);
#pragma unroll
            for (int k = 0; k < L::kParts; ++k) {
                const uint32_t lo = next_part(v[0], v[1]), hi = next_part(v[2], v[3]);
                *(w2*)(p + k * L::kPartN) = w2{lo, hi};
            }
        } else {
            *(w4*)p = s.dy[q];
        }
    }
    __device__ __forceinline__ void place_x(uint8_t* buf, int q, float (&x)[8]) const {
        uint8_t* p = buf + L::kBufN + (bt + q * L::kRowsK) * L::kRowK + bk * 16;
        if constexpr (DT == GACT_DT_F32) {
#pragma unroll
            for (int k = 0; k < L::kParts; ++k) {
                const uint32_t w0 = next_part(x[0], x[1]), w1 = next_part(x[2], x[3]), w2_ = next_part(x[4], x[5]), w3_ = next_part(x[6], x[7]);
                *(w4*)(p + k * L::kPartK) = w4{w0, w1, w2_, w3_};
            }
        } else {
            *(w4*)p = w4{bf16_pair_rne(x[0], x[1]), bf16_pair_rne(x[2], x[3]), bf16_pair_rne(x[4], x[5]), bf16_pair_rne(x[6], x[7])};
        }
    }
    __device__ __forceinline__ void place(S& s, uint8_t* buf) const {
        if (with_dy()) {
#pragma unroll
            for (int q = 0; q < L::kPieces; ++q) place_dy(s, buf, q);
        }
        if (!with_x()) return;
#pragma unroll
        for (int q = 0; q < L::kBlocks; ++q) {
            float x[8];
            s.codes[q].part();
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = s.codes[q].value(j);
            place_x(buf, q, x);
        }
    }
    // adds a chunk's rows of dy to the sums of the thread's columns
    __device__ __forceinline__ void add_db(const S& s, float (&sum)[8]) const {
        if (!with_dy()) return;
#pragma unroll
        for (int q = 0; q < L::kPieces; ++q)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t v = s.dy[q][j];
                if (DT == GACT_DT_F32) sum[j] += __builtin_bit_cast(float, v);
                else {
                    sum[2 * j] += __builtin_bit_cast(float, v << 16);
                    sum[2 * j + 1] += __builtin_bit_cast(float, v & 0xFFFF0000u);
                }
            }
    }
};

// An element of dW over the tokens t .. end - 1 in binary32.  What bfloat16 has no number for, an infinity and elements from
// 2^128 - 2^119 on, leaves an infinity and its rest of the other sign in the parts, and so NaN in the sums: those that are not finite
// are added again, one by one.  Ms, 169343 x 256 x 256 from Python: 0.13 with none, 0.7 with a NaN in dy, which is in a row of dW, 28 with
// nothing else.  (As a function that is called it leaves no kernel its registers: 18 to 179 spilled in the large form.)
template <int BITS>
__device__ __forceinline__ float weight_element(const WeightArgs& a, uint32_t t, uint32_t end, uint32_t n, uint32_t k) {
    float s = 0.0f;
    for (; t < end; ++t) {
        const uint64_t e = (uint64_t)t * a.K + k;
        const uint32_t g = divided((uint32_t)(e >> 5), a.by_group), bit = (uint32_t)(e % 8) * BITS;
        const uint32_t q = a.packed[(e >> 3) * BITS + (bit >> 3)] >> (bit & 7u) & ((1u << BITS) - 1u);
        const float x = (float)q * a.gscale[g];
        s = __builtin_fmaf(((const float*)a.dy)[(int64_t)t * a.dy_stride + n], x + a.gmin[g], s);
    }
    return s;
}

// Where 1024 threads leave 128 registers, some forms spill: long tiles of uneven codes 25 to 36 without a buffer and 6 with one at 8 bits
// (fp32; bf16 1 to 8), tall tiles of fp32 without a buffer 3 to 5; those of whole groups through a buffer none.
template <int DT, int BITS, int FORM, bool BUFFER, bool EVEN>
__global__ __launch_bounds__(weight_tile(DT, FORM).threads, weight_tile(DT, FORM).threads == 1024 ? 4 : 2) void weight_kernel(WeightArgs a) {
    typedef Tiling<DT, FORM> L;
    typedef Products<DT, FORM> Prod;
    typedef typename Prod::Op Op;
    typedef Loader<DT, BITS, FORM, BUFFER, EVEN> Load;
    constexpr int BN = L::BN, BK = L::BK, TN = L::TN, TK = L::TK;
    __shared__ __align__(16) uint8_t lds[L::kBufs][L::kBuf];
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
    const uint32_t all = (a.T + L::BT - 1) / L::BT;
    const uint32_t c0 = split * a.chunks, c1 = c0 + a.chunks < all ? c0 + a.chunks : all;

    const int team = wave >> 2, wn = (wave & 3) / L::kWavesK, wk = (wave & 3) % L::kWavesK;
    Prod prod(lane, team, wn, wk);
    wf16 (&acc)[TN][TK] = prod.acc;
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.0f;

    const bool with_db = a.db != nullptr && (a.db_partial || tile_k == 0);
    // the next chunk that this block adds to db
    uint32_t db_next = with_db && a.db_partial ? c0 + (tile_k + a.db_every - c0 % a.db_every) % a.db_every : with_db ? c0 : ~0u;
    const auto adds = [&](uint32_t chunk) {
        if (chunk != db_next) return false;
        db_next += a.db_every;
        return true;
    };
    const auto fetched = [&](uint32_t chunk) { return weight_fetched(chunk, c1); };
    if (c0 < c1) {
        Load load(a, n0, k0, c0);
        if constexpr (FORM == kWeightLarge && Prod::kSteps == 1) {
            // A chunk is one step: its operands are read at once, and behind the second barrier its place is free for the next one, which is
            // decoded and placed, and the one behind it fetched, between the products.  Without a question, as below.
            typename Load::S slot;
            Op x[TN], y[TK];
            load.fetch(slot, c0);
            if (adds(c0)) load.add_db(slot, sum);
            load.place(slot, lds[0]);
            load.fetch(slot, fetched(c0 + 1));
            for (uint32_t c = c0; c < c1; ++c) {
                __syncthreads();
                load.cut(fetched(c + 2), 0, L::kBlocks);
                prod.read(lds[0], 0, x, y);
                if (c + 1 < c1 && adds(c + 1)) load.add_db(slot, sum);
                __syncthreads();
                float v[L::kBlocks][8];
                constexpr int kValues = 8 * L::kBlocks;
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    prod.product(i, x, y);
#pragma unroll
                    for (int q = i * L::kPieces / TN; q < (i + 1) * L::kPieces / TN; ++q) {
                        load.place_dy(slot, lds[0], q);
                        load.fetch_dy(slot, fetched(c + 2), q);
                    }
#pragma unroll
                    for (int e = i * kValues / TN; e < (i + 1) * kValues / TN; ++e) {
                        if (e % 8 == 0) slot.codes[e / 8].part();
                        v[e / 8][e % 8] = slot.codes[e / 8].value(e % 8);
                        if (e % 8 == 7) {
                            load.place_x(lds[0], e / 8, v[e / 8]);
                            load.fetch_x(slot, fetched(c + 2), e / 8);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        } else if constexpr (FORM == kWeightLarge) {
            // Chunk c is multiplied while chunk c + 1 is placed, the first of its blocks decoded a step ahead, and c + 2 fetched, a little
            // of each behind every row of products, in this order: two wavefronts of a SIMD that do one after the other fall into
            // step and leave the matrix unit idle together.  A step's operands are read during the step before it, so that
            // all of a chunk's have been read by the beginning of its last step; there the one barrier of a chunk stands: behind
            // it chunk c + 1 is whole, and the place of chunk c is free.  Without a question, also behind the split's last
            // chunk, for which the last is fetched again (weight_fetched); nothing uses what is placed then.
            constexpr int kSteps = Prod::kSteps, kSlots = (kSteps - 1) * TN;
            constexpr int kEarly = kSteps == 2 ? L::kBlocks / 2 : 0, kValues = 8 * (L::kBlocks - kEarly);
            typename Load::S slot;
            Op x[2][TN], y[2][TK];
            float v[L::kBlocks][8];
            const auto decode = [&](uint32_t next, int e) {
                const int q = e / 8;
                if (e % 8 == 0) slot.codes[q].part();
                v[q][e % 8] = slot.codes[q].value(e % 8);
                if (e % 8 == 7) load.fetch_x(slot, next, q);
            };
            load.fetch(slot, c0);
            if (adds(c0)) load.add_db(slot, sum);
            load.place(slot, lds[0]);
            load.fetch(slot, fetched(c0 + 1));
            __syncthreads();
            prod.read(lds[0], 0, x[0], y[0]);
            load.cut(fetched(c0 + 2), 0, kEarly);
#pragma unroll
            for (int e = 0; e < 8 * kEarly; ++e) decode(fetched(c0 + 2), e);
            for (uint32_t c = c0; c < c1; ++c) {
                const uint32_t now = (c - c0) & 1u;
                const uint8_t* buf = lds[now];
                uint8_t* other = lds[now ^ 1u];
                if (c + 1 < c1 && adds(c + 1)) load.add_db(slot, sum);
                load.cut(fetched(c + 2), kEarly, L::kBlocks);
                load.cut(fetched(c + 3), 0, kEarly);
#pragma unroll
                for (int s = 0; s + 1 < kSteps; ++s)
#pragma unroll
                    for (int i = 0; i < TN; ++i) {
                        const int at = s * TN + i;
                        prod.product(i, x[s & 1], y[s & 1]);
                        if (i == 0) prod.read_k(buf, s + 1, y[(s + 1) & 1]);
                        prod.read_n(buf, s + 1, i, x[(s + 1) & 1]);
#pragma unroll
                        for (int q = 0; q < kEarly; ++q)
                            if (at == q) load.place_x(other, q, v[q]);
#pragma unroll
                        for (int e = at * kValues / kSlots; e < (at + 1) * kValues / kSlots; ++e) {
                            decode(fetched(c + 2), 8 * kEarly + e);
                            if (e % 8 == 7) load.place_x(other, kEarly + e / 8, v[kEarly + e / 8]);
                        }
#pragma unroll
                        for (int q = 0; q < L::kPieces; ++q)
                            if (at == q * kSlots / L::kPieces) {
                                load.place_dy(slot, other, q);
                                load.fetch_dy(slot, fetched(c + 2), q);
                            }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                __syncthreads();
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    prod.product(i, x[(kSteps - 1) & 1], y[(kSteps - 1) & 1]);
                    if (i == 0) prod.read_k(other, 0, y[0]);
                    prod.read_n(other, 0, i, x[0]);
#pragma unroll
                    for (int e = i * 8 * kEarly / TN; e < (i + 1) * 8 * kEarly / TN; ++e) decode(fetched(c + 3), e);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        } else {
            // Several chunks on their way: a chunk's products take a fraction of the time that its loads do.
            constexpr uint32_t kDepth = weight_depth(FORM, EVEN);
            typename Load::S slot[kDepth];
#pragma unroll
            for (uint32_t u = 0; u < kDepth; ++u)
                if (c0 + u < c1) load.fetch(slot[u], c0 + u);
            for (uint32_t first = c0; first < c1; first += kDepth)
#pragma unroll
                for (uint32_t u = 0; u < kDepth; ++u) {
                    const uint32_t c = first + u;
                    if (c >= c1) break;
                    uint8_t* buf = lds[(c - c0) & 1u];
                    if (adds(c)) load.add_db(slot[u], sum);
                    load.place(slot[u], buf);
                    if (c + kDepth < c1) load.fetch(slot[u], c + kDepth);
                    // the other buffer's readers were done when they came here the time before
                    __syncthreads();
                    prod.chunk(buf);
                }
        }
        __syncthreads();
    }

    // ---- the teams' sums, through shared memory.  Two teams: each hands half of its products to the other, a row of products at a
    // time, and is left with the other half's sums; more: the first adds them all.
    constexpr int kMine = L::kTeams == 2 ? TN / 2 : TN;             // rows of products that a wavefront writes
    const int first = L::kTeams == 2 ? team * kMine : 0;
    float* room = (float*)lds[0] + (tid & 255u);
    constexpr int kRow = TK * 16 * 256;
    if constexpr (L::kTeams == 2) {
        static_assert(TN % 2 == 0 && 2 * kRow * 4 <= L::kBufs * L::kBuf, "room");
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
        static_assert(TN == 1 && (L::kTeams - 1) * kRow * 4 <= L::kBufs * L::kBuf, "room");
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
    const uint32_t lane_n = n0 + (uint32_t)(wn * 32 * TN + first * 32 + 4 * low);
    const uint32_t lane_k = k0 + (uint32_t)(wk * 32 * TK + at_k);
    static_assert(kMine * 16 * TK <= 64, "a bit for each of a lane's elements");
    uint64_t again = 0;                                // those that are not finite (weight_element)
    const auto put = [&](auto* to) {
        typedef typename std::remove_pointer<decltype(to)>::type Out;
        to += (size_t)lane_n * a.K + lane_k;
#pragma unroll
        for (int i = 0; i < kMine; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t n = (uint32_t)(i * 32 + (r & 3) + 8 * (r >> 2));
                if (!inside && lane_n + n >= a.N) continue;
                Out* p = to + (size_t)n * a.K;
#pragma unroll
                for (int j = 0; j < TK; ++j) {
                    const uint32_t k = j * 32;
                    if (!inside && lane_k + k >= a.K) continue;
                    if constexpr (sizeof(Out) == 4) p[k] = acc[i][j][r];
                    else p[k] = (Out)bf16_pair_rne(acc[i][j][r], 0.0f);
                    if (DT == GACT_DT_F32 && !__builtin_isfinite(acc[i][j][r])) again |= 1ull << ((i * 16 + r) * TK + j);
                }
            }
    };
    if (L::kTeams <= 2 || team == 0) {
        if (!whole) put(a.partial + (size_t)split * a.N * a.K);
        else if (a.w_f32) put((float*)a.dw);
        else put((uint16_t*)a.dw);
        if constexpr (DT == GACT_DT_F32) {
            const uint32_t end = c1 * L::BT < a.T ? c1 * L::BT : a.T;
            for (; __builtin_expect(again != 0, 0); again &= again - 1) {
                const uint32_t bit = (uint32_t)__builtin_ctzll(again), j = bit % TK, r = bit / TK % 16u, i = bit / (TK * 16u);
                const uint32_t n = lane_n + i * 32 + (r & 3u) + 8 * (r >> 2), k = lane_k + j * 32;
                const float v = weight_element<BITS>(a, c0 * L::BT, end, n, k);
                const size_t at = (size_t)n * a.K + k;
                if (!whole) a.partial[(size_t)split * a.N * a.K + at] = v;
                else if (a.w_f32) ((float*)a.dw)[at] = v;
                else ((uint16_t*)a.dw)[at] = (uint16_t)bf16_pair_rne(v, 0.0f);
            }
        }
    }

    if (L::kTeams > 1) __syncthreads();
    if (!with_db) return;
    // db of the tile's rows: over the threads of a column, in their order
    float* sums = (float*)lds[0];
#pragma unroll
    for (int j = 0; j < L::kPiece; ++j) sums[(tid / L::kRowPieces) * BN + tid % L::kRowPieces * L::kPiece + j] = sum[j];
    __syncthreads();
    for (uint32_t i = tid; i < (uint32_t)BN; i += L::kThreads) {
        if (n0 + i >= a.N) continue;
        float s = 0.0f;
        for (uint32_t r = 0; r < (uint32_t)L::kRowsN && r < (uint32_t)L::BT; ++r) s += sums[r * BN + i];
        if (a.db_partial) a.db_partial[((size_t)split * a.db_every + tile_k) * a.N + n0 + i] = s;
        else if (a.w_f32) ((float*)a.db)[n0 + i] = s;
        else ((uint16_t*)a.db)[n0 + i] = (uint16_t)bf16_pair_rne(s, 0.0f);
    }
}

// ------------------------------------------------------------- host launchers
template <int DT, int BITS, int FORM>
static void launch_form(const WeightArgs& a, hipStream_t s) {
    const dim3 grid(a.tiles_n * a.tiles_k * a.splits), block(weight_tile(DT, FORM).threads);
    const bool buffer = weight_buffer(a, DT, FORM), even = weight_even(a, DT, FORM);
    if (buffer && even) hipLaunchKernelGGL((weight_kernel<DT, BITS, FORM, true, true>), grid, block, 0, s, a);
    else if (buffer) hipLaunchKernelGGL((weight_kernel<DT, BITS, FORM, true, false>), grid, block, 0, s, a);
    else if (even) hipLaunchKernelGGL((weight_kernel<DT, BITS, FORM, false, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((weight_kernel<DT, BITS, FORM, false, false>), grid, block, 0, s, a);
}
template <int DT, int BITS>
static void launch_bits(const WeightArgs& a, int form, hipStream_t s) {
    switch (form) {
        case kWeightLarge: launch_form<DT, BITS, kWeightLarge>(a, s); break;
        case kWeightSmall: launch_form<DT, BITS, kWeightSmall>(a, s); break;
        case kWeightLong: launch_form<DT, BITS, kWeightLong>(a, s); break;
        case kWeightWide: launch_form<DT, BITS, kWeightWide>(a, s); break;
        default: launch_form<DT, BITS, kWeightTall>(a, s); break;
    }
}
template <int DT>
static int launch_type(const WeightArgs& a, int form, int bits, hipStream_t s) {
    switch (bits) {
        case 1: launch_bits<DT, 1>(a, form, s); break;
        case 2: launch_bits<DT, 2>(a, form, s); break;
        case 4: launch_bits<DT, 4>(a, form, s); break;
        default: launch_bits<DT, 8>(a, form, s); break;
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace gact

#endif
