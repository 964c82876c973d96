// Global norm of a list of gradient buffers, and clipping by it, for MI355X (gfx950).
//
//   norm = sqrt(sum g^2) or max |g| over all buffers,   out = g min(1, max_norm / (norm + 1e-6))
//
// Bound by HBM: the norm reads every element once, clipping reads and writes it once more, unless nothing has to be
// scaled in place.  A launch is at most 1024 blocks, each with a run of neighbouring 16 KB chunks, so that a call
// leaves at most 1024 results whatever its size.  That is few enough for every block of the scaling launch to add them
// up itself, in the same order: clipping is two launches, with no third one between them, no counter that would have
// to start at zero and no block that waits for another, and can be captured into a graph as it is.  The squares are added in
// binary64: a sum of 10^9 of them in binary32 would lose what clipping compares.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gact_codec.h"
#include "gact_device.h"
#include "gact_norm.h"
#include "gact_sum.h"

namespace gact {

typedef uint32_t n4 __attribute__((ext_vector_type(4)));
typedef n4 n4_f32 __attribute__((aligned(4)));       // at any address that an element can have
typedef n4 n4_bf16 __attribute__((aligned(2)));

enum { kNorm2 = 0, kNormInf = 1 };

// A block's result: sum of squares, or the largest magnitude as its bits, whose order is that of the
// magnitudes, with infinity behind the numbers and NaN behind it (so that a NaN stays).
template <int KIND>
struct Acc {
    double   sum = 0.0;
    uint32_t top = 0;
    __device__ __forceinline__ void add(float v) {
        if (KIND == kNorm2) sum += (double)v * (double)v;
        else {
            const uint32_t m = __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu;
            top = m > top ? m : top;
        }
    }
    __device__ __forceinline__ double value() const { return KIND == kNorm2 ? sum : (double)__builtin_bit_cast(float, top); }
};
// Of two such results; NaN stays.
template <int KIND>
__device__ __forceinline__ double joined(double a, double b) {
    if (KIND == kNorm2) return a + b;
    return a != a || a > b ? a : b;
}
template <int KIND>
__device__ __forceinline__ double join_lanes(double v) {
    if (KIND == kNorm2) return add_lanes(v);
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v = joined<KIND>(v, __shfl_xor(v, m));
    return v;
}
// Over the block, in thread order of wavefronts; valid in every thread.
template <int KIND>
__device__ __forceinline__ double join_block(double v) {
    __shared__ double part[kNormWaves];
    v = join_lanes<KIND>(v);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < kNormWaves; ++w) v = joined<KIND>(v, part[w]);
    return v;
}
template <int KIND>
__device__ __forceinline__ double root(double v) { return KIND == kNorm2 ? __builtin_sqrt(v) : v; }

// The chunks of a block's run, buffer by buffer.
struct Walk {
    const NormBuffer* table;
    const uint32_t* first;
    uint32_t k, begin, end;                          // buffer; chunks of the run that are left
    __device__ __forceinline__ Walk(const NormBuffer* buffers, const uint32_t* firsts, const NormArgs& a, bool from_end)
        : table(buffers), first(firsts) {
        begin = (uint32_t)((uint64_t)a.chunks * blockIdx.x / a.blocks);
        end = (uint32_t)((uint64_t)a.chunks * (blockIdx.x + 1) / a.blocks);
        const uint32_t at = from_end ? end - 1 : begin;
        uint32_t lo = 0, hi = a.K;
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) >> 1;
            if (first[mid] <= at) lo = mid; else hi = mid;
        }
        k = lo;
    }
};

template <int DT, bool FULL>
__device__ __forceinline__ n4 load_piece(const void* in, int64_t e, int64_t n) {
    constexpr int P = DT == GACT_DT_F32 ? 4 : 8;
    n4 w = {0u, 0u, 0u, 0u};
    if (FULL || e + P <= n) {
        if (DT == GACT_DT_F32) w = *(const n4_f32*)((const uint32_t*)in + e);
        else w = *(const n4_bf16*)((const uint16_t*)in + e);
    } else if (e < n) {
        uint32_t t[4] = {0u, 0u, 0u, 0u};
        for (int j = 0; j < P; ++j)
            if (e + j < n) {
                if (DT == GACT_DT_F32) t[j & 3] = ((const uint32_t*)in)[e + j];
                else t[j >> 1] |= (uint32_t)((const uint16_t*)in)[e + j] << (16 * (j & 1));
            }
        w = n4{t[0], t[1], t[2], t[3]};
    }
    return w;
}
template <int DT>
__device__ __forceinline__ void widen(const n4 w, float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t c = w[k];
        if (DT == GACT_DT_F32) v[k] = __builtin_bit_cast(float, c);
        else { v[2 * k] = __builtin_bit_cast(float, c << 16); v[2 * k + 1] = __builtin_bit_cast(float, c & 0xFFFF0000u); }
    }
}

template <int KIND, int DT, bool FULL>
__device__ __forceinline__ void norm_chunk(const NormBuffer& b, int64_t chunk, Acc<KIND>& acc) {
    constexpr int P = DT == GACT_DT_F32 ? 4 : 8;
    n4 w[kNormPieces];
#pragma unroll
    for (int i = 0; i < kNormPieces; ++i)
        w[i] = load_piece<DT, FULL>(b.in, chunk * norm_chunk_elems(DT) + (i * kNormThreads + (int)threadIdx.x) * P, b.n);
#pragma unroll
    for (int i = 0; i < kNormPieces; ++i) {
        float v[8];
        widen<DT>(w[i], v);
#pragma unroll
        for (int j = 0; j < P; ++j) acc.add(v[j]);
    }
}

template <int KIND>
__device__ __forceinline__ void norm_run(Walk walk, const NormArgs& a) {
    Acc<KIND> acc;
    for (uint32_t c = walk.begin; c < walk.end; ++c) {
        while (walk.first[walk.k + 1] <= c) ++walk.k;
        const NormBuffer b = walk.table[walk.k];
        const int64_t chunk = c - walk.first[walk.k];
        if (walk.k < a.f32) {
            if ((chunk + 1) * norm_chunk_elems(GACT_DT_F32) <= b.n) norm_chunk<KIND, GACT_DT_F32, true>(b, chunk, acc);
            else norm_chunk<KIND, GACT_DT_F32, false>(b, chunk, acc);
        } else {
            if ((chunk + 1) * norm_chunk_elems(GACT_DT_BF16) <= b.n) norm_chunk<KIND, GACT_DT_BF16, true>(b, chunk, acc);
            else norm_chunk<KIND, GACT_DT_BF16, false>(b, chunk, acc);
        }
    }
    const double v = join_block<KIND>(acc.value());
    if (threadIdx.x == 0) a.partial[blockIdx.x] = v;
}
template <int KIND>
__global__ __launch_bounds__(kNormThreads) void grad_norm_kernel(NormArgs a) {
    norm_run<KIND>(Walk(a.table, a.first, a, false), a);
}
template <int KIND>
__global__ __launch_bounds__(kNormThreads) void grad_norm_inline_kernel(NormArgs a, NormTable t) {
    norm_run<KIND>(Walk(t.t, t.first, a, false), a);
}

// The results of all blocks, in every thread.
template <int KIND>
__device__ __forceinline__ double join_results(const NormArgs& a) {
    double v = 0.0;                                  // of neither kind does it change a result
#pragma unroll
    for (uint32_t i = 0; i < kNormBlocks; i += kNormThreads)
        if (i + threadIdx.x < a.blocks) v = joined<KIND>(v, a.partial[i + threadIdx.x]);
    return root<KIND>(join_block<KIND>(v));
}

template <int KIND>
__global__ __launch_bounds__(kNormThreads) void norm_finish_kernel(NormArgs a) {
    const double norm = join_results<KIND>(a);
    if (threadIdx.x == 0) *a.norm = norm;
}

template <int DT, bool FULL>
__device__ __forceinline__ void clip_chunk(const NormBuffer& b, int64_t chunk, double c) {
    constexpr int P = DT == GACT_DT_F32 ? 4 : 8;
    n4 w[kNormPieces];
    const int64_t e0 = chunk * norm_chunk_elems(DT) + (int)threadIdx.x * P;
#pragma unroll
    for (int i = 0; i < kNormPieces; ++i) w[i] = load_piece<DT, FULL>(b.in, e0 + i * kNormThreads * P, b.n);
#pragma unroll
    for (int i = 0; i < kNormPieces; ++i) {
        const int64_t e = e0 + i * kNormThreads * P;
        float v[8];
        widen<DT>(w[i], v);
        // in binary64, so that a binary32 result is rounded once
#pragma unroll
        for (int j = 0; j < P; ++j) v[j] = (float)((double)v[j] * c);
        n4 o;
        if (DT == GACT_DT_F32)
            o = n4{__builtin_bit_cast(uint32_t, v[0]), __builtin_bit_cast(uint32_t, v[1]), __builtin_bit_cast(uint32_t, v[2]),
                   __builtin_bit_cast(uint32_t, v[3])};
        else
            o = n4{bf16_pair_rne(v[0], v[1]), bf16_pair_rne(v[2], v[3]), bf16_pair_rne(v[4], v[5]), bf16_pair_rne(v[6], v[7])};
        if (FULL || e + P <= b.n) {
            if (DT == GACT_DT_F32) *(n4_f32*)((uint32_t*)b.out + e) = o;
            else *(n4_bf16*)((uint16_t*)b.out + e) = o;
        } else if (e < b.n) {
            for (int j = 0; j < P; ++j)
                if (e + j < b.n) {
                    if (DT == GACT_DT_F32) ((uint32_t*)b.out)[e + j] = o[j & 3];
                    else ((uint16_t*)b.out)[e + j] = (uint16_t)(o[j >> 1] >> (16 * (j & 1)));
                }
        }
    }
}

// GIVEN: the norm is there; else it comes from the blocks' results, and block 0 leaves it.
template <int KIND, bool GIVEN>
__device__ __forceinline__ void clip_run(const NormBuffer* buffers, const uint32_t* firsts, const NormArgs& a) {
    double norm;
    if (GIVEN) norm = *a.norm;
    else {
        norm = join_results<KIND>(a);
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
    }
    double c = a.max_norm / (norm + 1e-6);
    c = c > 1.0 ? 1.0 : c;                           // a NaN stays
    // Backwards: what the norm's launch has read last may still be in a cache.
    Walk walk(buffers, firsts, a, true);
    for (uint32_t i = walk.end; i > walk.begin; --i) {
        while (walk.first[walk.k] > i - 1) --walk.k;
        const NormBuffer b = walk.table[walk.k];
        if (c == 1.0 && b.in == b.out) continue;
        const int64_t chunk = i - 1 - walk.first[walk.k];
        if (walk.k < a.f32) {
            if ((chunk + 1) * norm_chunk_elems(GACT_DT_F32) <= b.n) clip_chunk<GACT_DT_F32, true>(b, chunk, c);
            else clip_chunk<GACT_DT_F32, false>(b, chunk, c);
        } else {
            if ((chunk + 1) * norm_chunk_elems(GACT_DT_BF16) <= b.n) clip_chunk<GACT_DT_BF16, true>(b, chunk, c);
            else clip_chunk<GACT_DT_BF16, false>(b, chunk, c);
        }
    }
}

template <int KIND, bool GIVEN>
__global__ __launch_bounds__(kNormThreads) void grad_clip_kernel(NormArgs a) {
    clip_run<KIND, GIVEN>(a.table, a.first, a);
}
template <int KIND, bool GIVEN>
__global__ __launch_bounds__(kNormThreads) void grad_clip_inline_kernel(NormArgs a, NormTable t) {
    clip_run<KIND, GIVEN>(t.t, t.first, a);
}

// Part of a table, from the arguments to the workspace: a graph that holds it can be replayed.
__global__ void table_piece_kernel(uint32_t* __restrict__ dst, TablePiece piece, unsigned words) {
    for (unsigned i = threadIdx.x; i < words; i += blockDim.x) dst[i] = piece.w[i];
}

}  // namespace gact

namespace gact {
template <int KIND>
static void launch_norm(const NormTable* t, const NormArgs& a, hipStream_t s) {
    if (t) hipLaunchKernelGGL(grad_norm_inline_kernel<KIND>, dim3(a.blocks), dim3(kNormThreads), 0, s, a, *t);
    else hipLaunchKernelGGL(grad_norm_kernel<KIND>, dim3(a.blocks), dim3(kNormThreads), 0, s, a);
}
template <int KIND, bool GIVEN>
static void launch_clip(const NormTable* t, const NormArgs& a, hipStream_t s) {
    if (t) hipLaunchKernelGGL((grad_clip_inline_kernel<KIND, GIVEN>), dim3(a.blocks), dim3(kNormThreads), 0, s, a, *t);
    else hipLaunchKernelGGL((grad_clip_kernel<KIND, GIVEN>), dim3(a.blocks), dim3(kNormThreads), 0, s, a);
}
}  // namespace gact

// `t` where the table travels in the arguments, else null.  finish: a launch behind it adds the results up and
// leaves the norm.
extern "C" int gact_launch_grad_norm(const gact::NormTable* t, const gact::NormArgs* a, int kind, int finish, void* stream) {
    using namespace gact;
    hipStream_t s = (hipStream_t)stream;
    if (a->blocks != 0) {
        if (kind == kNorm2) launch_norm<kNorm2>(t, *a, s);
        else launch_norm<kNormInf>(t, *a, s);
        if (hipGetLastError() != hipSuccess) return -1;
    }
    if (!finish) return 0;
    if (kind == kNorm2) hipLaunchKernelGGL(norm_finish_kernel<kNorm2>, dim3(1), dim3(kNormThreads), 0, s, *a);
    else hipLaunchKernelGGL(norm_finish_kernel<kNormInf>, dim3(1), dim3(kNormThreads), 0, s, *a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

extern "C" int gact_launch_grad_clip(const gact::NormTable* t, const gact::NormArgs* a, int kind, int given, void* stream) {
    using namespace gact;
    hipStream_t s = (hipStream_t)stream;
    if (given) launch_clip<kNorm2, true>(t, *a, s);
    else if (kind == kNorm2) launch_clip<kNorm2, false>(t, *a, s);
    else launch_clip<kNormInf, false>(t, *a, s);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

extern "C" int gact_launch_table_piece(void* dst, const gact::TablePiece* piece, unsigned words, void* stream) {
    hipLaunchKernelGGL(gact::table_piece_kernel, dim3(1), dim3(256), 0, (hipStream_t)stream, (uint32_t*)dst, *piece, words);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}
