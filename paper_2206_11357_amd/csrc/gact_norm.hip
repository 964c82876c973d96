// Global norm of a list of gradient buffers, and clipping by it, for MI355X (gfx950).
//
//   norm = sqrt(sum g^2) or max |g| over all buffers,   out = g min(1, max_norm / (norm + 1e-6))
//
// Bound by HBM: the norm reads every element once, clipping reads and writes it once more, unless nothing has to be
// scaled in place.  The norm's launch is at most 1536 blocks (scaling has up to 8192), each with a run of neighbouring 16 KB
// chunks, so that it leaves at most 1536 results whatever the list's size.  That is few enough for every block of the scaling launch to add them
// up itself, in the same order: clipping is two launches, with no third one between them, no counter that would have
// to start at zero and no block that waits for another, and can be captured into a graph as it is.  (A norm alone has a
// second launch of one block.)  The squares are added in binary64: a sum of 10^9 of them in binary32 would lose what clipping
// compares.
//
// Us and TB/s: norm of 101 M bf16 elements 31.4 (6.4), of 304 M at odd addresses 92 (6.6), of 302 M fp32 178 (6.8);
// scaling 302 M fp32 behind it 430 (5.6), 101 M bf16 by a given norm 59 (6.8).  A large read reaches 7.0; a copy what the cache lets
// it, 6.8 for 200 MB, 5.7 for 400 MB, 5.3 for 1.2 GB, 5.0 for 4 GB, all fp32.  Lists of less than some MB: 3.3 + 4.1, what two
// launches take.
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

// A 16-byte piece.  ONCE: it is not wanted in a cache (kNormOnceBytes, clip_run).
template <int DT, bool ONCE>
__device__ __forceinline__ n4 load_piece(const uint8_t* p) {
    if (DT == GACT_DT_F32) return ONCE ? __builtin_nontemporal_load((const n4_f32*)p) : *(const n4_f32*)p;
    return ONCE ? __builtin_nontemporal_load((const n4_bf16*)p) : *(const n4_bf16*)p;
}
template <int DT>
__device__ __forceinline__ void store_piece(uint8_t* p, n4 w) {
    if (DT == GACT_DT_F32) __builtin_nontemporal_store(w, (n4_f32*)p);
    else __builtin_nontemporal_store(w, (n4_bf16*)p);
}
template <int DT>
constexpr int kSize = DT == GACT_DT_F32 ? 4 : 2;
template <int DT>
__device__ __forceinline__ float load_element(const uint8_t* p) {
    if (DT == GACT_DT_F32) return *(const float*)p;
    return __builtin_bit_cast(float, (uint32_t)*(const uint16_t*)p << 16);
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

constexpr int kChunkBytes = kNormThreads * kNormPieces * 16;
constexpr int kTogether = 2;                        // chunks whose loads are out together

// A run of neighbouring chunks [begin, end), buffer by buffer, forwards or (BACK) from the end: part(buffer, number of its first
// chunk, number of chunks) for each.  Chunks are whole but for a buffer's last.
template <bool BACK, typename PART>
__device__ __forceinline__ void each_part(const NormBuffer* table, const uint32_t* first, uint32_t K, uint32_t begin, uint32_t end,
                                          const PART& part) {
    uint32_t lo = 0, hi = K;
    const uint32_t at = BACK ? end - 1 : begin;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (first[mid] <= at) lo = mid; else hi = mid;
    }
    if (!BACK) {
        for (uint32_t k = lo; begin < end; ++k) {
            const uint32_t stop = first[k + 1] < end ? first[k + 1] : end;
            part(k, begin - first[k], stop - begin);
            begin = stop;
        }
    } else {
        for (uint32_t k = lo; begin < end; --k) {
            const uint32_t start = first[k] > begin ? first[k] : begin;
            part(k, start - first[k], end - start);
            end = start;
        }
    }
}

template <int KIND, bool ONCE, int DT>
__device__ __forceinline__ void norm_part(const NormBuffer& b, uint32_t chunk, uint32_t chunks, Acc<KIND>& acc) {
    constexpr int P = 16 / kSize<DT>;
    if (chunk == 0 && threadIdx.x < (uint32_t)b.head)
        acc.add(load_element<DT>((const uint8_t*)b.in - (threadIdx.x + 1) * kSize<DT>));
    const uint8_t* p = (const uint8_t*)b.in + (int64_t)chunk * kChunkBytes;
    const uint32_t mine = threadIdx.x * 16;
    const int64_t left = b.n - (int64_t)chunk * norm_chunk_elems(DT);
    const uint32_t whole = left >= (int64_t)chunks * norm_chunk_elems(DT) ? chunks : chunks - 1;
    uint32_t i = 0;
    for (; i + kTogether <= whole; i += kTogether, p += kTogether * kChunkBytes) {
        n4 w[kTogether * kNormPieces];
#pragma unroll
        for (int k = 0; k < kTogether * kNormPieces; ++k) w[k] = load_piece<DT, ONCE>((p + k * kNormThreads * 16) + mine);
#pragma unroll
        for (int k = 0; k < kTogether * kNormPieces; ++k) {
            float v[8];
            widen<DT>(w[k], v);
#pragma unroll
            for (int j = 0; j < P; ++j) acc.add(v[j]);
        }
    }
    for (; i < whole; ++i, p += kChunkBytes) {
        n4 w[kNormPieces];
#pragma unroll
        for (int k = 0; k < kNormPieces; ++k) w[k] = load_piece<DT, ONCE>((p + k * kNormThreads * 16) + mine);
#pragma unroll
        for (int k = 0; k < kNormPieces; ++k) {
            float v[8];
            widen<DT>(w[k], v);
#pragma unroll
            for (int j = 0; j < P; ++j) acc.add(v[j]);
        }
    }
    if (whole == chunks) return;
    // the buffer's last chunk: pieces up to the one that its end cuts, whose elements go to a lane each
    const uint32_t rest = (uint32_t)(left - (int64_t)whole * norm_chunk_elems(DT)), in_pieces = rest & ~(uint32_t)(P - 1);
#pragma unroll
    for (int k = 0; k < kNormPieces; ++k) {
        const uint32_t e = (k * kNormThreads + threadIdx.x) * P;
        if (e >= in_pieces) continue;
        float v[8];
        widen<DT>(load_piece<DT, ONCE>(p + e * kSize<DT>), v);
#pragma unroll
        for (int j = 0; j < P; ++j) acc.add(v[j]);
    }
    if (threadIdx.x < rest - in_pieces) acc.add(load_element<DT>(p + (in_pieces + threadIdx.x) * kSize<DT>));
}

template <int KIND, bool ONCE>
__device__ __forceinline__ void norm_run(const NormBuffer* table, const uint32_t* first, const NormArgs& a) {
    const uint32_t begin = (uint32_t)((uint64_t)a.chunks * blockIdx.x / a.blocks);
    const uint32_t end = (uint32_t)((uint64_t)a.chunks * (blockIdx.x + 1) / a.blocks);
    Acc<KIND> acc;
    each_part<false>(table, first, a.K, begin, end, [&](uint32_t k, uint32_t chunk, uint32_t chunks) {
        const NormBuffer b = table[k];
        if (k < a.f32) norm_part<KIND, ONCE, GACT_DT_F32>(b, chunk, chunks, acc);
        else norm_part<KIND, ONCE, GACT_DT_BF16>(b, chunk, chunks, acc);
    });
    const double v = join_block<KIND>(acc.value());
    if (threadIdx.x == 0) a.partial[blockIdx.x] = v;
}
template <int KIND, bool ONCE>
__global__ __launch_bounds__(kNormThreads) void grad_norm_kernel(NormArgs a) {
    norm_run<KIND, ONCE>(a.table, a.first, a);
}
template <int KIND, bool ONCE>
__global__ __launch_bounds__(kNormThreads) void grad_norm_inline_kernel(NormArgs a, NormTable t) {
    norm_run<KIND, ONCE>(t.t, t.first, a);
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

// c times a piece, in binary64, so that a binary32 result is rounded once.  (A bf16 result goes by way of binary32, which
// moves the half of a step by 2^-24 of the value.)
template <int DT>
__device__ __forceinline__ n4 scaled(const n4 w, double c) {
    constexpr int P = 16 / kSize<DT>;
    float v[8];
    widen<DT>(w, v);
#pragma unroll
    for (int j = 0; j < P; ++j) v[j] = (float)((double)v[j] * c);
    if (DT == GACT_DT_F32)
        return n4{__builtin_bit_cast(uint32_t, v[0]), __builtin_bit_cast(uint32_t, v[1]), __builtin_bit_cast(uint32_t, v[2]),
                  __builtin_bit_cast(uint32_t, v[3])};
    return n4{bf16_pair_rne(v[0], v[1]), bf16_pair_rne(v[2], v[3]), bf16_pair_rne(v[4], v[5]), bf16_pair_rne(v[6], v[7])};
}

template <int DT>
__device__ __forceinline__ void clip_element(const uint8_t* in, uint8_t* out, double c) {
    const float v = (float)((double)load_element<DT>(in) * c);
    if (DT == GACT_DT_F32) *(float*)out = v;
    else *(uint16_t*)out = (uint16_t)bf16_pair_rne(v, 0.0f);
}

template <int DT, bool ONCE, int CHUNKS>
__device__ __forceinline__ void clip_chunks(const uint8_t* in, uint8_t* out, uint32_t mine, double c) {
    n4 w[CHUNKS * kNormPieces];
#pragma unroll
    for (int k = 0; k < CHUNKS * kNormPieces; ++k) w[k] = load_piece<DT, ONCE>((in + k * kNormThreads * 16) + mine);
#pragma unroll
    for (int k = 0; k < CHUNKS * kNormPieces; ++k) store_piece<DT>((out + k * kNormThreads * 16) + mine, scaled<DT>(w[k], c));
}

template <int DT, bool ONCE>
__device__ __forceinline__ void clip_part(const NormBuffer& b, uint32_t chunk, uint32_t chunks, double c) {
    constexpr int P = 16 / kSize<DT>;
    if (chunk == 0 && threadIdx.x < (uint32_t)b.head) {
        const uint32_t back = (threadIdx.x + 1) * kSize<DT>;
        clip_element<DT>((const uint8_t*)b.in - back, (uint8_t*)b.out - back, c);
    }
    const uint8_t* in = (const uint8_t*)b.in + (int64_t)chunk * kChunkBytes;
    uint8_t* out = (uint8_t*)b.out + (int64_t)chunk * kChunkBytes;
    const uint32_t mine = threadIdx.x * 16;
    const int64_t left = b.n - (int64_t)chunk * norm_chunk_elems(DT);
    const uint32_t whole = left >= (int64_t)chunks * norm_chunk_elems(DT) ? chunks : chunks - 1;
    if (whole != chunks) {                           // as in norm_part
        const int64_t o = (int64_t)whole * kChunkBytes;
        const uint32_t rest = (uint32_t)(left - (int64_t)whole * norm_chunk_elems(DT)), in_pieces = rest & ~(uint32_t)(P - 1);
#pragma unroll
        for (int k = 0; k < kNormPieces; ++k) {
            const uint32_t e = (k * kNormThreads + threadIdx.x) * P;
            if (e < in_pieces) store_piece<DT>(out + o + e * kSize<DT>, scaled<DT>(load_piece<DT, ONCE>(in + o + e * kSize<DT>), c));
        }
        if (threadIdx.x < rest - in_pieces) {
            const int64_t at = o + (in_pieces + threadIdx.x) * kSize<DT>;
            clip_element<DT>(in + at, out + at, c);
        }
    }
    uint32_t i = whole;
    for (; i >= kTogether; i -= kTogether)
        clip_chunks<DT, ONCE, kTogether>(in + (int64_t)(i - kTogether) * kChunkBytes, out + (int64_t)(i - kTogether) * kChunkBytes, mine, c);
    for (; i > 0; --i) clip_chunks<DT, ONCE, 1>(in + (int64_t)(i - 1) * kChunkBytes, out + (int64_t)(i - 1) * kChunkBytes, mine, c);
}

// GIVEN: the norm is there; else it comes from the blocks' results, and block 0 leaves it.
// What comes out is not wanted in a cache, where it would push out what is still to be read: 100 M bf16 elements by a
// given norm 84 us with ordinary stores, 62; 100 M fp32 behind their norm 139, 124.  Nor is what is read a second time (fp32,
// 100 M: 152 us with ordinary loads, 124), but by a given norm it may well be there from what has made it (78, 62).
template <int KIND, bool GIVEN>
__device__ __forceinline__ void clip_run(const NormBuffer* table, const uint32_t* first, const NormArgs& a) {
    double norm;
    if (GIVEN) norm = *a.norm;
    else {
        norm = join_results<KIND>(a);
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
    }
    double c = a.max_norm / (norm + 1e-6);
    c = c > 1.0 ? 1.0 : c;                           // a NaN stays
    const uint32_t begin = (uint32_t)((uint64_t)a.chunks * blockIdx.x / a.clip_blocks);
    const uint32_t end = (uint32_t)((uint64_t)a.chunks * (blockIdx.x + 1) / a.clip_blocks);
    // Backwards: what the norm's launch has read last may still be in a cache.
    each_part<true>(table, first, a.K, begin, end, [&](uint32_t k, uint32_t chunk, uint32_t chunks) {
        const NormBuffer b = table[k];
        if (c == 1.0 && b.in == b.out) return;
        if (k < a.f32) clip_part<GACT_DT_F32, !GIVEN>(b, chunk, chunks, c);
        else clip_part<GACT_DT_BF16, !GIVEN>(b, chunk, chunks, c);
    });
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
template <int KIND, bool ONCE>
static void launch_norm(const NormTable* t, const NormArgs& a, hipStream_t s) {
    if (t) hipLaunchKernelGGL((grad_norm_inline_kernel<KIND, ONCE>), dim3(a.blocks), dim3(kNormThreads), 0, s, a, *t);
    else hipLaunchKernelGGL((grad_norm_kernel<KIND, ONCE>), dim3(a.blocks), dim3(kNormThreads), 0, s, a);
}
template <int KIND, bool GIVEN>
static void launch_clip(const NormTable* t, const NormArgs& a, hipStream_t s) {
    if (t) hipLaunchKernelGGL((grad_clip_inline_kernel<KIND, GIVEN>), dim3(a.clip_blocks), dim3(kNormThreads), 0, s, a, *t);
    else hipLaunchKernelGGL((grad_clip_kernel<KIND, GIVEN>), dim3(a.clip_blocks), dim3(kNormThreads), 0, s, a);
}
}  // namespace gact

// `t` where the table travels in the arguments, else null.  finish: a launch behind it adds the results up and
// leaves the norm.
extern "C" int gact_launch_grad_norm(const gact::NormTable* t, const gact::NormArgs* a, int kind, int once, int finish, void* stream) {
    using namespace gact;
    hipStream_t s = (hipStream_t)stream;
    if (a->blocks != 0) {
        if (kind == kNorm2 && once) launch_norm<kNorm2, true>(t, *a, s);
        else if (kind == kNorm2) launch_norm<kNorm2, false>(t, *a, s);
        else if (once) launch_norm<kNormInf, true>(t, *a, s);
        else launch_norm<kNormInf, false>(t, *a, s);
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
