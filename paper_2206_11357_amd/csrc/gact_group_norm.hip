// Group normalisation with an activation over channels-last maps, its compressed context and its gradients, for MI355X (gfx950).
//
//   over a group's M = P D elements of a sample:  m = mean x,  r = 1 / sqrt(mean (x - m)^2 + eps)
//   n = (x - m) r,  z = n w + b,  y = act(z)
//   dz = dy act'(z),  g = dz w,  dx = r (g - mean g - n mean(g n)),  dw = sum dz n,  db = sum dz
//
// Eight consecutive channels a lane: one block of the compressor's noise generator and `bits` whole bytes of its string, so that
// the pass that writes y leaves the compressed context of x from the registers that hold x, and the backward passes take x
// from the codes.  m and r are kept from the forward pass in binary32.
// Forward: statistics (x read once), then y and the context (x read again, from the cache where it holds it).  A thread of the
// first pass takes several pixels at a time: their mean, their squared distances from it, and both are merged with what it has
// (T. Chan, G. Golub, R. LeVeque 1979), so that nothing cancels.  Backward: sums of dz and dz n over the pixels for each
// channel and sample, from which the groups' means and dw, db follow; then dx.
// Where a sample's group fits a workgroup's registers, both are one pass over memory (and dw, db a second launch where there
// are several samples).  Measured, us: 64 x 3136 x 256 fp32, 2 bits, held 137 forward, 110 backward (HBM: 631 and 448 MB as
// counted, x a second time for its codes); 32 x 1024 x 512 bf16, SiLU, 4 bits, held 25.2 (calls in a row: norm without a context
// 16.3, compressor alone 9.4, both 25.9) and 21.0; 1 x 262144 x 128 bf16, SiLU, in passes 13.2 + 4.4 + 26.2 (reads at 5.1 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gact_block8.h"
#include "gact_codec.h"
#include "gact_device.h"
#include "gact_group_norm.h"

namespace gact {

typedef float hf2 __attribute__((ext_vector_type(2)));

// ----------------------------------------------------------------- activation
// exp(-z).  The exponent's rounding, z times 2^-24 of the result, is taken back: fp32 results keep their last bits.
template <int DT>
__device__ __forceinline__ float exp_neg(float z) {
    constexpr float kLog2e = 0x1.715476p+0f, kLog2eLow = 0x1.4ae0cp-26f;        // their sum: log2 e
    const float e = __builtin_amdgcn_exp2f(-z * kLog2e);
    if (DT == GACT_DT_BF16) return e;
    const float c = __builtin_amdgcn_fmed3f(z, -150.0f, 150.0f);
    const float low = __builtin_fmaf(-c, kLog2eLow, __builtin_fmaf(-c, kLog2e, c * kLog2e));
    return e * __builtin_fmaf(low, 0x1.62e43p-1f, 1.0f);
}
template <int DT>
__device__ __forceinline__ float inverse(float v) {
    return DT == GACT_DT_BF16 ? __builtin_amdgcn_rcpf(v) : 1.0f / v;
}
template <int DT, bool SILU>
__device__ __forceinline__ float activate(float z) {
    return SILU ? z * inverse<DT>(1.0f + exp_neg<DT>(z)) : z;
}
// act'(z)
template <int DT>
__device__ __forceinline__ float silu_slope(float z) {
    const float p = inverse<DT>(1.0f + exp_neg<DT>(z));
    return p * __builtin_fmaf(z, 1.0f - p, 1.0f);
}

// ------------------------------------------------------------------- channels
// What belongs to a lane's eight channels: weights; and of their groups, which are one where D is a multiple of eight.
__device__ __forceinline__ void load_channels(const void* p, int f32, float without, uint32_t c, float (&v)[8]) {
    if (!p) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = without;
    } else if (f32) widen8<GACT_DT_F32>(load8<GACT_DT_F32>((const uint8_t*)p, c * 4u), v);
    else widen8<GACT_DT_BF16>(load8<GACT_DT_BF16>((const uint8_t*)p, c * 2u), v);
}
template <bool UNI>
struct OfGroups {
    static constexpr int N = UNI ? 1 : 8;
    float v[N];
    // of the groups of channels c .. c + 7 of a sample, whose values `p` holds, `step` floats apart
    __device__ __forceinline__ void load(const GnArgs& a, const float* p, int step, uint32_t c) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = p[(size_t)divided(c + (uint32_t)k, a.by_d) * step];
    }
    // the same of sums in a.slices parts, which follow each other, two floats apart
    __device__ __forceinline__ void add(const GnArgs& a, const float* p, uint32_t c) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float* q = p + (size_t)divided(c + (uint32_t)k, a.by_d) * a.slices * 2;
            v[k] = q[0];
            for (uint32_t s = 1; s < a.slices; ++s) v[k] += q[2 * s];
        }
    }
    __device__ __forceinline__ float operator[](int k) const { return v[UNI ? 0 : k]; }
};
// A workgroup's place in a pass over pixels.
struct Column {
    uint32_t sample, chunk, c8, row;
    bool     holds;
    __device__ __forceinline__ Column(const GnArgs& a, uint32_t block) {
        const uint32_t slab = block % a.slabs;
        block /= a.slabs;
        sample = block / a.chunks;
        chunk = block - sample * a.chunks;
        row = divided(threadIdx.x, a.by_cols);
        const uint32_t col = threadIdx.x - row * a.cols;
        c8 = slab * a.cols + col;
        holds = row < a.rows && c8 < a.C8;
    }
    __device__ __forceinline__ size_t partial(const GnArgs& a) const { return ((size_t)sample * a.chunks + chunk) * a.C8 + c8; }
};

// ------------------------------------------------------------------ statistics
// Number, mean and squared distances from it of a thread's elements, for each group (a column's, or a channel's).
template <bool UNI>
struct Moments {
    static constexpr int N = UNI ? 1 : 8;
    float n, mean[N], m2[N];
    __device__ __forceinline__ void merge(float other, const float (&om)[N], const float (&o2)[N]) {
        const float all = n + other;
        const float f = all > 0.0f ? other / all : 0.0f;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float d = om[k] - mean[k];
            mean[k] = __builtin_fmaf(d, f, mean[k]);
            m2[k] += __builtin_fmaf(d * d, f * n, o2[k]);
        }
        n = all;
    }
};
template <int DT, bool UNI>
__global__ __launch_bounds__(kGnThreads) void gn_stats_kernel(GnArgs a) {
    constexpr int N = UNI ? 1 : 8, U = (int)gn_batch(DT);
    __shared__ float lds[kGnThreads][2 * N + 1];
    const Column at(a, blockIdx.x);
    Moments<UNI> s = {};
    const uint8_t* x = (const uint8_t*)a.x.p;
    const int64_t first = (int64_t)at.sample * a.x.sample + (int64_t)at.c8 * 8;
    for (uint32_t batch = at.chunk; at.holds && batch < a.batches; batch += a.chunks) {
        const uint32_t p = batch * a.batch + at.row;
        if (p >= a.P) break;
        Raw<DT> raw[U];
        float on[U], count = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t q = p + (uint32_t)u * a.rows;
            on[u] = q < a.P ? 1.0f : 0.0f;
            count += on[u];
            raw[u] = load8<DT>(x, (first + (int64_t)(q < a.P ? q : p) * a.x.pixel) * kSize<DT>);
        }
        float mean[N], m2[N];
#pragma unroll
        for (int k = 0; k < N; ++k) mean[k] = m2[k] = 0.0f;
        const float all = UNI ? 8.0f * count : count, inv = 1.0f / all;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[8];
            widen8<DT>(raw[u], v);
#pragma unroll
            for (int k = 0; k < 8; ++k) if (on[u] != 0.0f) mean[UNI ? 0 : k] += v[k];
        }
#pragma unroll
        for (int k = 0; k < N; ++k) mean[k] *= inv;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[8];
            widen8<DT>(raw[u], v);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float d = v[k] - mean[UNI ? 0 : k];
                if (on[u] != 0.0f) m2[UNI ? 0 : k] = __builtin_fmaf(d, d, m2[UNI ? 0 : k]);
            }
        }
        s.merge(all, mean, m2);
    }
    // over the rows of a column, halves at a time
    float* mine = lds[threadIdx.x];
    mine[0] = s.n;
#pragma unroll
    for (int k = 0; k < N; ++k) { mine[1 + k] = s.mean[k]; mine[1 + N + k] = s.m2[k]; }
    for (uint32_t left = a.rows; left > 1;) {
        const uint32_t half = (left + 1) >> 1;
        __syncthreads();
        if (at.holds && at.row + half < left) {
            const float* o = lds[threadIdx.x + half * a.cols];
            float om[N], o2[N];
#pragma unroll
            for (int k = 0; k < N; ++k) { om[k] = o[1 + k]; o2[k] = o[1 + N + k]; }
            s.merge(o[0], om, o2);
            mine[0] = s.n;
#pragma unroll
            for (int k = 0; k < N; ++k) { mine[1 + k] = s.mean[k]; mine[1 + N + k] = s.m2[k]; }
        }
        left = half;
    }
    if (!at.holds || at.row != 0) return;
    float* out = a.partial + at.partial(a) * (2 * N);
#pragma unroll
    for (int k = 0; k < N; ++k) { out[2 * k] = s.mean[k]; out[2 * k + 1] = s.m2[k]; }
}

// Sum over the wavefront, in all lanes.
__device__ __forceinline__ double over_wave(double v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m);
    return v;
}
__device__ __forceinline__ uint32_t gn_wave() { return (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// Sum over the workgroup, in all threads, of two values.
__device__ __forceinline__ void over_block(double& u, double& v, double (&lds)[2][kGnThreads / 64]) {
    u = over_wave(u);
    v = over_wave(v);
    if ((threadIdx.x & 63u) == 0) {
        lds[0][threadIdx.x >> 6] = u;
        lds[1][threadIdx.x >> 6] = v;
    }
    __syncthreads();
    u = v = 0.0;
#pragma unroll
    for (int k = 0; k < kGnThreads / 64; ++k) {
        u += lds[0][k];
        v += lds[1][k];
    }
    __syncthreads();
}

// m and r of a sample's group, a workgroup each, from its columns' (channels') in all chunks, in binary64.
template <bool UNI>
__global__ __launch_bounds__(kGnThreads) void gn_finish_kernel(GnArgs a) {
    __shared__ double lds[2][kGnThreads / 64];
    const uint32_t i = blockIdx.x, sample = i / a.H, h = i - sample * a.H;
    const uint32_t each = UNI ? a.D / 8 : a.D, row = UNI ? a.C8 : a.C, items = each * a.chunks;
    const float* p = a.partial + ((size_t)sample * a.chunks * row + (size_t)h * each) * 2;
    // elements of a chunk's column: whole batches, but for the sample's last
    const uint32_t last = (a.batches - 1) % a.chunks, missing = a.batches * a.batch - a.P;
    const auto elements = [&](uint32_t chunk) {
        const uint32_t batches = (a.batches - chunk + a.chunks - 1) / a.chunks;
        return (UNI ? 8.0 : 1.0) * (double)(batches * a.batch - (chunk == last ? missing : 0));
    };
    // distances from the first part's mean, so that their squares cancel nothing
    const double from = (double)p[0], whole = (double)a.P * a.D;
    double off = 0.0, m2 = 0.0;
#pragma unroll 4
    for (uint32_t k = threadIdx.x; k < items; k += kGnThreads) {
        const uint32_t chunk = k / each;
        const hf2 v = *(const hf2*)(p + ((size_t)chunk * row + (k - chunk * each)) * 2);
        const double n = elements(chunk), d = (double)v.x - from;
        off += n * d;
        m2 += (double)v.y + n * d * d;
    }
    over_block(off, m2, lds);
    off /= whole;
    const double mean = from + off;
    m2 = m2 / whole - off * off;
    m2 = m2 > 0.0 || m2 != m2 ? m2 : 0.0;
    if (threadIdx.x != 0) return;
    a.mean[i] = (float)mean;
    a.rstd[i] = (float)(1.0 / sqrt(m2 + (double)a.eps));
}

// ------------------------------------------------------------------ y, context
// Leaves the context of a pass, 64 blocks of eight that follow each other in x laid out contiguously.
template <int BITS>
__device__ __forceinline__ void gn_compress_pass(const GnArgs& a, uint32_t pass, uint32_t lane, bool active, const float (&v)[8]) {
    const uint32_t e = pass * 64u + lane;
    float mn, step;
    const uint64_t codes = compress8<BITS>(v, active, 1 << a.block_shift, (uint64_t)pass * 64u, lane, a.seed_lo, a.seed_hi, mn, step);
    if (!active) return;
    store_codes<BITS>(a.packed + (uint64_t)e * BITS, codes);
    if ((lane & ((1u << a.block_shift) - 1u)) == 0) {
        a.gmin[e >> a.block_shift] = mn;
        a.gscale[e >> a.block_shift] = step;
    }
}
// The packed string ends at a multiple of 16 bytes, zeros behind the last code.
template <int BITS>
__device__ __forceinline__ void gn_zero_pad(const GnArgs& a, uint32_t lane) {
    const uint64_t bytes = (uint64_t)a.blocks8 * BITS;
    if (lane < (uint32_t)(0u - bytes & 15u)) a.packed[bytes + lane] = 0;
}

template <int DT, int BITS, bool UNI, bool SILU>
__global__ __launch_bounds__(kGnThreads) void gn_apply_kernel(GnArgs a) {
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t pass = blockIdx.x * (kGnThreads / 64) + gn_wave();
    if constexpr (BITS != 0)
        if (pass == 0) gn_zero_pad<BITS>(a, lane);
    if (pass >= a.stride_passes || pass >= a.passes) return;
    uint32_t e = pass * 64u + lane;                    // the lane's block of eight
    uint32_t q = divided(e, a.by_c8);                  // its pixel, of all samples'
    const uint32_t c = (e - q * a.C8) * 8u;
    const uint32_t e_step = a.stride_passes * 64u, q_step = e_step / a.C8;
    float w[8], b[8], rw[8];
    load_channels(a.w, a.w_f32, 1.0f, c, w);
    load_channels(a.b, a.w_f32, 0.0f, c, b);
    uint32_t sample = ~0u;
    OfGroups<UNI> m;
    for (;; ) {
        const bool active = e < a.blocks8;
        if (!active) q = a.B * a.P - 1;
        const uint32_t s = divided(q, a.by_p), p = q - s * a.P;
        const int64_t at = (int64_t)s * a.x.sample + (int64_t)p * a.x.pixel + c;
        const Raw<DT> raw = load8<DT>((const uint8_t*)a.x.p, at * kSize<DT>);
        if (s != sample) {
            m.load(a, a.mean + (size_t)s * a.H, 1, c);
            OfGroups<UNI> r;
            r.load(a, a.rstd + (size_t)s * a.H, 1, c);
#pragma unroll
            for (int k = 0; k < 8; ++k) rw[k] = r[k] * w[k];
            sample = s;
        }
        float v[8], y[8];
        widen8<DT>(raw, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = activate<DT, SILU>(__builtin_fmaf(v[k] - m[k], rw[k], b[k]));
        if (active)
            store8<DT>((uint8_t*)a.y.p, ((int64_t)s * a.y.sample + (int64_t)p * a.y.pixel + c) * kSize<DT>, y);
        if constexpr (BITS != 0) gn_compress_pass<BITS>(a, pass, lane, active, v);
        if (a.passes - pass <= a.stride_passes) return;
        pass += a.stride_passes;
        e += e_step;
        q += q_step;
    }
}

// ------------------------------------------------------------------- gradients
// n = (code step + minimum - m) r of a block of eight: where m and r are one, code (step r) + (minimum - m) r, an operation a
// value instead of four.
template <int BITS, bool UNI>
__device__ __forceinline__ void gn_normal(uint64_t codes, float mn, float step, const OfGroups<UNI>& m, const OfGroups<UNI>& r,
                                          float (&n)[8]) {
    if constexpr (UNI) {
        const float scale = step * r[0], shift = (mn - m[0]) * r[0];
        float q[8];
        codes_of<BITS>(codes, q);
#pragma unroll
        for (int k = 0; k < 8; ++k) n[k] = __builtin_fmaf(q[k], scale, shift);
    } else {
        decompress8<BITS>(codes, mn, step, n);
#pragma unroll
        for (int k = 0; k < 8; ++k) n[k] = (n[k] - m[k]) * r[k];
    }
}
// dy and x of a block of eight: from its codes or as they are.
template <int DT, int BITS>
struct GnInput {
    Raw<DT> dy, x;
    uint64_t codes;
    float mn, step;
    __device__ __forceinline__ void load(const GnArgs& a, uint32_t sample, uint32_t p, uint32_t c8) {
        dy = load8<DT>((const uint8_t*)a.dy.p, ((int64_t)sample * a.dy.sample + (int64_t)p * a.dy.pixel + (int64_t)c8 * 8) * kSize<DT>);
        load_x(a, sample, p, c8);
    }
    __device__ __forceinline__ void load_x(const GnArgs& a, uint32_t sample, uint32_t p, uint32_t c8) {
        if constexpr (BITS != 0) {
            const uint32_t e = (sample * a.P + p) * a.C8 + c8;
            codes = load_codes<BITS>(a.packed + (uint64_t)e * BITS);
            mn = a.gmin[e >> a.block_shift];
            step = a.gscale[e >> a.block_shift];
        } else {
            x = load8<DT>((const uint8_t*)a.x.p, ((int64_t)sample * a.x.sample + (int64_t)p * a.x.pixel + (int64_t)c8 * 8) * kSize<DT>);
        }
    }
    // n and dz
    template <bool UNI, bool SILU>
    __device__ __forceinline__ void take(const OfGroups<UNI>& m, const OfGroups<UNI>& r, const float (&w)[8], const float (&b)[8],
                                         float (&n)[8], float (&dz)[8]) const {
        widen8<DT>(dy, dz);
        if constexpr (BITS != 0) {
            gn_normal<BITS, UNI>(codes, mn, step, m, r, n);
        } else {
            widen8<DT>(x, n);
#pragma unroll
            for (int k = 0; k < 8; ++k) n[k] = (n[k] - m[k]) * r[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (SILU) dz[k] *= silu_slope<DT>(__builtin_fmaf(n[k], w[k], b[k]));
    }
};

// n of a block of eight.
template <int DT, int BITS, bool UNI>
__device__ __forceinline__ void gn_load_n(const GnArgs& a, uint32_t sample, uint32_t p, uint32_t c8, const OfGroups<UNI>& m,
                                          const OfGroups<UNI>& r, float (&n)[8]) {
    if constexpr (BITS != 0) {
        const uint32_t e = (sample * a.P + p) * a.C8 + c8;
        gn_normal<BITS, UNI>(load_codes<BITS>(a.packed + (uint64_t)e * BITS), a.gmin[e >> a.block_shift], a.gscale[e >> a.block_shift], m, r, n);
    } else {
        widen8<DT>(load8<DT>((const uint8_t*)a.x.p, ((int64_t)sample * a.x.sample + (int64_t)p * a.x.pixel + (int64_t)c8 * 8) * kSize<DT>), n);
#pragma unroll
        for (int k = 0; k < 8; ++k) n[k] = (n[k] - m[k]) * r[k];
    }
}

// A thread's pixels, U at a time.
template <int DT, int U>
struct GnPixels {
    static constexpr uint32_t kTurns = gn_batch(DT) / U;
    uint32_t batch, turn, p;
    __device__ __forceinline__ GnPixels(const GnArgs& a, const Column& at) : batch(at.chunk), turn(0), p(at.chunk * a.batch + at.row) {}
    __device__ __forceinline__ bool more(const GnArgs& a) const { return batch < a.batches && p < a.P; }
    __device__ __forceinline__ void next(const GnArgs& a, const Column& at) {
        if (++turn == kTurns) {
            turn = 0;
            batch += a.chunks;
            p = batch * a.batch + at.row;
        } else {
            p += U * a.rows;
            // the sample's last batch ends here
            if (p >= a.P) batch = a.batches;
        }
    }
    __device__ __forceinline__ bool holds(const GnArgs& a, int u) const { return p + (uint32_t)u * a.rows < a.P; }
    __device__ __forceinline__ uint32_t within(const GnArgs& a, int u) const { return holds(a, u) ? p + (uint32_t)u * a.rows : p; }
};

template <int DT, int BITS, bool UNI, bool SILU>
__global__ __launch_bounds__(kGnThreads) void gn_sums_kernel(GnArgs a) {
    constexpr int U = 2;
    __shared__ float lds[kGnThreads * 17];             // 16 values a thread, and one to shift the banks
    const Column at(a, blockIdx.x);
    const uint32_t c = at.c8 * 8u;
    float s0[8], s1[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) s0[k] = s1[k] = 0.0f;
    if (at.holds) {
        float w[8], b[8];
        load_channels(a.w, a.w_f32, 1.0f, c, w);
        load_channels(a.b, a.w_f32, 0.0f, c, b);
        OfGroups<UNI> m, r;
        m.load(a, a.mean + (size_t)at.sample * a.H, 1, c);
        r.load(a, a.rstd + (size_t)at.sample * a.H, 1, c);
        for (GnPixels<DT, U> px(a, at); px.more(a); px.next(a, at)) {
            GnInput<DT, BITS> in[U];
#pragma unroll
            for (int u = 0; u < U; ++u) in[u].load(a, at.sample, px.within(a, u), at.c8);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u > 0 && !px.holds(a, u)) break;
                float n[8], dz[8];
                in[u].template take<UNI, SILU>(m, r, w, b, n, dz);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    s0[k] += dz[k];
                    s1[k] = __builtin_fmaf(dz[k], n[k], s1[k]);
                }
            }
        }
    }
    float* mine = lds + threadIdx.x * 17;
#pragma unroll
    for (int k = 0; k < 8; ++k) { mine[k] = s0[k]; mine[8 + k] = s1[k]; }
    for (uint32_t left = a.rows; left > 1;) {
        const uint32_t half = (left + 1) >> 1;
        __syncthreads();
        if (at.holds && at.row + half < left) {
            const float* o = mine + half * a.cols * 17;
#pragma unroll
            for (int k = 0; k < 16; ++k) mine[k] += o[k];
        }
        left = half;
    }
    if (!at.holds || at.row != 0) return;
    float* out = a.partial + at.partial(a) * 16;
#pragma unroll
    for (int k = 0; k < 8; ++k) { out[2 * k] = mine[k]; out[2 * k + 1] = mine[8 + k]; }
}

// Of a slice of a sample's group, a workgroup each: the channels' sums over the chunks, and the slice's part of the means of g and g n,
// in binary64.
__global__ __launch_bounds__(kGnThreads) void gn_means_kernel(GnArgs a) {
    __shared__ double lds[2][kGnThreads];
    __shared__ double of_block[2][kGnThreads / 64];
    const uint32_t i = blockIdx.x / a.slices, slice = blockIdx.x - i * a.slices, sample = i / a.H, h = i - sample * a.H;
    // threads: the slice's channels, and as many parts of the chunks as fit
    const uint32_t wide = a.D - slice * 64u < 64u ? a.D - slice * 64u : 64u, parts = kGnThreads / wide;
    const uint32_t part = threadIdx.x / wide, d = threadIdx.x - part * wide, c = h * a.D + slice * 64u + d;
    double s0 = 0.0, s1 = 0.0, m1 = 0.0, m2 = 0.0;
    if (part < parts) {
        const float* p = a.partial + ((size_t)sample * a.chunks * a.C + c) * 2;
#pragma unroll 8
        for (uint32_t k = part; k < a.chunks; k += parts) {
            const hf2 v = *(const hf2*)(p + (size_t)k * a.C * 2);
            s0 += (double)v.x;
            s1 += (double)v.y;
        }
    }
    // over the parts, in their order
    lds[0][threadIdx.x] = s0;
    lds[1][threadIdx.x] = s1;
    __syncthreads();
    if (part == 0) {
        for (uint32_t k = 1; k < parts; ++k) {
            s0 += lds[0][d + k * wide];
            s1 += lds[1][d + k * wide];
        }
        *(hf2*)(a.sums + ((size_t)sample * a.C + c) * 2) = hf2{(float)s0, (float)s1};
        double w = 1.0;
        if (a.w) w = a.w_f32 ? (double)((const float*)a.w)[c]
                             : (double)__builtin_bit_cast(float, (uint32_t)((const uint16_t*)a.w)[c] << 16);
        m1 = w * s0;
        m2 = w * s1;
    }
    over_block(m1, m2, of_block);
    if (threadIdx.x != 0) return;
    *(hf2*)(a.means + 2 * (size_t)blockIdx.x) = hf2{(float)(m1 / ((double)a.P * a.D)), (float)(m2 / ((double)a.P * a.D))};
}

// into dw or db, if it is wanted
__device__ __forceinline__ void gn_put(const GnArgs& a, void* p, uint32_t c, float v) {
    if (!p) return;
    if (a.w_f32) ((float*)p)[c] = v;
    else ((uint16_t*)p)[c] = (uint16_t)bf16_pair_rne(v, 0.0f);
}
// dw and db of 32 channels: over the samples, eight parts of them, in binary64 and in a fixed order.
__device__ __forceinline__ void gn_weights(const GnArgs& a, uint32_t block, double (&lds)[2][kGnThreads]) {
    const uint32_t part = threadIdx.x >> 5, c = block * 32u + (threadIdx.x & 31u);
    double s0 = 0.0, s1 = 0.0;
    if (c < a.C)
        for (uint32_t s = part; s < a.B; s += kGnThreads / 32) {
            const float* p = a.sums + ((size_t)s * a.C + c) * 2;
            s0 += (double)p[0];
            s1 += (double)p[1];
        }
    lds[0][threadIdx.x] = s0;
    lds[1][threadIdx.x] = s1;
    __syncthreads();
    if (part != 0 || c >= a.C) return;
    for (uint32_t k = 1; k < kGnThreads / 32; ++k) {
        s0 += lds[0][threadIdx.x + 32 * k];
        s1 += lds[1][threadIdx.x + 32 * k];
    }
    gn_put(a, a.dw, c, (float)s1);
    gn_put(a, a.db, c, (float)s0);
}

template <int DT, int BITS, bool UNI, bool SILU>
__global__ __launch_bounds__(kGnThreads) void gn_dx_kernel(GnArgs a) {
    __shared__ double lds[2][kGnThreads];
    if (blockIdx.x >= a.dx_blocks) {
        gn_weights(a, blockIdx.x - a.dx_blocks, lds);
        return;
    }
    const Column at(a, blockIdx.x);
    if (!at.holds) return;
    const uint32_t c = at.c8 * 8u;
    float w[8], b[8];
    load_channels(a.w, a.w_f32, 1.0f, c, w);
    load_channels(a.b, a.w_f32, 0.0f, c, b);
    OfGroups<UNI> m, r, m1, m2;
    const size_t group = (size_t)at.sample * a.H;
    m.load(a, a.mean + group, 1, c);
    r.load(a, a.rstd + group, 1, c);
    m1.add(a, a.means + 2 * group * a.slices, c);
    m2.add(a, a.means + 2 * group * a.slices + 1, c);
    constexpr int U = 2;
    for (GnPixels<DT, U> px(a, at); px.more(a); px.next(a, at)) {
        GnInput<DT, BITS> in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) in[u].load(a, at.sample, px.within(a, u), at.c8);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u > 0 && !px.holds(a, u)) break;
            float n[8], dz[8];
            in[u].template take<UNI, SILU>(m, r, w, b, n, dz);
#pragma unroll
            for (int k = 0; k < 8; ++k) dz[k] = r[k] * __builtin_fmaf(-n[k], m2[k], __builtin_fmaf(dz[k], w[k], -m1[k]));
            store8<DT>((uint8_t*)a.dx.p, ((int64_t)at.sample * a.dx.sample + (int64_t)px.within(a, u) * a.dx.pixel + c) * kSize<DT>, dz);
        }
    }
}

// ------------------------------------------------------- maps held in registers
// A lane's place among the units that a workgroup holds.
struct WholePlace {
    uint32_t sample, col, row, rows, c8, unit, threads;
    int      wave, lane;
    bool     holds;
    __device__ __forceinline__ WholePlace(const GnArgs& a, uint32_t n_threads) : threads(n_threads) {
        // slabs of a cache line go to one XCD (every eighth workgroup): neighbours in this order
        const uint32_t per = a.norm_blocks >> 3, rest = a.norm_blocks & 7u, xcd = blockIdx.x & 7u;
        const uint32_t block = xcd * per + (xcd < rest ? xcd : rest) + (blockIdx.x >> 3);
        lane = (int)(threadIdx.x & 63u);
        wave = (int)gn_wave();
        sample = block / a.unit_slabs;
        col = threadIdx.x & ((1u << a.col_shift) - 1u);
        row = threadIdx.x >> a.col_shift;
        rows = threads >> a.col_shift;
        unit = ((block - sample * a.unit_slabs) << a.slab_shift) + (col >> a.unit_shift);
        const uint32_t cu = col & ((1u << a.unit_shift) - 1u);
        holds = unit < a.units && cu < a.unit_cols;
        c8 = unit * a.unit_cols + cu;
    }
};
// Sum of v over a slab's rows, for each of the lane's values; UNI: over its unit's columns too.  A wavefront's in binary32, theirs in
// binary64; in all lanes.
template <int NT, int N, bool UNI>
__device__ __forceinline__ void over_rows(const GnArgs& a, const WholePlace& at, float (&lds)[NT / 64][64 * N], float (&v)[N], double (&sum)[N]) {
    const int cols = 1 << a.col_shift, unit = UNI ? 1 << a.unit_shift : 1;
    for (int m = 1; m < 64; m <<= 1) {
        if (m >= unit && m < cols) continue;
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], m);
    }
    if (at.lane < cols) {
#pragma unroll
        for (int k = 0; k < N; ++k) lds[at.wave][at.lane * N + k] = v[k];
    }
    __syncthreads();
    const int c = at.lane & (cols - 1);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        sum[k] = 0.0;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) sum[k] += (double)lds[w][c * N + k];
    }
}
// Room for the sums of groups that are no whole columns: of the slab's channels, and of its groups.
template <int N>
struct GroupRoom {
    double of_channel[N][64 * 8];
    float  of_group[N][64 * 8];
};
template <>
struct GroupRoom<0> {};
// of_group: what finish makes of the groups' sums of of_channel, which the lanes of row 0 have filled.
template <int N, typename FINISH>
__device__ __forceinline__ void over_groups(const GnArgs& a, const WholePlace& at, GroupRoom<N>& room, FINISH finish) {
    __syncthreads();
    const uint32_t each = a.unit_cols * 8 / a.D;                        // groups of a unit
    for (uint32_t t = threadIdx.x; t < each << a.slab_shift; t += at.threads) {
        const uint32_t unit = t / each, first = (unit << a.unit_shift) * 8 + (t - unit * each) * a.D;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            double s = 0.0;
            for (uint32_t d = 0; d < a.D; ++d) s += room.of_channel[i][first + d];
            room.of_group[i][t] = finish(s);
        }
    }
    __syncthreads();
}
// of_group of the groups that the lane's channels are in.
__device__ __forceinline__ void of_lanes(const GnArgs& a, const WholePlace& at, const float (&of_group)[64 * 8], float (&v)[8]) {
    const uint32_t unit = at.col >> a.unit_shift, cu = at.col & ((1u << a.unit_shift) - 1u), each = a.unit_cols * 8 / a.D;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t t = unit * each + divided(cu * 8 + (uint32_t)k, a.by_d);
        v[k] = of_group[t < 512u ? t : 511u];          // (lanes that hold nothing)
    }
}
// What finish makes of a lane's groups' sums: of one group's, which all of its lanes have, or of the channels', which have to be added.
template <bool UNI, int N, int M, typename FINISH>
__device__ __forceinline__ void finish_sums(const GnArgs& a, const WholePlace& at, GroupRoom<M>& room, const double (&sum)[N], float (&v)[N], FINISH finish) {
    if constexpr (UNI) {
        v[0] = finish(sum[0]);
    } else {
        if (at.row == 0) {
#pragma unroll
            for (int k = 0; k < 8; ++k) room.of_channel[0][at.col * 8 + k] = sum[k];
        }
        over_groups<1>(a, at, room, finish);
        of_lanes(a, at, room.of_group[0], v);
    }
}

// Context of x by workgroups of their own, behind those that hold the maps.
template <int DT, int BITS, int NT>
__device__ __forceinline__ void gn_compress_blocks(const GnArgs& a) {
    const uint32_t lane = threadIdx.x & 63u, stride = (gridDim.x - a.norm_blocks) * (NT / 64);
    uint32_t pass = (blockIdx.x - a.norm_blocks) * (NT / 64) + gn_wave();
    if (pass == 0) gn_zero_pad<BITS>(a, lane);
    for (; pass < a.passes; pass += stride) {
        const uint32_t e = pass * 64u + lane;
        const bool active = e < a.blocks8;
        const uint32_t i = active ? e : a.blocks8 - 1, q = divided(i, a.by_c8), s = divided(q, a.by_p);
        const int64_t at = (int64_t)s * a.x.sample + (int64_t)(q - s * a.P) * a.x.pixel + (int64_t)(i - q * a.C8) * 8;
        float v[8];
        widen8<DT>(load8<DT>((const uint8_t*)a.x.p, at * kSize<DT>), v);
        gn_compress_pass<BITS>(a, pass, lane, active, v);
    }
}

// 1 / sqrt(v), rounded once: binary32's, and a step of Newton's in binary64.
__device__ __forceinline__ float inverse_root(double v) {
    const float r = 1.0f / __builtin_sqrtf((float)v);
    const double d = (double)r;
    return r > 0.0f ? (float)(d + 0.5 * d * (1.0 - v * d * d)) : r;      // (squares that have passed binary32: 0; NaN)
}

// One launch forward: x is read once for y; once more for a context, whose groups do not keep to the norm's.
template <int DT, bool UNI, bool SILU, int WHICH>
__global__ __launch_bounds__(kGnWhole[WHICH].threads) void gn_whole_kernel(GnArgs a, int bits) {
    constexpr int NT = (int)kGnWhole[WHICH].threads, R = (int)kGnWhole[WHICH].blocks, N = UNI ? 1 : 8;
    __shared__ float lds[2][NT / 64][64 * N];
    __shared__ GroupRoom<UNI ? 0 : 1> room;
    if (blockIdx.x >= a.norm_blocks) {
        switch (bits) {
            case 1: gn_compress_blocks<DT, 1, NT>(a); break;
            case 2: gn_compress_blocks<DT, 2, NT>(a); break;
            case 4: gn_compress_blocks<DT, 4, NT>(a); break;
            default: gn_compress_blocks<DT, 8, NT>(a); break;
        }
        return;
    }
    const WholePlace at(a, NT);
    const uint32_t c = at.c8 * 8u;
    const int64_t in = (int64_t)at.sample * a.x.sample + c;
    Raw<DT> raw[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const uint32_t p = at.row + (uint32_t)i * at.rows;
        raw[i] = Raw<DT>{};
        if (at.holds && p < a.P) raw[i] = load8<DT>((const uint8_t*)a.x.p, (in + (int64_t)p * a.x.pixel) * kSize<DT>);
    }
    float m[N], r[N];
    double sum[N];
#pragma unroll
    for (int k = 0; k < N; ++k) m[k] = r[k] = 0.0f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        float v[8];
        widen8<DT>(raw[i], v);
        if (UNI) m[0] += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        else
#pragma unroll
            for (int k = 0; k < 8; ++k) m[k % N] += v[k];
    }
    over_rows<NT, N, UNI>(a, at, lds[0], m, sum);
    finish_sums<UNI>(a, at, room, sum, m, [&](double v) { return (float)(v * a.inv); });
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (at.row + (uint32_t)i * at.rows >= a.P) continue;
        float v[8], s[8];
        widen8<DT>(raw[i], v);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float d = v[k] - m[k % N];
            s[k] = d * d;
        }
        if (UNI) r[0] += ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
        else
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k % N] += s[k];
    }
    if (!at.holds)
#pragma unroll
        for (int k = 0; k < N; ++k) r[k] = 0.0f;
    over_rows<NT, N, UNI>(a, at, lds[1], r, sum);
    finish_sums<UNI>(a, at, room, sum, r, [&](double v) { return inverse_root(v * a.inv + (double)a.eps); });
    if (!at.holds) return;
    if (a.mean && at.row == 0) {
        const uint32_t first = at.sample * a.H;
        if (UNI) {
            if ((at.col & ((1u << a.unit_shift) - 1u)) == 0) {
                a.mean[first + at.unit] = m[0];
                a.rstd[first + at.unit] = r[0];
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if ((c + (uint32_t)k) % a.D == 0) {
                    a.mean[first + (c + (uint32_t)k) / a.D] = m[k % N];
                    a.rstd[first + (c + (uint32_t)k) / a.D] = r[k % N];
                }
        }
    }
    float w[8], b[8];
    load_channels(a.w, a.w_f32, 1.0f, c, w);
    load_channels(a.b, a.w_f32, 0.0f, c, b);
    const int64_t out = (int64_t)at.sample * a.y.sample + c;
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] *= r[k % N];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const uint32_t p = at.row + (uint32_t)i * at.rows;
        if (p >= a.P) break;
        float v[8];
        widen8<DT>(raw[i], v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = activate<DT, SILU>(__builtin_fmaf(v[k] - m[k % N], w[k], b[k]));
        store8<DT>((uint8_t*)a.y.p, (out + (int64_t)p * a.y.pixel) * kSize<DT>, v);
    }
}

// Room for a slab's sums backward: of the lane's 16 values (its channels' dz, then dz n) by wavefronts, of the slab's channels, and of each
// column's g and g n; behind the wavefronts' sums, of groups that are no whole columns.
template <int NT>
struct SlabRoom {
    union {
        float of_wave[NT / 64][64 * 16];
        GroupRoom<2> of_groups;
    };
    double total[64 * 16], of_column[64][2];
};
// The slab's channels' sums of s, a wavefront's in binary32, theirs in binary64.
template <int NT>
__device__ __forceinline__ void over_slab(const GnArgs& a, const WholePlace& at, SlabRoom<NT>& room, float (&s)[16]) {
    const int cols = 1 << a.col_shift;
    for (int mask = cols; mask < 64; mask <<= 1)
#pragma unroll
        for (int k = 0; k < 16; ++k) s[k] += __shfl_xor(s[k], mask);
    if (at.lane < cols) {
#pragma unroll
        for (int k = 0; k < 16; ++k) room.of_wave[at.wave][at.lane * 16 + k] = s[k];
    }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < cols * 16; i += NT) {
        double v = 0.0;
#pragma unroll
        for (int k = 0; k < NT / 64; ++k) v += (double)room.of_wave[k][i];
        room.total[i] = v;
    }
    __syncthreads();
}
// mean g and mean g n of the lane's group, whose columns are whole.
template <int NT>
__device__ __forceinline__ void slab_means(const GnArgs& a, const WholePlace& at, SlabRoom<NT>& room, const float (&w)[8], float& m1, float& m2) {
    if ((int)threadIdx.x < 1 << a.col_shift) {
        double t0 = 0.0, t1 = 0.0;
        if (at.holds) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                t0 += (double)w[k] * room.total[threadIdx.x * 16 + k];
                t1 += (double)w[k] * room.total[threadIdx.x * 16 + 8 + k];
            }
        }
        room.of_column[threadIdx.x][0] = t0;
        room.of_column[threadIdx.x][1] = t1;
    }
    __syncthreads();
    const uint32_t first = at.col & ~((1u << a.unit_shift) - 1u);
    double t0 = 0.0, t1 = 0.0;
    for (uint32_t k = 0; k < a.unit_cols; ++k) {
        t0 += room.of_column[first + k][0];
        t1 += room.of_column[first + k][1];
    }
    m1 = (float)(t0 * a.inv);
    m2 = (float)(t1 * a.inv);
}
// dw and db of the lane's channels, or the sample's part of them.
template <int NT>
__device__ __forceinline__ void leave_weights(const GnArgs& a, const WholePlace& at, const SlabRoom<NT>& room) {
    if ((!a.dw && !a.db) || at.row != 0) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t c = at.c8 * 8u + (uint32_t)k;
        const float db = (float)room.total[at.col * 16 + k], dw = (float)room.total[at.col * 16 + 8 + k];
        if (a.B == 1) {
            gn_put(a, a.dw, c, dw);
            gn_put(a, a.db, c, db);
        } else {
            *(hf2*)(a.sums + ((size_t)at.sample * a.C + c) * 2) = hf2{db, dw};
        }
    }
}

// One launch backward for dx: dy is read once, dz stays in registers; x, mostly codes, is read again for dx.
template <int DT, int BITS, bool UNI, bool SILU, int WHICH>
__global__ __launch_bounds__(kGnWhole[WHICH].threads) void gn_whole_backward_kernel(GnArgs a) {
    constexpr int NT = (int)kGnWhole[WHICH].threads, R = (int)kGnWhole[WHICH].blocks;
    __shared__ SlabRoom<NT> slab;
    const WholePlace at(a, NT);
    const uint32_t c = at.c8 * 8u;
    float w[8], b[8], dz[R][8], s[16];
    OfGroups<UNI> m, r;
#pragma unroll
    for (int k = 0; k < 16; ++k) s[k] = 0.0f;
    if (at.holds) {
        load_channels(a.w, a.w_f32, 1.0f, c, w);
        load_channels(a.b, a.w_f32, 0.0f, c, b);
        m.load(a, a.mean + (size_t)at.sample * a.H, 1, c);
        r.load(a, a.rstd + (size_t)at.sample * a.H, 1, c);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const uint32_t p = at.row + (uint32_t)i * at.rows;
            if (p >= a.P) break;
            GnInput<DT, BITS> in;
            in.load(a, at.sample, p, at.c8);
            float n[8];
            in.template take<UNI, SILU>(m, r, w, b, n, dz[i]);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                s[k] += dz[i][k];
                s[8 + k] = __builtin_fmaf(dz[i][k], n[k], s[8 + k]);
            }
        }
    }
    over_slab<NT>(a, at, slab, s);
    float m1[UNI ? 1 : 8], m2[UNI ? 1 : 8];
    if constexpr (UNI) {
        slab_means<NT>(a, at, slab, w, m1[0], m2[0]);
    } else {
        if (at.row == 0) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    slab.of_groups.of_channel[i][at.col * 8 + k] = at.holds ? (double)w[k] * slab.total[at.col * 16 + 8 * i + k] : 0.0;
        }
        over_groups<2>(a, at, slab.of_groups, [&](double v) { return (float)(v * a.inv); });
        of_lanes(a, at, slab.of_groups.of_group[0], m1);
        of_lanes(a, at, slab.of_groups.of_group[1], m2);
    }
    if (!at.holds) return;
    leave_weights<NT>(a, at, slab);
    const int64_t out = (int64_t)at.sample * a.dx.sample + c;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const uint32_t p = at.row + (uint32_t)i * at.rows;
        if (p >= a.P) break;
        float n[8];
        gn_load_n<DT, BITS, UNI>(a, at.sample, p, at.c8, m, r, n);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            dz[i][k] = r[k] * __builtin_fmaf(-n[k], m2[k % (UNI ? 1 : 8)], __builtin_fmaf(dz[i][k], w[k], -m1[k % (UNI ? 1 : 8)]));
        }
        store8<DT>((uint8_t*)a.dx.p, (out + (int64_t)p * a.dx.pixel) * kSize<DT>, dz[i]);
    }
}
// The same for larger maps: few wavefronts with many registers each, which hold dy as it came, all of it on its way at once; x is
// loaded kAhead pixels ahead, both times.  (Of the 256 registers fp32 and SiLU need 1 to 2 more, at 8 bits 9 and 5.)
template <int DT, int BITS, bool SILU>
__global__ __launch_bounds__(kGnWhole[3].threads) void gn_held_backward_kernel(GnArgs a) {
    constexpr int NT = (int)kGnWhole[3].threads, R = (int)kGnWhole[3].blocks, kAhead = 4;
    __shared__ SlabRoom<NT> slab;
    const WholePlace at(a, NT);
    const uint32_t c = at.c8 * 8u;
    // lanes that hold nothing go through pixel 0 of column 0 without a part in the sums
    const uint32_t c8 = at.holds ? at.c8 : 0;
    const auto inside = [&](uint32_t p) { return p < a.P ? p : 0u; };
    // (an empty statement keeps the compiler from holding all addresses in registers)
    const auto step = [&](uint32_t& p) {
        p += at.rows;
        asm("" : "+v"(p));
    };
    uint32_t p = at.row;
    Raw<DT> dy[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        dy[i] = load8<DT>((const uint8_t*)a.dy.p, ((int64_t)at.sample * a.dy.sample + (int64_t)inside(p) * a.dy.pixel + (int64_t)c8 * 8) * kSize<DT>);
        step(p);
    }
    float w[8], b[8], s[16];
    load_channels(a.w, a.w_f32, 1.0f, c8 * 8u, w);
    load_channels(a.b, a.w_f32, 0.0f, c8 * 8u, b);
    OfGroups<true> m, r;
    m.load(a, a.mean + (size_t)at.sample * a.H, 1, c8 * 8u);
    r.load(a, a.rstd + (size_t)at.sample * a.H, 1, c8 * 8u);
#pragma unroll
    for (int k = 0; k < 16; ++k) s[k] = 0.0f;
    GnInput<DT, BITS> in[kAhead];
    p = at.row;
    uint32_t next = at.row;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        in[i].load_x(a, at.sample, inside(next), c8);
        step(next);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        float n[8], dz[8];
        GnInput<DT, BITS>& now = in[i % kAhead];
        now.dy = dy[i];
        now.template take<true, SILU>(m, r, w, b, n, dz);
        if (i + kAhead < R) now.load_x(a, at.sample, inside(next), c8);
        step(next);
        const bool counts = at.holds && p < a.P;
        step(p);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float v = counts ? dz[k] : 0.0f, u = counts ? n[k] : 0.0f;
            s[k] += v;
            s[8 + k] = __builtin_fmaf(v, u, s[8 + k]);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    over_slab<NT>(a, at, slab, s);
    float m1, m2;
    slab_means<NT>(a, at, slab, w, m1, m2);
    if (!at.holds) return;
    leave_weights<NT>(a, at, slab);
    const int64_t out = (int64_t)at.sample * a.dx.sample + c;
    p = next = at.row;
    asm("" : "+v"(p), "+v"(next));
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        in[i].load_x(a, at.sample, inside(next), c8);
        step(next);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        float n[8], dz[8];
        GnInput<DT, BITS>& now = in[i % kAhead];
        now.dy = dy[i];
        now.template take<true, SILU>(m, r, w, b, n, dz);
        if (i + kAhead < R) now.load_x(a, at.sample, inside(next), c8);
        step(next);
#pragma unroll
        for (int k = 0; k < 8; ++k) dz[k] = r[k] * __builtin_fmaf(-n[k], m2, __builtin_fmaf(dz[k], w[k], -m1));
        if (p < a.P) store8<DT>((uint8_t*)a.dx.p, (out + (int64_t)p * a.dx.pixel) * kSize<DT>, dz);
        step(p);
        __builtin_amdgcn_sched_barrier(0);
    }
}
__global__ __launch_bounds__(kGnThreads) void gn_weights_kernel(GnArgs a) {
    __shared__ double lds[2][kGnThreads];
    gn_weights(a, blockIdx.x, lds);
}

__global__ __launch_bounds__(kGnThreads) void gn_zero_kernel(GnArgs a) {
    const uint32_t c = blockIdx.x * kGnThreads + threadIdx.x;
    if (c >= a.C) return;
    for (void* p : {a.dw, a.db}) {
        if (!p) continue;
        if (a.w_f32) ((float*)p)[c] = 0.0f;
        else ((uint16_t*)p)[c] = 0;
    }
}

// ------------------------------------------------------------- host launchers
// Passes over memory, for maps of any size.
template <int DT, int BITS, bool UNI, bool SILU>
static void gn_launch(bool backward, const GnArgs& a, hipStream_t s) {
    const uint32_t slots = a.B * a.chunks * a.slabs;
    if (!backward) {
        hipLaunchKernelGGL((gn_stats_kernel<DT, UNI>), dim3(slots), dim3(kGnThreads), 0, s, a);
        hipLaunchKernelGGL((gn_finish_kernel<UNI>), dim3(a.B * a.H), dim3(kGnThreads), 0, s, a);
        const uint32_t waves = a.stride_passes < a.passes ? a.stride_passes : a.passes;
        hipLaunchKernelGGL((gn_apply_kernel<DT, BITS, UNI, SILU>), dim3((waves + 3) / 4), dim3(kGnThreads), 0, s, a);
    } else {
        GnArgs d = a;
        d.dx_blocks = slots;
        hipLaunchKernelGGL((gn_sums_kernel<DT, BITS, UNI, SILU>), dim3(slots), dim3(kGnThreads), 0, s, a);
        hipLaunchKernelGGL(gn_means_kernel, dim3(a.B * a.H * a.slices), dim3(kGnThreads), 0, s, a);
        const uint32_t extra = a.dw || a.db ? (a.C + 31) / 32 : 0;
        hipLaunchKernelGGL((gn_dx_kernel<DT, BITS, UNI, SILU>), dim3(slots + extra), dim3(kGnThreads), 0, s, d);
    }
}
template <int DT, int BITS, bool UNI, bool SILU, int WHICH>
static void gn_launch_whole(bool backward, const GnArgs& a, hipStream_t s) {
    constexpr uint32_t NT = kGnWhole[WHICH].threads;
    if (!backward) {
        // two passes a wavefront of those that compress
        uint32_t extra = BITS ? gn_up(a.passes, NT / 64 * 2) : 0;
        if (extra > 4096) extra = 4096;
        if (BITS && a.x.p == a.y.p) {                  // in place: x is compressed before it is overwritten
            GnArgs x = a;
            x.norm_blocks = 0;
            hipLaunchKernelGGL((gn_whole_kernel<DT, UNI, SILU, WHICH>), dim3(extra), dim3(NT), 0, s, x, BITS);
            extra = 0;
        }
        hipLaunchKernelGGL((gn_whole_kernel<DT, UNI, SILU, WHICH>), dim3(a.norm_blocks + extra), dim3(NT), 0, s, a, BITS);
    } else {
        hipLaunchKernelGGL((gn_whole_backward_kernel<DT, BITS, UNI, SILU, WHICH>), dim3(a.norm_blocks), dim3(NT), 0, s, a);
        if (a.B > 1 && (a.dw || a.db)) hipLaunchKernelGGL(gn_weights_kernel, dim3((a.C + 31) / 32), dim3(kGnThreads), 0, s, a);
    }
}
template <int DT, int BITS, bool SILU>
static void gn_launch_held(const GnArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((gn_held_backward_kernel<DT, BITS, SILU>), dim3(a.norm_blocks), dim3(kGnWhole[3].threads), 0, s, a);
    if (a.B > 1 && (a.dw || a.db)) hipLaunchKernelGGL(gn_weights_kernel, dim3((a.C + 31) / 32), dim3(kGnThreads), 0, s, a);
}
template <int DT, int BITS, bool UNI, bool SILU>
static void gn_launch_sized(bool backward, const GnArgs& a, int whole, hipStream_t s) {
    if (whole == 0) gn_launch<DT, BITS, UNI, SILU>(backward, a, s);
    else if (whole == 1) gn_launch_whole<DT, BITS, UNI, SILU, 0>(backward, a, s);
    else if (whole == 2) gn_launch_whole<DT, BITS, UNI, SILU, 1>(backward, a, s);
    else if constexpr (UNI) {
        if (whole == 3) gn_launch_whole<DT, BITS, UNI, SILU, 2>(backward, a, s);
        else if constexpr (gn_held(DT, BITS, SILU)) gn_launch_held<DT, BITS, SILU>(a, s);
    }
}
template <int DT, int BITS>
static void gn_launch_form(bool backward, const GnArgs& a, int act, int whole, hipStream_t s) {
    if (gn_uniform(a)) {
        if (act) gn_launch_sized<DT, BITS, true, true>(backward, a, whole, s);
        else gn_launch_sized<DT, BITS, true, false>(backward, a, whole, s);
    } else {
        if (act) gn_launch_sized<DT, BITS, false, true>(backward, a, whole, s);
        else gn_launch_sized<DT, BITS, false, false>(backward, a, whole, s);
    }
}
template <int DT>
static void gn_launch_bits(bool backward, const GnArgs& a, int bits, int act, int whole, hipStream_t s) {
    switch (bits) {
        case 0: gn_launch_form<DT, 0>(backward, a, act, whole, s); break;
        case 1: gn_launch_form<DT, 1>(backward, a, act, whole, s); break;
        case 2: gn_launch_form<DT, 2>(backward, a, act, whole, s); break;
        case 4: gn_launch_form<DT, 4>(backward, a, act, whole, s); break;
        default: gn_launch_form<DT, 8>(backward, a, act, whole, s); break;
    }
}
static int gn_launch_any(bool backward, const GnArgs& a, int dtype, int bits, int act, int whole, hipStream_t s) {
    if (dtype == GACT_DT_F32) gn_launch_bits<GACT_DT_F32>(backward, a, bits, act, whole, s);
    else gn_launch_bits<GACT_DT_BF16>(backward, a, bits, act, whole, s);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace gact

extern "C" int gact_launch_group_norm(const gact::GnArgs* a, int dtype, int bits, int act, int whole, void* stream) {
    return gact::gn_launch_any(false, *a, dtype, bits, act, whole, (hipStream_t)stream);
}
extern "C" int gact_launch_group_norm_backward(const gact::GnArgs* a, int dtype, int bits, int act, int whole, void* stream) {
    return gact::gn_launch_any(true, *a, dtype, bits, act, whole, (hipStream_t)stream);
}
extern "C" int gact_launch_group_norm_zero(const gact::GnArgs* a, void* stream) {
    hipLaunchKernelGGL(gact::gn_zero_kernel, dim3((a->C + gact::kGnThreads - 1) / gact::kGnThreads), dim3(gact::kGnThreads), 0,
                       (hipStream_t)stream, *a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}
