// Norms of queries and keys for each head with the position rotation in the same pass, and their gradients, for
// MI355X (gfx950).
//
//   r = 1 / sqrt(mean x^2 + eps),  n = x r w,  y = R(position) n                    (a head of a token: a row)
//   dn = R^T dy,  g = dn w,  dx = r (g - x r mean(g x r)),  dw = sum over rows of dn x r
// R turns the pairs (i, i + rot/2) or (2i, 2i + 1) of the first `rot` elements by the position's angles.
//
// Bound by HBM: each input is read once, each output written once.  Eight consecutive elements a lane, so that a
// head is 1, 2, 4 ... 64 neighbouring lanes (the last ones idle where dim / 8 is no power of two), a wavefront
// takes as many rows at a time as fit, and a row's sums are a few lane moves.  The partner of an element under
// rotation is in the same lane, or in the same place of another lane of the head.
//
// A lane's eight elements are one block of the compressor's noise generator and `bits` whole bytes of the packed
// string, and a group is a power of two of neighbouring lanes: so the forward pass leaves the compressed context of x
// (codes, minima and steps as gact_compress gives them) from the registers that hold x for the norm, and the
// backward pass takes x from the codes, which are never written out decompressed.  r is kept from the forward pass
// in binary32: dn x^ r and the first term of dx are then linear in x^, so that the rounding noise leaves their
// expectation where it is (Sec. 3.1 asks it of the compressor); from x^ itself r would be biased.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gact_codec.h"
#include "gact_device.h"
#include "gact_heads.h"

namespace gact {

typedef uint32_t h4 __attribute__((ext_vector_type(4)));
typedef uint32_t h2 __attribute__((ext_vector_type(2)));
typedef float    hf4 __attribute__((ext_vector_type(4)));
// at any address that an element can have
typedef h4  h4_any __attribute__((aligned(2)));
typedef hf4 hf4_any __attribute__((aligned(4)));

constexpr int kHeadThreads = 64 * kHeadWaves;

__device__ __forceinline__ uint32_t divided(uint32_t x, const Divisor& d) {
    return d.magic == 0 ? x : (uint32_t)(((uint64_t)x * d.magic) >> 32) >> d.shift;
}

// ------------------------------------------------------------------ lane moves
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ void swap_halves(float v, float& a, float& b) {
    typedef uint32_t pair __attribute__((ext_vector_type(2)));
    const uint32_t w = __builtin_bit_cast(uint32_t, v);
    const pair p = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const uint32_t x = p.x, y = p.y;
    a = __builtin_bit_cast(float, x);
    b = __builtin_bit_cast(float, y);
}
// Sum over `lanes` neighbouring lanes, a power of two, in all of them.
__device__ __forceinline__ float add_over(float v, int lanes) {
    if (lanes > 1) v += dpp<0xB1>(v);                  // quad_perm [1,0,3,2]
    if (lanes > 2) v += dpp<0x4E>(v);                  // quad_perm [2,3,0,1]
    if (lanes > 4) v += dpp<0x141>(v);                 // row_half_mirror
    if (lanes > 8) v += dpp<0x140>(v);                 // row_mirror
    if (lanes > 16) v += swizzle_xor16(v);
    if (lanes > 32) { float a, b; swap_halves(v, a, b); v = a + b; }
    return v;
}
__device__ __forceinline__ void minmax_over(float& mn, float& mx, int lanes) {
    group_minmax_pow2(mn, mx, lanes);
    if (lanes > 32) {
        float a, b;
        swap_halves(mn, a, b);
        mn = fmin2(a, b);
        swap_halves(mx, a, b);
        mx = fmax2(a, b);
    }
}

// ------------------------------------------------------------------- elements
template <int DT>
struct Raw {
    h4 w[DT == GACT_DT_F32 ? 2 : 1];
};
template <int DT>
__device__ __forceinline__ Raw<DT> load8(const void* base, int64_t e) {
    Raw<DT> r;
    if (DT == GACT_DT_F32) {
        const float* p = (const float*)base + e;
        r.w[0] = __builtin_bit_cast(h4, *(const hf4_any*)p);
        r.w[DT == GACT_DT_F32 ? 1 : 0] = __builtin_bit_cast(h4, *(const hf4_any*)(p + 4));
    } else {
        r.w[0] = *(const h4_any*)((const uint16_t*)base + e);
    }
    return r;
}
template <int DT>
__device__ __forceinline__ void widen8(const Raw<DT>& r, float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (DT == GACT_DT_F32) {
            const uint32_t a = r.w[0][k], b = r.w[DT == GACT_DT_F32 ? 1 : 0][k];
            v[k] = __builtin_bit_cast(float, a);
            v[4 + k] = __builtin_bit_cast(float, b);
        } else {
            const uint32_t a = r.w[0][k];
            v[2 * k] = __builtin_bit_cast(float, a << 16);
            v[2 * k + 1] = __builtin_bit_cast(float, a & 0xFFFF0000u);
        }
    }
}
template <int DT>
__device__ __forceinline__ void store8(void* base, int64_t e, const float (&v)[8]) {
    if (DT == GACT_DT_F32) {
        float* p = (float*)base + e;
        *(hf4_any*)p = hf4{v[0], v[1], v[2], v[3]};
        *(hf4_any*)(p + 4) = hf4{v[4], v[5], v[6], v[7]};
    } else {
        *(h4_any*)((uint16_t*)base + e) = h4{bf16_pair_rne(v[0], v[1]), bf16_pair_rne(v[2], v[3]),
                                             bf16_pair_rne(v[4], v[5]), bf16_pair_rne(v[6], v[7])};
    }
}
__device__ __forceinline__ float load_weight(const void* w, int w_f32, int d) {
    if (w_f32) return ((const float*)w)[d];
    return __builtin_bit_cast(float, (uint32_t)((const uint16_t*)w)[d] << 16);
}

// ------------------------------------------------------------------- rotation
// A lane's place: of the 64 >> lanes_shift rows of a pass, the one that it works on, and its elements d .. d + 7.
struct Place {
    int lane, row, j, d;
    bool in_head;                                      // d is one of the head's elements
    __device__ __forceinline__ Place(const HeadArgs& a) {
        lane = threadIdx.x & 63;
        row = lane >> a.lanes_shift;
        j = lane & ((1 << a.lanes_shift) - 1);
        d = j * 8;
        in_head = d < a.dim;
    }
};

// A row's token and head, and where its elements begin in a tensor.
struct Row {
    uint32_t token, head, batch, at;                   // at: the token's place in its sequence
    __device__ __forceinline__ Row(const HeadArgs& a, const HeadPart& p, uint32_t row) {
        token = divided(row, p.by_heads);
        head = row - token * p.heads;
        batch = divided(token, a.by_seq);
        at = token - batch * a.seq;
    }
    __device__ __forceinline__ int64_t in(const HeadTensor& t) const {
        return (int64_t)batch * t.batch + (int64_t)at * t.token + (int64_t)head * t.head;
    }
};

// Cosines and sines of the lane's elements at one position.  HALVES: pairs (i, i + rot/2), eight angles a lane, the same
// in the lane that holds the partners; else pairs (2i, 2i + 1), four angles.  A position outside the table reads
// nothing and turns by NaN.
template <bool HALVES>
struct Angles {
    static constexpr int N = HALVES ? 8 : 4;
    float c[N], s[N];
    int partner = 0;                                   // HALVES: the lane with the elements' partners
    float sign = 1.0f;                                 // HALVES: of the sine, in the lane's own element
    bool turned = false;
    __device__ __forceinline__ Angles(const HeadArgs& a, const Place& at) {
#pragma unroll
        for (int k = 0; k < N; ++k) { c[k] = 1.0f; s[k] = 0.0f; }
        turned = at.j < a.rot_lanes;
        if (HALVES) {
            const int half = a.rot_lanes >> 1;
            const bool second = at.j >= half;
            partner = turned ? (second ? at.lane - half : at.lane + half) : at.lane;
            sign = second ? 1.0f : -1.0f;
        }
    }
    __device__ __forceinline__ void load(const HeadArgs& a, const Place& at, const Row& r) {
        if (!turned) return;
        const int64_t position = a.positions ? a.positions[r.token] : (int64_t)r.at;
        const int half = a.rot_lanes >> 1;
        const int first = HALVES ? 8 * (at.j < half ? at.j : at.j - half) : 4 * at.j;
        if ((uint64_t)position < (uint64_t)a.n_positions) {
            const int64_t o = position * (a.rot_lanes * 4) + first;
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                const hf4 cc = *(const hf4_any*)(a.cos + o + k), ss = *(const hf4_any*)(a.sin + o + k);
#pragma unroll
                for (int i = 0; i < 4; ++i) { c[k + i] = cc[i]; s[k + i] = ss[i]; }
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) c[k] = s[k] = __builtin_nanf("");
        }
    }
    // v turned by the angles (BACK: by their negatives)
    template <bool BACK>
    __device__ __forceinline__ void turn(float (&v)[8]) const {
        if (HALVES) {
            const float sg = BACK ? -sign : sign;
            float p[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) p[k] = lane_read(v[k], partner);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float t = __builtin_fmaf(p[k], sg * s[k % N], v[k] * c[k % N]);
                v[k] = turned ? t : v[k];
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float x = v[2 * k], y = v[2 * k + 1], sn = BACK ? -s[k] : s[k];
                const float tx = __builtin_fmaf(-y, sn, x * c[k]), ty = __builtin_fmaf(x, sn, y * c[k]);
                v[2 * k] = turned ? tx : x;
                v[2 * k + 1] = turned ? ty : y;
            }
        }
    }
};

// ------------------------------------------------------------------- context
// Group of element d of row `row`.
__device__ __forceinline__ int64_t group_of(const HeadArgs& a, uint32_t row, int d) {
    return a.groups_per_row ? (int64_t)row * a.groups_per_row + (d >> a.group_shift) : (int64_t)(row >> a.row_shift);
}

// Codes of eight elements, the first in the low bits: compress_tile's rounding (its comment derives it) of one
// block of noise.
template <int BITS>
__device__ __forceinline__ uint64_t codes8(const float (&v)[8], float mn, float inv, const uint32_t (&r)[4]) {
    constexpr uint32_t B = (1u << BITS) - 1u;
    constexpr int kPerNib = BITS <= 4 ? 4 / BITS : 1;
    const float ninv = -(inv * 0x1p17f);
    float tn[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        tn[j] = (v[j] - mn) * (ninv * (float)(1 << (kPerNib == 4 ? (j & 3) : kPerNib == 2 ? 2 * (j & 1) : 0)));
    if (BITS <= 4) {
        constexpr float m = 12582912.0f;                                   // 1.5 * 2^23
        if (kPerNib == 1) add8_round_down(tn, m + 1.0f, m + 1.0f, m + 1.0f, m + 1.0f);
        if (kPerNib == 2) add8_round_down(tn, m + 1.0f, m + 4.0f, m + 1.0f, m + 4.0f);
        if (kPerNib == 4) add8_round_down(tn, m + 1.0f, m + 2.0f, m + 4.0f, m + 8.0f);
        uint32_t y[8], nib[8] = {};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t n1 = __builtin_bit_cast(uint32_t, tn[j]), w = r[j >> 1];
            if (kPerNib == 1) y[j] = (j & 1) ? mad_hi16<2>(w, n1) : mad_lo16<2>(w, n1);
            if (kPerNib == 2) y[j] = (j & 1) ? mad_hi16<8>(w, n1) : mad_lo16<2>(w, n1);
            if (kPerNib == 4) y[j] = (j & 1) ? ((j & 2) ? mad_hi16<16>(w, n1) : mad_hi16<4>(w, n1))
                                             : ((j & 2) ? mad_lo16<8>(w, n1) : mad_lo16<2>(w, n1));
        }
#pragma unroll
        for (int i = 0; i < 8 / kPerNib; ++i) {
            uint32_t n = y[i * kPerNib];
            if (kPerNib == 2) n = select_bits(3u << 19, y[i * kPerNib + 1 % kPerNib], n);
            if (kPerNib == 4) {
                n = select_bits(1u << 18, y[i * kPerNib + 1 % kPerNib], n);
                n = select_bits(1u << 20, y[i * kPerNib + 3 % kPerNib], select_bits(1u << 19, y[i * kPerNib + 2 % kPerNib], n));
            }
            nib[i] = n;
        }
        constexpr uint32_t kept = BITS == 4 ? 0xFFFFFFFFu : (1u << (8 * BITS % 32)) - 1u;
        return negate_fields<BITS < 8 ? BITS : 1>(gather_nibbles(nib)) & kept;
    }
    uint32_t out[2] = {0u, 0u};
#pragma unroll
    for (int j = 7; j >= 0; --j) {
        const uint32_t n1 = (uint32_t)(cvt_floor_i32(tn[j]) + 1);
        const uint32_t y = (j & 1) ? mad_hi16<2>(r[j >> 1], n1) : mad_lo16<2>(r[j >> 1], n1);
        int32_t nq = (int32_t)y >> 17;
        nq = nq > -(int32_t)B ? nq : -(int32_t)B;
        out[j >> 2] = ((j & 3) == 3 ? 0u : out[j >> 2] << 8) + (uint32_t)nq;
        if ((j & 3) == 0) out[j >> 2] = 0u - out[j >> 2];
    }
    return (uint64_t)out[1] << 32 | out[0];
}

template <int BITS>
__device__ __forceinline__ void store_codes(uint8_t* packed, int64_t e, uint64_t codes) {
    uint8_t* p = packed + (e >> 3) * BITS;
    if (BITS == 1) *p = (uint8_t)codes;
    if (BITS == 2) *(uint16_t*)p = (uint16_t)codes;
    if (BITS == 4) *(uint32_t*)p = (uint32_t)codes;
    if (BITS == 8) *(uint64_t*)p = codes;
}
template <int BITS>
__device__ __forceinline__ uint64_t load_codes(const uint8_t* packed, int64_t e) {
    const uint8_t* p = packed + (e >> 3) * BITS;
    if (BITS == 1) return *p;
    if (BITS == 2) return *(const uint16_t*)p;
    if (BITS == 4) return *(const uint32_t*)p;
    return *(const uint64_t*)p;
}

// Leaves the context of a pass: v holds the lane's elements of row `row`, e the first one's index.
template <int BITS>
__device__ __forceinline__ void compress_pass(const HeadArgs& a, const HeadPart& p, const Place& at, uint32_t row,
                                              bool active, const float (&v)[8]) {
    const int64_t e = (int64_t)row * a.dim + at.d;
    uint32_t r[4];
    philox_head_any((uint64_t)e >> 3, p.seed_lo, p.seed_hi, r);
    philox_rounds<3>(r[0], r[1], r[2], r[3], p.seed_lo, p.seed_hi);
    float mn = fmin3(v[0], v[1], v[2]), mx = fmax3(v[0], v[1], v[2]);
    mn = fmin3(mn, v[3], v[4]); mx = fmax3(mx, v[3], v[4]);
    mn = fmin3(mn, v[5], v[6]); mx = fmax3(mx, v[5], v[6]);
    mn = fmin3(mn, v[7], v[7]); mx = fmax3(mx, v[7], v[7]);
    if (!active) { mn = __builtin_inff(); mx = -__builtin_inff(); }
    minmax_over(mn, mx, a.group_lanes);
    mn = mn + 0.0f;                                    // store -0 as +0
    const float range = mx - mn;
    float inv = 0.0f, step = 0.0f;
    if (range >= 0x1p-100f) { inv = (float)((1u << BITS) - 1u) / range; step = div_levels<BITS>(range); }
    const uint64_t codes = codes8<BITS>(v, mn, inv, r);
    if (!active) return;
    store_codes<BITS>(p.packed, e, codes);
    if ((at.lane & (a.group_lanes - 1)) == 0) {
        const int64_t g = group_of(a, row, at.d);
        p.gmin[g] = mn;
        p.gscale[g] = step;
    }
}

// The packed string ends at a multiple of 16 bytes; what is behind the last code is zero.
template <int BITS>
__device__ __forceinline__ void zero_pad(const HeadArgs& a, const HeadPart& p, int lane) {
    const int64_t bytes = ((int64_t)p.rows * a.dim >> 3) * BITS;
    if (lane < (int)(-bytes & 15)) p.packed[bytes + lane] = 0;
}

// -------------------------------------------------------------------- kernels
// Part and wavefront of a workgroup.
__device__ __forceinline__ int part_of(const HeadArgs& a, uint32_t& block) {
    block = blockIdx.x;
    if (block < a.part[0].blocks) return 0;
    block -= a.part[0].blocks;
    return 1;
}

template <int DT, int BITS, bool HALVES>
__global__ __launch_bounds__(kHeadThreads) void heads_kernel(HeadArgs a) {
    uint32_t block;
    const HeadPart& p = a.part[part_of(a, block)];
    const Place at(a);
    const uint32_t wave = block * kHeadWaves + (threadIdx.x >> 6);
    const uint32_t first = wave * p.run;
    if (first >= p.passes) return;
    const uint32_t end = first + p.run < p.passes ? first + p.run : p.passes;
    float w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = p.w && at.in_head ? load_weight(p.w, a.w_f32, at.d + k) : 1.0f;
    Angles<HALVES> angles(a, at);
    uint32_t token = 0xFFFFFFFFu;
    const int lanes = 1 << a.lanes_shift, rows = 64 >> a.lanes_shift;
    for (uint32_t pass = first; pass < end; ++pass) {
        const uint32_t row = pass * (uint32_t)rows + (uint32_t)at.row;
        const bool active = at.in_head && row < p.rows;
        const Row r(a, p, row < p.rows ? row : p.rows - 1);
        Raw<DT> raw = {};
        if (active) raw = load8<DT>(p.in.p, r.in(p.in) + at.d);
        if (__any(r.token != token)) {
            token = r.token;
            angles.load(a, at, r);
        }
        float v[8];
        widen8<DT>(raw, v);
        float ss = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) ss = __builtin_fmaf(v[k], v[k], ss);
        ss = add_over(ss, lanes);
        const float rstd = 1.0f / __builtin_sqrtf(__builtin_fmaf(ss, a.inv_dim, a.eps));
        float n[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) n[k] = v[k] * rstd * w[k];
        angles.template turn<false>(n);
        if (active) store8<DT>(p.out.p, r.in(p.out) + at.d, n);
        if (active && p.rstd && at.j == 0) p.rstd[row] = rstd;
        if constexpr (BITS != 0) compress_pass<BITS>(a, p, at, row, active, v);
    }
    if constexpr (BITS != 0)
        if (end == p.passes) zero_pad<BITS>(a, p, at.lane);
}

template <int DT, int BITS, bool HALVES>
__global__ __launch_bounds__(kHeadThreads) void heads_backward_kernel(HeadArgs a) {
    __shared__ float lds[kHeadWaves][64 * 8];
    uint32_t block;
    const HeadPart& p = a.part[part_of(a, block)];
    const Place at(a);
    const uint32_t wave = block * kHeadWaves + (threadIdx.x >> 6);
    const uint32_t first = wave * p.run < p.passes ? wave * p.run : p.passes;
    const uint32_t end = p.passes - first > p.run ? first + p.run : p.passes;
    float w[8], dw[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        w[k] = p.w && at.in_head ? load_weight(p.w, a.w_f32, at.d + k) : 1.0f;
        dw[k] = 0.0f;
    }
    Angles<HALVES> angles(a, at);
    uint32_t token = 0xFFFFFFFFu;
    const int lanes = 1 << a.lanes_shift, rows = 64 >> a.lanes_shift;
    for (uint32_t pass = first; pass < end; ++pass) {
        const uint32_t row = pass * (uint32_t)rows + (uint32_t)at.row;
        const bool active = at.in_head && row < p.rows;
        const Row r(a, p, row < p.rows ? row : p.rows - 1);
        Raw<DT> raw = {}, raw_x = {};
        uint64_t codes = 0;
        float mn = 0.0f, step = 0.0f, rstd = 0.0f;
        if (active) {
            raw = load8<DT>(p.in.p, r.in(p.in) + at.d);
            rstd = p.rstd[row];
            if constexpr (BITS != 0) {
                codes = load_codes<BITS>(p.packed, (int64_t)row * a.dim + at.d);
                const int64_t g = group_of(a, row, at.d);
                mn = p.gmin[g];
                step = p.gscale[g];
            } else {
                raw_x = load8<DT>(p.x.p, r.in(p.x) + at.d);
            }
        }
        if (__any(r.token != token)) {
            token = r.token;
            angles.load(a, at, r);
        }
        float dn[8], x[8];
        widen8<DT>(raw, dn);
        if constexpr (BITS != 0) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t q = (uint32_t)(codes >> (k * BITS)) & ((1u << BITS) - 1u);
                const float t = (float)q * step;
                x[k] = t + mn;
            }
        } else {
            widen8<DT>(raw_x, x);
        }
        angles.template turn<true>(dn);
        float s = 0.0f, g[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            x[k] *= rstd;
            g[k] = dn[k] * w[k];
            s = __builtin_fmaf(g[k], x[k], s);
        }
        s = add_over(s, lanes) * a.inv_dim;
        if (active) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                dw[k] = __builtin_fmaf(dn[k], x[k], dw[k]);
                g[k] = rstd * __builtin_fmaf(-x[k], s, g[k]);
            }
            store8<DT>(p.out.p, r.in(p.out) + at.d, g);
        }
    }
    if (!p.partial) return;
    // over the wavefront's rows, then over the block's wavefronts
    float* mine = lds[threadIdx.x >> 6];
#pragma unroll
    for (int k = 0; k < 8; ++k) mine[k * 64 + at.lane] = dw[k];
    __syncthreads();
    for (int d = (int)threadIdx.x; d < a.dim; d += kHeadThreads) {
        float sum = 0.0f;
        for (int v = 0; v < kHeadWaves; ++v)
            for (int c = 0; c < rows; ++c) sum += lds[v][(d & 7) * 64 + c * lanes + (d >> 3)];
        p.partial[(size_t)block * a.dim + d] = sum;
    }
}

// dw of one part: its blocks' sums, 32 elements a block of 16 x 32 threads, added in binary64 and in a fixed order.
constexpr int kDwRows = 16, kDwColumns = 32;
__global__ __launch_bounds__(kDwRows * kDwColumns) void heads_dw_kernel(HeadArgs a) {
    __shared__ double lds[kDwRows][kDwColumns];
    const HeadPart& p = a.part[blockIdx.y];
    if (!p.dw) return;
    const int col = threadIdx.x % kDwColumns, row = threadIdx.x / kDwColumns, d = blockIdx.x * kDwColumns + col;
    double sum = 0.0;
    if (d < a.dim)
        for (uint32_t b = row; b < p.blocks; b += kDwRows) sum += (double)p.partial[(size_t)b * a.dim + d];
    lds[row][col] = sum;
    __syncthreads();
    if (row != 0 || d >= a.dim) return;
    for (int k = 1; k < kDwRows; ++k) sum += lds[k][col];
    if (a.w_f32) ((float*)p.dw)[d] = (float)sum;
    else ((uint16_t*)p.dw)[d] = (uint16_t)bf16_pair_rne((float)sum, 0.0f);
}

// ------------------------------------------------------------- host launchers
template <int DT, int BITS, bool HALVES>
static void launch(bool backward, const HeadArgs& a, unsigned blocks, hipStream_t s) {
    if (backward) hipLaunchKernelGGL((heads_backward_kernel<DT, BITS, HALVES>), dim3(blocks), dim3(kHeadThreads), 0, s, a);
    else hipLaunchKernelGGL((heads_kernel<DT, BITS, HALVES>), dim3(blocks), dim3(kHeadThreads), 0, s, a);
}
template <int DT, bool HALVES>
static void launch_bits(bool backward, const HeadArgs& a, int bits, unsigned blocks, hipStream_t s) {
    switch (bits) {
        case 0: launch<DT, 0, HALVES>(backward, a, blocks, s); break;
        case 1: launch<DT, 1, HALVES>(backward, a, blocks, s); break;
        case 2: launch<DT, 2, HALVES>(backward, a, blocks, s); break;
        case 4: launch<DT, 4, HALVES>(backward, a, blocks, s); break;
        default: launch<DT, 8, HALVES>(backward, a, blocks, s); break;
    }
}
static int launch_any(bool backward, const HeadArgs& a, int dtype, int bits, int halves, hipStream_t s) {
    const unsigned blocks = a.part[0].blocks + a.part[1].blocks;
    if (dtype == GACT_DT_F32) {
        if (halves) launch_bits<GACT_DT_F32, true>(backward, a, bits, blocks, s);
        else launch_bits<GACT_DT_F32, false>(backward, a, bits, blocks, s);
    } else {
        if (halves) launch_bits<GACT_DT_BF16, true>(backward, a, bits, blocks, s);
        else launch_bits<GACT_DT_BF16, false>(backward, a, bits, blocks, s);
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace gact

extern "C" int gact_launch_heads(const gact::HeadArgs* a, int dtype, int bits, int halves, int backward, void* stream) {
    return gact::launch_any(backward != 0, *a, dtype, bits, halves, (hipStream_t)stream);
}

extern "C" int gact_launch_heads_dw(const gact::HeadArgs* a, int parts, void* stream) {
    hipLaunchKernelGGL(gact::heads_dw_kernel, dim3((a->dim + gact::kDwColumns - 1) / gact::kDwColumns, parts),
                       dim3(gact::kDwRows * gact::kDwColumns), 0, (hipStream_t)stream, *a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}
