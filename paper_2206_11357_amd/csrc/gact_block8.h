// Eight consecutive elements a lane, for the kernels of gact_heads.hip and gact_group_norm.hip: loads and stores, sums and
// extremes over neighbouring lanes, and the quantizer of a block of eight, which is one block of its noise generator and
// `bits` whole bytes of the packed string.
#ifndef GACT_BLOCK8_H
#define GACT_BLOCK8_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gact_codec.h"
#include "gact_device.h"

namespace gact {

typedef uint32_t h4 __attribute__((ext_vector_type(4)));
typedef uint32_t h2 __attribute__((ext_vector_type(2)));
typedef float    hf4 __attribute__((ext_vector_type(4)));
// at any address that an element can have
typedef h4  h4_any __attribute__((aligned(2)));
typedef hf4 hf4_any __attribute__((aligned(4)));

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
// Minimum and maximum of a group, over four lanes or more.
__device__ __forceinline__ void minmax_over(float& mn, float& mx, int lanes) {
    mn = min_xor2(min_xor1(mn));
    mx = max_xor2(max_xor1(mx));
    if (lanes > 4) {
        mn = min_half_mirror(mn);
        mx = max_half_mirror(mx);
        if (lanes > 8) {
            mn = min_mirror(mn);
            mx = max_mirror(mx);
            if (lanes > 16) {
                mn = fmin2(mn, swizzle_xor16(mn));
                mx = fmax2(mx, swizzle_xor16(mx));
                if (lanes > 32) {
                    float a, b;
                    swap_halves(mn, a, b);
                    mn = fmin2(a, b);
                    swap_halves(mx, a, b);
                    mx = fmax2(a, b);
                }
            }
        }
    }
}

// ------------------------------------------------------------------- elements
template <int DT>
struct Raw {
    h4 w[DT == GACT_DT_F32 ? 2 : 1];
};
template <int DT>
constexpr int kSize = DT == GACT_DT_F32 ? 4 : 2;
// Addresses are a base of the wavefront's and an offset of the lane's, in bytes: 32 bits where the part is steady, which a load
// takes as they are.
template <int DT, typename OFFSET>
__device__ __forceinline__ Raw<DT> load8(const uint8_t* base, OFFSET at) {
    Raw<DT> r;
    if (DT == GACT_DT_F32) {
        r.w[0] = __builtin_bit_cast(h4, *(const hf4_any*)(base + at));
        r.w[DT == GACT_DT_F32 ? 1 : 0] = __builtin_bit_cast(h4, *(const hf4_any*)(base + at + 16));
    } else {
        r.w[0] = *(const h4_any*)(base + at);
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
template <int DT, typename OFFSET>
__device__ __forceinline__ void store8(uint8_t* base, OFFSET at, const float (&v)[8]) {
    if (DT == GACT_DT_F32) {
        *(hf4_any*)(base + at) = hf4{v[0], v[1], v[2], v[3]};
        *(hf4_any*)(base + at + 16) = hf4{v[4], v[5], v[6], v[7]};
    } else {
        *(h4_any*)(base + at) = h4{bf16_pair_rne(v[0], v[1]), bf16_pair_rne(v[2], v[3]),
                                             bf16_pair_rne(v[4], v[5]), bf16_pair_rne(v[6], v[7])};
    }
}

// ---------------------------------------------------------------------- codes
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
__device__ __forceinline__ void store_codes(uint8_t* p, uint64_t codes) {
    if (BITS == 1) *p = (uint8_t)codes;
    if (BITS == 2) *(uint16_t*)p = (uint16_t)codes;
    if (BITS == 4) *(uint32_t*)p = (uint32_t)codes;
    if (BITS == 8) *(uint64_t*)p = codes;
}
template <int BITS>
__device__ __forceinline__ uint64_t load_codes(const uint8_t* p) {
    if (BITS == 1) return *p;
    if (BITS == 2) return *(const uint16_t*)p;
    if (BITS == 4) return *(const uint32_t*)p;
    return *(const uint64_t*)p;
}

// Eight codes as numbers.
template <int BITS>
__device__ __forceinline__ void codes_of(uint64_t codes, float (&q)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        // a nibble of every byte of a word, so that the bytes convert in place
        const uint32_t word = BITS == 8 && k >= 4 ? (uint32_t)(codes >> 32) : (uint32_t)codes;
        q[k] = (float)(BITS == 8 ? word >> (8 * (k & 3)) & 0xFFu
                     : BITS == 4 ? ((k & 1 ? word >> 4 : word) & 0x0F0F0F0Fu) >> (8 * (k >> 1)) & 0xFFu
                     : word >> (k * BITS) & ((1u << BITS) - 1u));
    }
}
// x of eight elements from their codes.
template <int BITS>
__device__ __forceinline__ void decompress8(uint64_t codes, float mn, float step, float (&x)[8]) {
    codes_of<BITS>(codes, x);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float t = x[k] * step;
        x[k] = t + mn;
    }
}

// Codes, minimum and step of a pass's groups, `lanes` neighbouring lanes each; `block` is the noise generator's first block of the
// pass (the wavefront's), `mine` what the lane adds to it.  A lane that is not active holds no element.
template <int BITS>
__device__ __forceinline__ uint64_t compress8(const float (&v)[8], bool active, int lanes, uint64_t block, uint32_t mine,
                                              uint32_t seed_lo, uint32_t seed_hi, float& mn, float& step) {
    uint32_t r[4];
    // the high word of the block's number is the wavefront's, unless the low one wraps in this pass
    if (__builtin_expect((uint32_t)block <= 0xFFFFFFFFu - 64u, 1))
        philox_head_uniform((uint32_t)block + mine, PhiloxUniform((uint32_t)(block >> 32), seed_lo, seed_hi), seed_lo, seed_hi, r);
    else philox_head_any(block + mine, seed_lo, seed_hi, r);
    philox_rounds<3>(r[0], r[1], r[2], r[3], seed_lo, seed_hi);
    mn = fmin3(v[0], v[1], v[2]);
    float mx = fmax3(v[0], v[1], v[2]);
    mn = fmin3(mn, v[3], v[4]); mx = fmax3(mx, v[3], v[4]);
    mn = fmin3(mn, v[5], v[6]); mx = fmax3(mx, v[5], v[6]);
    mn = fmin3(mn, v[7], v[7]); mx = fmax3(mx, v[7], v[7]);
    if (!active) { mn = __builtin_inff(); mx = -__builtin_inff(); }
    minmax_over(mn, mx, lanes);
    mn = mn + 0.0f;                                    // store -0 as +0
    const float range = mx - mn;
    float inv = 0.0f;
    step = 0.0f;
    if (range >= 0x1p-100f) { inv = (float)((1u << BITS) - 1u) / range; step = div_levels<BITS>(range); }
    return codes8<BITS>(v, mn, inv, r);
}

}  // namespace gact

#endif
