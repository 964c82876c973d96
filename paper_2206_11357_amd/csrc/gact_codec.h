// The quantizer's parts that act on registers, for the kernels of gact_kernels.hip, gact_heads.hip and
// gact_group_norm.hip: lane moves and group statistics, the noise generator, rounding and packing.  The exact arithmetic is stated in include/gact.h.
#ifndef GACT_CODEC_H
#define GACT_CODEC_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gact {

// ---------------------------------------------------------------- lane moves
__device__ __forceinline__ float swizzle_xor16(float v) {
    // bit-mask mode: and 0x1f, or 0, xor 0x10 (lane ^ 16 inside each half wave)
    return __builtin_bit_cast(
        float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), (16 << 10) | 0x1F));
}
__device__ __forceinline__ float lane_read(float v, int src_lane) {
    return __builtin_bit_cast(
        float, __builtin_amdgcn_ds_bpermute(src_lane << 2, __builtin_bit_cast(int, v)));
}

// min / max of finite values (v_min_f32 / v_min3_f32).  The sign of a zero
// result is not defined by these; the stored minimum is canonicalised later.
__device__ __forceinline__ float fmin2(float a, float b) { return __builtin_fminf(a, b); }
__device__ __forceinline__ float fmax2(float a, float b) { return __builtin_fmaxf(a, b); }

// v = min / max(v, v of the DPP-selected lane) in one instruction.  Written as
// assembly because the compiler otherwise moves the DPP operand into its own
// register and re-canonicalises both inputs (4 instructions per step).
// A DPP operand must not be read in the two issue slots after a vector
// instruction has written it, and the compiler's hazard pass does not look
// inside an assembly statement, so each statement brings its own wait states.
#define GACT_DPP_MINMAX(NAME, OP, CTRL)                                                  \
    __device__ __forceinline__ float NAME(float v) {                                     \
        float r;                                                                          \
        asm("s_nop 1\n\t" OP " %0, %1, %1 " CTRL " row_mask:0xf bank_mask:0xf"          \
            : "=v"(r) : "v"(v));                                                          \
        return r;                                                                         \
    }
GACT_DPP_MINMAX(min_xor1, "v_min_f32_dpp", "quad_perm:[1,0,3,2]")
GACT_DPP_MINMAX(max_xor1, "v_max_f32_dpp", "quad_perm:[1,0,3,2]")
GACT_DPP_MINMAX(min_xor2, "v_min_f32_dpp", "quad_perm:[2,3,0,1]")
GACT_DPP_MINMAX(max_xor2, "v_max_f32_dpp", "quad_perm:[2,3,0,1]")
GACT_DPP_MINMAX(min_half_mirror, "v_min_f32_dpp", "row_half_mirror")
GACT_DPP_MINMAX(max_half_mirror, "v_max_f32_dpp", "row_half_mirror")
GACT_DPP_MINMAX(min_mirror, "v_min_f32_dpp", "row_mirror")
GACT_DPP_MINMAX(max_mirror, "v_max_f32_dpp", "row_mirror")
#undef GACT_DPP_MINMAX

// All lanes of a group (lpg neighbouring lanes, lpg a power of two <= 32,
// groups aligned to lpg) end up with the group's min and max.  After the two
// quad steps all lanes of a quad agree, so the 8- and 16-lane mirrors pair
// each lane with one from the other half.
__device__ __forceinline__ void group_minmax_pow2(float& mn, float& mx, int lpg) {
    if (lpg > 1)  { mn = min_xor1(mn);        mx = max_xor1(mx); }
    if (lpg > 2)  { mn = min_xor2(mn);        mx = max_xor2(mx); }
    if (lpg > 4)  { mn = min_half_mirror(mn); mx = max_half_mirror(mx); }
    if (lpg > 8)  { mn = min_mirror(mn);      mx = max_mirror(mx); }
    if (lpg > 16) { mn = fmin2(mn, swizzle_xor16(mn)); mx = fmax2(mx, swizzle_xor16(mx)); }
}

// ------------------------------------------------------------------- Philox
// Philox4x32-10 (Salmon et al., SC'11) on counter (c0, c1, 0, 0), key (k0, k1).
constexpr uint32_t kPhiloxM0 = 0xD2511F53u, kPhiloxM1 = 0xCD9E8D57u;
constexpr uint32_t kPhiloxW0 = 0x9E3779B9u, kPhiloxW1 = 0xBB67AE85u;

// three-input xor in one v_bitop3_b32 (truth table 0x96)
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
    return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}

// rounds FIRST .. 9 (round r uses the key bumped r times)
template <int FIRST>
__device__ __forceinline__ void philox_rounds(uint32_t& c0, uint32_t& c1, uint32_t& c2, uint32_t& c3,
                                              uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = FIRST; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)kPhiloxM0 * c0;
        const uint64_t p1 = (uint64_t)kPhiloxM1 * c2;
        const uint32_t n0 = xor3((uint32_t)(p1 >> 32), c1, k0 + (uint32_t)r * kPhiloxW0);
        const uint32_t n2 = xor3((uint32_t)(p0 >> 32), c3, k1 + (uint32_t)r * kPhiloxW1);
        c1 = (uint32_t)p1;
        c3 = (uint32_t)p0;
        c0 = n0;
        c2 = n2;
    }
}

// Rounds 0..2 of a block whose counter is (c0, c1u, 0, 0) with the high word c1u
// and the key uniform over the wavefront -- the case for every block of a tile
// unless the low counter word wraps inside the tile.  Counter words 2 and 3
// being zero, part of these rounds is the same for every lane and is computed
// once per wavefront, on the scalar unit (PhiloxUniform):
//   round 0: M1 * 0 = 0, so word 0 becomes c1u ^ k0 (uniform) and word 1 is 0;
//   round 1: M0 * (uniform word 0) is a scalar product; its low half is the
//            new, uniform, word 3;
//   round 2: the uniform word 3 and the key fold into one scalar operand.
// Four 32 x 32 -> 64 multiplies per block instead of six.
struct PhiloxUniform {
    uint32_t f2, g2;
    __device__ __forceinline__ PhiloxUniform(uint32_t c1u, uint32_t k0, uint32_t k1) {
        const uint32_t a0 = c1u ^ k0;                                      // round 0, word 0
        const uint64_t P0 = (uint64_t)kPhiloxM0 * a0;                       // round 1 product
        f2 = (uint32_t)(P0 >> 32) ^ (k1 + kPhiloxW1);                       // round 1: word 2 = f2 ^ old word 3
        g2 = (uint32_t)P0 ^ (k1 + 2u * kPhiloxW1);                          // round 2: word 2 = hi(M0 word 0) ^ g2
    }
};
__device__ __forceinline__ void philox_head_uniform(uint32_t c0, const PhiloxUniform& u, uint32_t k0,
                                                    uint32_t k1, uint32_t st[4]) {
    const uint64_t p0 = (uint64_t)kPhiloxM0 * c0;                           // round 0
    const uint32_t a2 = (uint32_t)(p0 >> 32) ^ k1;
    const uint32_t a3 = (uint32_t)p0;
    const uint64_t p1 = (uint64_t)kPhiloxM1 * a2;                           // round 1
    const uint32_t b0 = (uint32_t)(p1 >> 32) ^ (k0 + kPhiloxW0);
    const uint32_t b1 = (uint32_t)p1;
    const uint32_t b2 = a3 ^ u.f2;
    const uint64_t q0 = (uint64_t)kPhiloxM0 * b0;                           // round 2
    const uint64_t q1 = (uint64_t)kPhiloxM1 * b2;
    st[0] = xor3((uint32_t)(q1 >> 32), b1, k0 + 2u * kPhiloxW0);
    st[1] = (uint32_t)q1;
    st[2] = (uint32_t)(q0 >> 32) ^ u.g2;
    st[3] = (uint32_t)q0;
}

// The same three rounds for any per-lane 64-bit block number.
__device__ __forceinline__ void philox_head_any(uint64_t blk, uint32_t k0, uint32_t k1, uint32_t st[4]) {
    uint32_t c0 = (uint32_t)blk, c1 = (uint32_t)(blk >> 32), c2 = 0u, c3 = 0u;
#pragma unroll
    for (int r = 0; r < 3; ++r) {
        const uint64_t p0 = (uint64_t)kPhiloxM0 * c0;
        const uint64_t p1 = (uint64_t)kPhiloxM1 * c2;
        const uint32_t n0 = xor3((uint32_t)(p1 >> 32), c1, k0 + (uint32_t)r * kPhiloxW0);
        const uint32_t n2 = xor3((uint32_t)(p0 >> 32), c3, k1 + (uint32_t)r * kPhiloxW1);
        c1 = (uint32_t)p1;
        c3 = (uint32_t)p0;
        c0 = n0;
        c2 = n2;
    }
    st[0] = c0; st[1] = c1; st[2] = c2; st[3] = c3;
}

// Three-input min / max of finite values.  As assembly because the compiler
// puts a canonicalising v_max_f32 x, x in front of values it cannot prove to be
// free of signalling NaNs (everything that was widened from bf16 with bit
// operations); non-finite input is outside the contract.
__device__ __forceinline__ float fmin3(float a, float b, float c) {
    float r;
    asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float fmax3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// x[j] <- x[j] + b[j % 4] for eight values, rounded toward minus infinity.  The
// wavefront's binary32 rounding mode (MODE bits 1:0) is switched to round-down
// for exactly these eight additions and back to nearest-even; the block is one
// volatile statement, so no other floating-point instruction can be scheduled
// into it and everything outside keeps the nearest-even contract.
__device__ __forceinline__ void add8_round_down(float (&x)[8], float b0, float b1, float b2, float b3) {
    asm volatile(
        "s_setreg_imm32_b32 hwreg(HW_REG_MODE, 0, 2), 2\n\t"
        "v_add_f32 %0, %8, %0\n\t"
        "v_add_f32 %1, %9, %1\n\t"
        "v_add_f32 %2, %10, %2\n\t"
        "v_add_f32 %3, %11, %3\n\t"
        "v_add_f32 %4, %8, %4\n\t"
        "v_add_f32 %5, %9, %5\n\t"
        "v_add_f32 %6, %10, %6\n\t"
        "v_add_f32 %7, %11, %7\n\t"
        "s_setreg_imm32_b32 hwreg(HW_REG_MODE, 0, 2), 0"
        : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7])
        : "s"(b0), "s"(b1), "s"(b2), "s"(b3));
}

// Instructions the compiler does not select on its own.
// floor(x) as int32 in one instruction.
__device__ __forceinline__ int32_t cvt_floor_i32(float x) {
    int32_t r;
    asm("v_cvt_flr_i32_f32 %0, %1" : "=v"(r) : "v"(x));
    return r;
}
// M * (low / high 16 bits of w) + c
template <int M>
__device__ __forceinline__ uint32_t mad_lo16(uint32_t w, uint32_t c) {
    uint32_t r;
    asm("v_mad_u32_u16 %0, %1, %3, %2" : "=v"(r) : "v"(w), "v"(c), "n"(M));
    return r;
}
template <int M>
__device__ __forceinline__ uint32_t mad_hi16(uint32_t w, uint32_t c) {
    uint32_t r;
    asm("v_mad_u32_u16 %0, %1, %3, %2 op_sel:[1,0,0,0]" : "=v"(r) : "v"(w), "v"(c), "n"(M));
    return r;
}
// bits of a where m is set, of b elsewhere
__device__ __forceinline__ uint32_t select_bits(uint32_t m, uint32_t a, uint32_t b) {
    return __builtin_amdgcn_bitop3_b32(m, a, b, 0xCA);
}

// two fp32 -> two bf16 (low half = a), round to nearest even: v_cvt_pk_bf16_f32
typedef float  f2v  __attribute__((ext_vector_type(2)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair_rne(float a, float b) {
    const f2v v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf2v));
}

// range / (2^BITS - 1), correctly rounded, for range >= 2^-100: a product with the rounded reciprocal
// and one fused correction (P. Markstein, IBM J. Res. Dev. 34 (1990) 111: four instructions with the
// fix-up instead of the eleven of a general division).  Every significand was compared with the division
// on the host for the divisors 3, 15 and 255; the result does not depend on the exponent as long as the
// remainder (down to 2^-149) and the quotient are exact.  The fix-up gives an infinite range, whose
// correction is inf - inf, its infinite quotient.
template <int BITS>
__device__ __forceinline__ float div_levels(float range) {
    constexpr float Bf = (float)((1u << BITS) - 1u), r = 1.0f / Bf;
    if (BITS == 1) return range;
    const float q = range * r;
    return __builtin_amdgcn_div_fixupf(__builtin_fmaf(__builtin_fmaf(-q, Bf, range), r, q), Bf, range);
}

// Eight 4-bit fields, each in bits 17..20 of its word, to one word: field k in bits 4k..4k+3.
// Byte 2 of a word holds its field; three byte permutes gather four of them.
__device__ __forceinline__ uint32_t gather_nibbles(const uint32_t (&n)[8]) {
    uint32_t d[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        d[h] = __builtin_amdgcn_perm(n[2 + h], n[0 + h], 0x0C0C0602u);
        d[h] = __builtin_amdgcn_perm(n[4 + h], d[h], 0x0C060100u);
        d[h] = __builtin_amdgcn_perm(n[6 + h], d[h], 0x06020100u);
    }
    return select_bits(0x0F0F0F0Fu, d[0] >> 1, d[1] << 3);
}

// every BITS-wide field f of w replaced by -f modulo 2^BITS
template <int BITS>
__device__ __forceinline__ uint32_t negate_fields(uint32_t w) {
    if (BITS == 1) return w;
    constexpr uint32_t one = BITS == 2 ? 0x55555555u : 0x11111111u, top = one << (BITS - 1);
    return ((~w & ~top) + one) ^ (~w & top);
}

}  // namespace gact

#endif
