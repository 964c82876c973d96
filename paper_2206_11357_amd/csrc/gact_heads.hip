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
//
// Us and TB/s of what is read and written: 8192 tokens of 32 + 8 heads of 128, bf16, head by head 28.5 (5.9); with 4-bit
// contexts, 32768 tokens 167 (4.6), backward 150 (5.2); 8192 tokens of 16 + 16 of 64, 21.6 (3.5) and 15.8 (4.9); fp32, 12608
// of 16 + 16 of 64, 2 bits 44.4 (4.9) and 47.0 (4.7).  A copy reaches 6.8 where the cache holds its 200 MB, 5.7 for 400 MB, 5.0 for
// 4 GB.  The compressing forward pass in bf16 is bound by its arithmetic, the noise and the rounding: without them 150 us of the 167.
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

// ------------------------------------------------------------------- rotation
// How a part's passes lie in its tensors (lay_out_heads on the host).
//   kAny      any number of heads: each lane finds its row's token and addresses for itself
//   kSteady   a token's heads are a multiple of a pass's rows, or they divide them and the passes of a sequence come out
//             even: the addresses are the wavefront's, counted on from pass to pass, and what a lane adds to them is the
//             same in every pass
//   3 .. 5    the same, and the log2 of a head's lanes, all of which hold elements (heads of 64, 128, 256): no lane is ever
//             idle, and row sums are so many lane moves without a question
// Us, bf16, kAny | kSteady | the last: 8192 tokens of 32 + 8 heads of 128 34.2 | 30.6 | 29.6; 32768 tokens with 4-bit contexts
// 198 | 180 | 172, backward 194 | 165 | 150; backward of 8192 tokens of 16 + 16 of 64, 20.1 | 18.4 | 16.1.
constexpr bool steady(int mode) { return mode != kAny; }
constexpr bool full(int mode) { return mode >= kFullModes; }
template <int MODE>
__device__ __forceinline__ int lanes_shift(const HeadArgs& a) { return full(MODE) ? MODE : a.lanes_shift; }

// A lane's place: of the 64 >> lanes_shift rows of a pass, the one that it works on, and its elements d .. d + 7.
template <int MODE>
struct Place {
    int lane, row, j, d, shift;
    bool in_head;                                      // d is one of the head's elements
    __device__ __forceinline__ Place(const HeadArgs& a) {
        shift = lanes_shift<MODE>(a);
        lane = threadIdx.x & 63;
        row = lane >> shift;
        j = lane & ((1 << shift) - 1);
        d = j * 8;
        in_head = full(MODE) || d < a.dim;
    }
    // whether the lane holds elements of a pass that begins with row `first`
    __device__ __forceinline__ bool holds(const HeadPart& p, uint32_t first) const {
        return full(MODE) || (in_head && (steady(MODE) || first + (uint32_t)row < p.rows));
    }
    // the lane's weights; 1 without
    __device__ __forceinline__ void weights(const HeadArgs& a, const HeadPart& p, float (&w)[8]) const {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = 1.0f;
        if (!p.w || !in_head) return;
        if (a.w_f32) widen8<GACT_DT_F32>(load8<GACT_DT_F32>((const uint8_t*)p.w, (uint32_t)d * 4u), w);
        else widen8<GACT_DT_BF16>(load8<GACT_DT_BF16>((const uint8_t*)p.w, (uint32_t)d * 2u), w);
    }
};

// Where a unit begins, in the first TENSORS tensors of its part.
template <int MODE, int TENSORS>
struct Unit {
    UnitPlace at;
    int64_t   first[TENSORS];                          // elements in front of the rows
    __device__ __forceinline__ Unit(const HeadArgs& a, const HeadPart& p, const Place<MODE>& place, uint32_t unit)
        : at(unit_place(a, p, steady(MODE), unit, (uint32_t)place.row, place.shift)) {
#pragma unroll
        for (int k = 0; k < TENSORS; ++k) first[k] = unit_first(p.t[k], steady(MODE), at);
    }
};
// kAny: the whole of what is in front of a lane's row is its own
template <int MODE>
struct LaneOffset {
    typedef uint32_t type;
};
template <>
struct LaneOffset<kAny> {
    typedef int64_t type;
};

// Where the lane's elements stand in the rotation.
template <bool HALVES>
struct Turn {
    bool  turned, second;                              // the lane's elements are rotated; HALVES: are of the second half
    int   partner, first;                              // HALVES: the lane with the elements' partners; the first angle
    template <typename PLACE>
    __device__ __forceinline__ Turn(const HeadArgs& a, const PLACE& at) {
        const int half = a.rot_lanes >> 1;
        turned = at.j < a.rot_lanes;
        second = at.j >= half;
        partner = !turned ? at.lane : second ? at.lane - half : at.lane + half;
        first = HALVES ? 8 * (second ? at.j - half : at.j) : 4 * at.j;
    }
};

// Cosines and sines of the lane's elements at one position.  HALVES: pairs (i, i + rot/2), eight angles a lane, the same in
// the lane that holds the partners, the sine with the sign that the forward pass gives the partner; else pairs (2i, 2i + 1),
// four angles.  Behind rot the angles are 0.  A position outside the tables reads nothing and turns by NaN.
template <bool HALVES>
struct Angles {
    static constexpr int N = HALVES ? 8 : 4;
    float c[N], s[N];
    __device__ __forceinline__ Angles() {
#pragma unroll
        for (int k = 0; k < N; ++k) { c[k] = 1.0f; s[k] = 0.0f; }
    }
    template <int MODE, int TENSORS>
    __device__ __forceinline__ void load(const HeadArgs& a, const HeadPart& p, const Turn<HALVES>& turn,
                                         const Unit<MODE, TENSORS>& u, uint32_t lane_token) {
        if (a.rot_lanes == 0) return;
        int64_t position = (int64_t)(u.at.at + lane_token);
        if (a.positions) {
            // nothing writes them while the kernel runs: a scalar load where the token is the wavefront's
            if (steady(MODE) && p.tokens_per_pass == 1)
                position = ((const __attribute__((address_space(4))) int64_t*)(uintptr_t)a.positions)[u.at.token];
            else position = a.positions[u.at.token + lane_token];
        }
        if (!turn.turned) return;
        const bool inside = (uint64_t)position < (uint64_t)a.n_positions;
        const int64_t o = position * (a.rot_lanes * 4) + turn.first;
        const float nan = __builtin_nanf("");
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            hf4 cc = {nan, nan, nan, nan}, ss = cc;
            if (inside) { cc = *(const hf4_any*)(a.cos + o + k); ss = *(const hf4_any*)(a.sin + o + k); }
#pragma unroll
            for (int i = 0; i < 4; ++i) { c[k + i] = cc[i]; s[k + i] = HALVES && !turn.second ? -ss[i] : ss[i]; }
        }
    }
    // v turned by the angles (BACK: by their negatives); behind rot it stays, infinities too, which 0 times would make NaN.
    // (A lane's partner is turned as it is.)
    template <bool BACK>
    __device__ __forceinline__ void turn(float (&v)[8], const Turn<HALVES>& at) const {
        if (!at.turned) return;
        if (HALVES) {
            float p[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) p[k] = lane_read(v[k], at.partner);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __builtin_fmaf(BACK ? -p[k] : p[k], s[k % N], v[k] * c[k % N]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float x = v[2 * k], y = v[2 * k + 1];
                v[2 * k] = __builtin_fmaf(BACK ? y : -y, s[k], x * c[k]);
                v[2 * k + 1] = __builtin_fmaf(BACK ? -x : x, s[k], y * c[k]);
            }
        }
    }
};

// ------------------------------------------------------------------- context
// Where a pass's context lies: rows, and blocks of eight elements, each `bits` bytes of the packed string and one of noise.
template <int BITS>
struct Spot {
    float*   rstd;
    uint8_t* packed;
    float*   gmin;
    float*   gscale;
    uint64_t block;
    uint32_t row;
    int      blocks, groups, rows;                     // of a pass
    __device__ __forceinline__ Spot(const HeadArgs& a, const HeadPart& p, uint32_t pass, int shift) {
        rows = 64 >> shift;
        blocks = rows * (a.dim >> 3);
        groups = a.groups_per_row ? rows * a.groups_per_row : rows >> a.row_shift;
        row = pass * (uint32_t)rows;
        rstd = p.rstd + row;
        block = (uint64_t)pass * (uint32_t)blocks;
        packed = p.packed + block * BITS;
        gmin = p.gmin + (int64_t)pass * groups;
        gscale = p.gscale + (int64_t)pass * groups;
    }
    __device__ __forceinline__ void next() {
        row += (uint32_t)rows;
        rstd += rows;
        block += (uint32_t)blocks;
        packed += blocks * BITS;
        gmin += groups;
        gscale += groups;
    }
};
// The lane's own in it.
template <typename PLACE>
__device__ __forceinline__ uint32_t lane_block(const HeadArgs& a, const PLACE& at) { return at.row * (a.dim >> 3) + at.j; }
template <typename PLACE>
__device__ __forceinline__ uint32_t lane_group(const HeadArgs& a, const PLACE& at) {
    return a.groups_per_row ? at.row * a.groups_per_row + (at.d >> a.group_shift) : at.row >> a.row_shift;
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

// Leaves the context of a pass, whose elements v holds.
template <int BITS, typename PLACE>
__device__ __forceinline__ void compress_pass(const HeadArgs& a, const HeadPart& p, const PLACE& at, const Spot<BITS>& spot,
                                              uint32_t my_block, uint32_t my_group, bool active, const float (&v)[8]) {
    uint32_t r[4];
    // the high word of the block's number is the wavefront's, unless the low one wraps in this pass
    if (__builtin_expect((uint32_t)spot.block <= 0xFFFFFFFFu - 64u, 1))
        philox_head_uniform((uint32_t)spot.block + my_block,
                            PhiloxUniform((uint32_t)(spot.block >> 32), p.seed_lo, p.seed_hi), p.seed_lo, p.seed_hi, r);
    else philox_head_any((uint64_t)spot.block + my_block, p.seed_lo, p.seed_hi, r);
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
    store_codes<BITS>(spot.packed + my_block * BITS, codes);
    if ((at.lane & (a.group_lanes - 1)) == 0) {
        spot.gmin[my_group] = mn;
        spot.gscale[my_group] = step;
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
__device__ __forceinline__ uint32_t wave_of_block() { return (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// What a wavefront loads behind its last unit, for nothing, so that no load stands behind a branch: the part's first unit, which
// all take and a cache has, or, where arithmetic bounds the pass, its own once more.  Us, its own | the first: fp32, 8192 tokens
// of 16 + 16 heads of 64 25.8 | 23.2, of 4 + 4 of 256 27.9 | 25.5, backward 40 | 39; bf16, 8192 of 32 + 8 of 128 29.4 | 28.2; with
// 4-bit contexts, 65536 of 4 + 1 of 128 51 | 54, 13107 of 32 + 8 63 | 65, 16384 of 16 + 16 of 64 34.4 | 35.1.
template <int DT, int BITS>
__device__ __forceinline__ uint32_t behind_last(uint32_t unit) {
    return DT == GACT_DT_BF16 && BITS != 0 ? unit : 0;
}

template <int DT, int BITS, bool HALVES, int MODE>
__device__ __forceinline__ void heads_run(const HeadArgs& a, const HeadPart& p, uint32_t unit) {
    const Place<MODE> at(a);
    const uint32_t my_token = lane_token(p, steady(MODE), (uint32_t)at.row);
    typedef typename LaneOffset<MODE>::type Offset;
    const auto mine = [&](const HeadTensor& t) {
        return (Offset)((lane_first(p, t, steady(MODE), (uint32_t)at.row, my_token) + at.d) * kSize<DT>);
    };
    // a tensor's elements from `first` on: kAny adds them to the lane's offset instead
    const auto base = [&](const HeadTensor& t, int64_t first) { return (uint8_t*)t.p + (steady(MODE) ? first * kSize<DT> : 0); };
    const auto lane_at = [&](Offset lane, int64_t first) { return steady(MODE) ? lane : (Offset)(lane + first * kSize<DT>); };
    const Offset in_lane = mine(p.t[kIn]), out_lane = mine(p.t[kOut]);
    const int lanes = 1 << at.shift;
    const uint32_t my_group = BITS != 0 ? lane_group(a, at) : 0, my_block = lane_block(a, at);
    float w[8];
    at.weights(a, p, w);
    const Turn<HALVES> turn(a, at);
    Angles<HALVES> angles;
    const auto fetch = [&](int64_t from, uint32_t row) {
        Raw<DT> raw = {};
        if (at.holds(p, row)) raw = load8<DT>(base(p.t[kIn], from), lane_at(in_lane, from));
        return raw;
    };
    const uint32_t passes = steady(MODE) ? p.run : 1;
    const bool keep = p.rstd != nullptr;
    Unit<MODE, 2> u(a, p, at, unit);
    Raw<DT> ahead = fetch(u.first[kIn], unit * passes << (6 - at.shift));
    for (;;) {
        angles.load(a, p, turn, u, my_token);
        // a pass's elements are always on their way, without a branch, while the one before is worked on
        const uint32_t following = p.units - unit > p.waves ? unit + p.waves : behind_last<DT, BITS>(unit);
        const Unit<MODE, 2> next(a, p, at, following);
        int64_t in = u.first[kIn], out = u.first[kOut];
        Spot<BITS> spot(a, p, unit * passes, at.shift);
        for (uint32_t i = 1; i <= passes; ++i) {
            const Raw<DT> raw = ahead;
            in += p.t[kIn].pass;
            const bool last = i == passes;
            ahead = fetch(last ? next.first[kIn] : in, last ? following * passes << (6 - at.shift) : spot.row + (uint32_t)spot.rows);
            const bool active = at.holds(p, spot.row);
            float v[8], n[8], ss = 0.0f;
            widen8<DT>(raw, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                ss = __builtin_fmaf(v[k], v[k], ss);
                n[k] = v[k] * w[k];
            }
            angles.template turn<false>(n, turn);
            ss = add_over(ss, lanes);
            const float rstd = __builtin_amdgcn_rsqf(__builtin_fmaf(ss, a.inv_dim, a.eps));
#pragma unroll
            for (int k = 0; k < 8; ++k) n[k] *= rstd;
            if (active) store8<DT>(base(p.t[kOut], out), lane_at(out_lane, out), n);
            if (active && keep && at.j == 0) spot.rstd[(uint32_t)at.row] = rstd;
            if constexpr (BITS != 0) compress_pass<BITS>(a, p, at, spot, my_block, my_group, active, v);
            out += p.t[kOut].pass;
            spot.next();
        }
        if (following <= unit) return;
        unit = following;
        u = next;
    }
}

template <int DT, int BITS, bool HALVES, int MODE>
__global__ __launch_bounds__(kHeadThreads) void heads_kernel(HeadArgs a) {
    uint32_t block;
    const HeadPart& p = a.part[part_of(a, block)];
    const uint32_t unit = block * kHeadWaves + wave_of_block();
    if (unit >= p.units) return;
    if constexpr (BITS != 0)
        if (unit == 0) zero_pad<BITS>(a, p, (int)threadIdx.x);
    heads_run<DT, BITS, HALVES, MODE>(a, p, unit);
}

// x of eight elements from their codes.
template <int BITS>
__device__ __forceinline__ void decompress8(uint64_t codes, float mn, float step, float (&x)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        // a nibble of every byte of a word, so that the bytes convert in place
        const uint32_t word = BITS == 8 && k >= 4 ? (uint32_t)(codes >> 32) : (uint32_t)codes;
        const uint32_t q = BITS == 8 ? word >> (8 * (k & 3)) & 0xFFu
                         : BITS == 4 ? ((k & 1 ? word >> 4 : word) & 0x0F0F0F0Fu) >> (8 * (k >> 1)) & 0xFFu
                         : word >> (k * BITS) & ((1u << BITS) - 1u);
        const float t = (float)q * step;
        x[k] = t + mn;
    }
}

template <int DT, int BITS, bool HALVES, int MODE>
__device__ __forceinline__ void backward_run(const HeadArgs& a, const HeadPart& p, const Place<MODE>& at, uint32_t unit,
                                             float (&dw)[8]) {
    constexpr int kTensors = BITS == 0 ? 3 : 2;
    const uint32_t my_token = lane_token(p, steady(MODE), (uint32_t)at.row);
    typedef typename LaneOffset<MODE>::type Offset;
    const auto mine = [&](const HeadTensor& t) {
        return (Offset)((lane_first(p, t, steady(MODE), (uint32_t)at.row, my_token) + at.d) * kSize<DT>);
    };
    // a tensor's elements from `first` on: kAny adds them to the lane's offset instead
    const auto base = [&](const HeadTensor& t, int64_t first) { return (uint8_t*)t.p + (steady(MODE) ? first * kSize<DT> : 0); };
    const auto lane_at = [&](Offset lane, int64_t first) { return steady(MODE) ? lane : (Offset)(lane + first * kSize<DT>); };
    const Offset in_lane = mine(p.t[kIn]), out_lane = mine(p.t[kOut]);
    const Offset x_lane = BITS == 0 ? mine(p.t[kX]) : 0;
    const int lanes = 1 << at.shift;
    const uint32_t my_group = BITS != 0 ? lane_group(a, at) : 0, my_block = lane_block(a, at);
    float w[8];
    at.weights(a, p, w);
    const Turn<HALVES> turn(a, at);
    Angles<HALVES> angles;
    struct Input {
        Raw<DT> dy, x;
        uint64_t codes;
        float mn, step, rstd;
    };
    const auto fetch = [&](int64_t dy, int64_t x, const Spot<BITS>& from) {
        Input in = {};
        if (at.holds(p, from.row)) {
            in.dy = load8<DT>(base(p.t[kIn], dy), lane_at(in_lane, dy));
            in.rstd = from.rstd[(uint32_t)at.row];
            if constexpr (BITS != 0) {
                in.codes = load_codes<BITS>(from.packed + my_block * BITS);
                in.mn = from.gmin[my_group];
                in.step = from.gscale[my_group];
            } else {
                in.x = load8<DT>(base(p.t[kX], x), lane_at(x_lane, x));
            }
        }
        return in;
    };
    const uint32_t passes = steady(MODE) ? p.run : 1;
    Unit<MODE, kTensors> u(a, p, at, unit);
    Spot<BITS> spot(a, p, unit * passes, at.shift);
    Input ahead = fetch(u.first[kIn], u.first[kTensors - 1], spot);
    for (;;) {
        angles.load(a, p, turn, u, my_token);
        const uint32_t following = p.units - unit > p.waves ? unit + p.waves : behind_last<DT, BITS>(unit);
        const Unit<MODE, kTensors> next(a, p, at, following);
        const Spot<BITS> next_spot(a, p, following * passes, at.shift);
        int64_t dy = u.first[kIn], out = u.first[kOut], xs = u.first[kTensors - 1];
        for (uint32_t i = 1; i <= passes; ++i) {
            const Input in = ahead;
            const bool active = at.holds(p, spot.row);
            dy += p.t[kIn].pass;
            xs += p.t[kTensors - 1].pass;
            spot.next();
            const bool last = i == passes;
            if (last) spot = next_spot;
            ahead = fetch(last ? next.first[kIn] : dy, last ? next.first[kTensors - 1] : xs, spot);
            float dn[8], x[8], s = 0.0f;
            widen8<DT>(in.dy, dn);
            if constexpr (BITS != 0) decompress8<BITS>(in.codes, in.mn, in.step, x);
            else widen8<DT>(in.x, x);
            angles.template turn<true>(dn, turn);
            // r g and r mean(g x)
            float g[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                dn[k] *= in.rstd;
                g[k] = dn[k] * w[k];
                s = __builtin_fmaf(g[k], x[k], s);
            }
            s = add_over(s, lanes) * a.inv_dim * (in.rstd * in.rstd);
            if (active) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    dw[k] = __builtin_fmaf(dn[k], x[k], dw[k]);
                    g[k] = __builtin_fmaf(-x[k], s, g[k]);
                }
                store8<DT>(base(p.t[kOut], out), lane_at(out_lane, out), g);
            }
            out += p.t[kOut].pass;
        }
        if (following <= unit) return;
        unit = following;
        u = next;
    }
}

template <int DT, int BITS, bool HALVES, int MODE>
__global__ __launch_bounds__(kHeadThreads, head_backward_waves(DT)) void heads_backward_kernel(HeadArgs a) {
    __shared__ float lds[kHeadWaves][64 * 8];
    uint32_t block;
    const HeadPart& p = a.part[part_of(a, block)];
    const uint32_t unit = block * kHeadWaves + wave_of_block();
    const Place<MODE> at(a);
    float dw[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) dw[k] = 0.0f;
    if (unit < p.units) backward_run<DT, BITS, HALVES, MODE>(a, p, at, unit, dw);
    if (!p.partial) return;
    // over the wavefront's rows, then over the block's wavefronts
    float* mine = lds[threadIdx.x >> 6];
#pragma unroll
    for (int k = 0; k < 8; ++k) mine[k * 64 + at.lane] = dw[k];
    __syncthreads();
    const int lanes = 1 << at.shift, rows = 64 >> at.shift;
    for (int d = (int)threadIdx.x; d < a.dim; d += kHeadThreads) {
        float sum = 0.0f;
        for (int v = 0; v < kHeadWaves; ++v)
            for (int c = 0; c < rows; ++c) sum += lds[v][(d & 7) * 64 + c * lanes + (d >> 3)];
        p.partial[(size_t)block * a.dim + d] = sum;
    }
}

// dw of one part: its blocks' sums, eight elements a block of 8 x 128 threads, added in binary64 and in a fixed order.
constexpr int kDwColumns = 8, kDwRows = 128, kDwThreads = kDwColumns * kDwRows;
__global__ __launch_bounds__(kDwThreads) void heads_dw_kernel(HeadArgs a) {
    __shared__ double lds[kDwThreads / 64][kDwColumns];
    const HeadPart& p = a.part[blockIdx.y];
    if (!p.dw) return;
    const int col = threadIdx.x % kDwColumns, row = threadIdx.x / kDwColumns, d = blockIdx.x * kDwColumns + col;
    constexpr int kEach = (int)(kHeadBackwardBlocks + kDwRows - 1) / kDwRows;
    float v[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const uint32_t i = (uint32_t)(k * kDwRows + row);
        v[k] = i < p.blocks ? p.partial[i * (uint32_t)a.dim + (uint32_t)d] : 0.0f;
    }
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) sum += (double)v[k];
#pragma unroll
    for (int m = 32; m >= kDwColumns; m >>= 1) sum += __shfl_xor(sum, m);
    if ((threadIdx.x & 63) < kDwColumns) lds[threadIdx.x >> 6][col] = sum;
    __syncthreads();
    if (threadIdx.x >= kDwColumns) return;
    sum = 0.0;
#pragma unroll
    for (int k = 0; k < kDwThreads / 64; ++k) sum += lds[k][threadIdx.x];
    if (a.w_f32) ((float*)p.dw)[d] = (float)sum;
    else ((uint16_t*)p.dw)[d] = (uint16_t)bf16_pair_rne((float)sum, 0.0f);
}

// ------------------------------------------------------------- host launchers
template <int DT, int BITS, bool HALVES, int MODE>
static void launch(bool backward, const HeadArgs& a, unsigned blocks, hipStream_t s) {
    if (backward) hipLaunchKernelGGL((heads_backward_kernel<DT, BITS, HALVES, MODE>), dim3(blocks), dim3(kHeadThreads), 0, s, a);
    else hipLaunchKernelGGL((heads_kernel<DT, BITS, HALVES, MODE>), dim3(blocks), dim3(kHeadThreads), 0, s, a);
}
template <int DT, int BITS, bool HALVES>
static void launch_mode(bool backward, const HeadArgs& a, int mode, unsigned blocks, hipStream_t s) {
    switch (mode) {
        case kAny: launch<DT, BITS, HALVES, kAny>(backward, a, blocks, s); break;
        case kSteady: launch<DT, BITS, HALVES, kSteady>(backward, a, blocks, s); break;
        case 3: launch<DT, BITS, HALVES, 3>(backward, a, blocks, s); break;
        case 4: launch<DT, BITS, HALVES, 4>(backward, a, blocks, s); break;
        default: launch<DT, BITS, HALVES, 5>(backward, a, blocks, s); break;
    }
}
template <int DT, bool HALVES>
static void launch_bits(bool backward, const HeadArgs& a, int mode, int bits, unsigned blocks, hipStream_t s) {
    switch (bits) {
        case 0: launch_mode<DT, 0, HALVES>(backward, a, mode, blocks, s); break;
        case 1: launch_mode<DT, 1, HALVES>(backward, a, mode, blocks, s); break;
        case 2: launch_mode<DT, 2, HALVES>(backward, a, mode, blocks, s); break;
        case 4: launch_mode<DT, 4, HALVES>(backward, a, mode, blocks, s); break;
        default: launch_mode<DT, 8, HALVES>(backward, a, mode, blocks, s); break;
    }
}
static int launch_any(bool backward, const HeadArgs& a, int mode, int dtype, int bits, int halves, hipStream_t s) {
    const unsigned blocks = a.part[0].blocks + a.part[1].blocks;
    if (dtype == GACT_DT_F32) {
        if (halves) launch_bits<GACT_DT_F32, true>(backward, a, mode, bits, blocks, s);
        else launch_bits<GACT_DT_F32, false>(backward, a, mode, bits, blocks, s);
    } else {
        if (halves) launch_bits<GACT_DT_BF16, true>(backward, a, mode, bits, blocks, s);
        else launch_bits<GACT_DT_BF16, false>(backward, a, mode, bits, blocks, s);
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace gact

extern "C" int gact_launch_heads(const gact::HeadArgs* a, int mode, int dtype, int bits, int halves, int backward, void* stream) {
    return gact::launch_any(backward != 0, *a, mode, dtype, bits, halves, (hipStream_t)stream);
}

extern "C" int gact_launch_heads_dw(const gact::HeadArgs* a, int parts, void* stream) {
    hipLaunchKernelGGL(gact::heads_dw_kernel, dim3(a->dim / gact::kDwColumns, parts), dim3(gact::kDwThreads), 0, (hipStream_t)stream, *a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}
