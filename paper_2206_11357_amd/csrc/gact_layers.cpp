// Entry points of layers whose context is read as codes (include/gact.h): argument checks and launch plans.  The kernels
// are in gact_weight.hip and gact_group_norm.hip.
#include <hip/hip_runtime.h>

#include <cmath>

#include "gact.h"
#include "gact_device.h"
#include "gact_group_norm.h"
#include "gact_weight.h"

namespace {

bool bits_ok(int bits) { return bits == 1 || bits == 2 || bits == 4 || bits == 8; }
bool group_ok(int g) { return g >= 32 && g <= 1024 && g % 32 == 0; }
bool dtype_ok(int dt) { return dt == GACT_F32 || dt == GACT_BF16; }
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t size_of(int dt) { return dt == GACT_F32 ? 4 : 2; }

constexpr int64_t kMost = 0x7FFFFFFFll;

bool weight_sizes_ok(int64_t T, int64_t N, int64_t K) {
    if (T < 0 || N < 0 || K < 0 || T > kMost || N >= 1 << 28 || K >= 1 << 22) return false;
    return (uint64_t)T * (uint64_t)K < 1ull << 34 && (uint64_t)N * (uint64_t)K < 1ull << 34;
}

// -------------------------------------------------------------------- group norm
bool norm_sizes_ok(int64_t B, int64_t P, int C, int H) {
    if (B < 0 || P < 0 || B > kMost || P > kMost || C < 8 || C % 8 != 0 || C > 1 << 20 || H < 1 || C % H != 0) return false;
    return (uint64_t)B * (uint64_t)P <= (uint64_t)kMost && (uint64_t)B * (uint64_t)C < 1ull << 30 &&
           (uint64_t)B * (uint64_t)P * (uint64_t)C < 1ull << 34;
}
void norm_sizes(int64_t B, int64_t P, int C, int H, int dtype, gact::GnArgs* a) {
    a->B = (uint32_t)B;
    a->P = (uint32_t)P;
    a->C = (uint32_t)C;
    a->H = (uint32_t)H;
    a->D = (uint32_t)(C / H);
    gact::plan_group_norm(a, dtype);
}

// Whether two pixels of a tensor can share memory: unless, in the order of their sizes, each stride passes what lies below it.
bool pixels_overlap(const int64_t (&stride)[2], const gact_channel_norm* h) {
    const auto size = [](int64_t v) { return v < 0 ? 0 - (uint64_t)v : (uint64_t)v; };
    uint64_t s[2] = {size(stride[0]), size(stride[1])}, n[2] = {(uint64_t)h->batch, (uint64_t)h->pixels};
    const int low = s[0] < s[1] ? 0 : 1;
    uint64_t extent = (uint64_t)h->channels;
    for (const int k : {low, 1 - low}) {
        if (n[k] < 2) continue;
        if (s[k] < extent || s[k] >= (uint64_t)1 << 48) return true;               // (behind that products would wrap)
        extent += s[k] * (n[k] - 1);
    }
    return false;
}
bool same_strides(const int64_t (&a)[2], const int64_t (&b)[2], const gact_channel_norm* h) {
    return (a[0] == b[0] || h->batch < 2) && (a[1] == b[1] || h->pixels < 2);
}
// Whether an output is another of the call's buffers, as far as pointers and strides show it.
bool norm_overlaps(const gact_channel_norm* h, bool backward, bool compressed) {
    const void* out = backward ? h->dx : h->y;
    const void* in = backward ? h->dy : h->x;
    const auto& out_stride = backward ? h->dx_stride : h->y_stride;
    const auto& in_stride = backward ? h->dy_stride : h->x_stride;
    if (pixels_overlap(out_stride, h)) return true;
    if (out == in && !same_strides(out_stride, in_stride, h)) return true;
    const void* others[] = {h->w, h->b, h->mean, h->rstd, compressed ? h->packed : nullptr, compressed ? (const void*)h->gmin : nullptr,
                            compressed ? (const void*)h->gscale : nullptr, backward ? h->dw : nullptr, backward ? h->db : nullptr,
                            backward && !compressed ? h->x : nullptr};
    for (const void* p : others) if (p && p == out) return true;
    if (backward) {
        for (const void* p : {(const void*)h->dw, (const void*)h->db})
            if (p && (p == h->w || p == h->b || p == h->mean || p == h->rstd || p == h->dy)) return true;
        return h->dw && h->dw == h->db;
    }
    return (h->mean && h->mean == h->rstd) || (compressed && (h->packed == h->gmin || h->packed == h->gscale || h->gmin == h->gscale));
}

// Checks a call; fills *a, *bits (0 without a context) and *whole (plan_whole).
int stage_norm(const gact_channel_norm* h, bool backward, void* ws, size_t ws_bytes, gact::GnArgs* a, int* bits, int* whole) {
    if (!h) return GACT_E_ARG;
    if (h->bits != GACT_BITS_UNCOMPRESSED && !bits_ok(h->bits)) return GACT_E_BITS;
    *bits = h->bits == GACT_BITS_UNCOMPRESSED ? 0 : h->bits;
    if (!dtype_ok(h->dtype) || !dtype_ok(h->w_dtype) || (h->act != GACT_ACT_NONE && h->act != GACT_ACT_SILU)) return GACT_E_ARG;
    if (!norm_sizes_ok(h->batch, h->pixels, h->channels, h->groups)) return GACT_E_ARG;
    if (!backward && !(std::isnormal(h->eps) && h->eps > 0.0f)) return GACT_E_ARG;
    const int G = h->group_size;
    if (*bits != 0 && (G < 32 || G > 512 || (G & (G - 1)) != 0)) return GACT_E_GROUP;
    const size_t size = size_of(h->dtype), w_size = size_of(h->w_dtype);
    if (!aligned(h->w, w_size) || !aligned(h->b, w_size)) return GACT_E_ARG;
    if (backward && ((h->dw && (!h->w || !aligned(h->dw, w_size))) || (h->db && (!h->b || !aligned(h->db, w_size))))) return GACT_E_ARG;
    const bool empty = h->batch == 0 || h->pixels == 0;
    if (!empty) {
        const void* in = backward ? h->dy : h->x;
        const void* out = backward ? h->dx : h->y;
        if (!in || !out || !aligned(in, size) || !aligned(out, size) || !aligned(h->mean, 4) || !aligned(h->rstd, 4)) return GACT_E_ARG;
        if (!h->mean != !h->rstd || (!h->mean && (backward || *bits != 0))) return GACT_E_ARG;
        if (backward && *bits == 0 && (!h->x || !aligned(h->x, size))) return GACT_E_ARG;
        if (*bits != 0 && (!h->packed || !h->gmin || !h->gscale || !aligned(h->packed, 16) || !aligned(h->gmin, 4) ||
                           !aligned(h->gscale, 4)))
            return GACT_E_ARG;
        if (norm_overlaps(h, backward, *bits != 0)) return GACT_E_ARG;
    }
    const auto tensor = [](const void* p, const int64_t (&stride)[2]) {
        return gact::GnTensor{const_cast<void*>(p), stride[0], stride[1]};
    };
    a->x = tensor(h->x, h->x_stride);
    a->y = tensor(h->y, h->y_stride);
    a->dy = tensor(h->dy, h->dy_stride);
    a->dx = tensor(h->dx, h->dx_stride);
    a->w = h->w;
    a->b = h->b;
    a->dw = h->dw;
    a->db = h->db;
    a->mean = h->mean;
    a->rstd = h->rstd;
    a->packed = (uint8_t*)h->packed;
    a->gmin = h->gmin;
    a->gscale = h->gscale;
    a->seed_lo = (uint32_t)h->seed;
    a->seed_hi = (uint32_t)(h->seed >> 32);
    a->eps = h->eps;
    a->w_f32 = h->w_dtype == GACT_F32;
    if (empty) {
        a->C = (uint32_t)h->channels;
        return GACT_OK;
    }
    if (*bits != 0) while ((8 << a->block_shift) < G) ++a->block_shift;
    norm_sizes(h->batch, h->pixels, h->channels, h->groups, h->dtype, a);
    *whole = gact::plan_whole(a, h->dtype, backward, gact::gn_held(h->dtype, *bits, h->act == GACT_ACT_SILU));
    // (4096: workgroups that compress, and those that add dw)
    const uint64_t B = a->B;
    if (*whole ? !gact::launchable(B * a->unit_slabs + 4096, gact::kGnWhole[*whole - 1].threads)
               : !gact::launchable(B * a->chunks * a->slabs + a->C / 32 + 1, gact::kGnThreads) ||
                     !gact::launchable(B * a->H * a->slices, gact::kGnThreads))
        return GACT_E_ARG;
    uint8_t* at = (uint8_t*)ws;
    const size_t need = backward ? gact::gn_backward_bytes(*a, *whole) : gact::gn_forward_bytes(*a, *whole);
    if (need > 0 && (!at || !aligned(at, 16) || ws_bytes < need)) return GACT_E_ARG;
    if (*whole) {
        a->sums = (float*)at;
        return GACT_OK;
    }
    a->partial = (float*)at;
    at += gact::gn_partial_bytes(*a);
    if (backward) {
        a->sums = (float*)at;
        a->means = (float*)(at + gact::gn_sums_bytes(*a));
    } else if (!a->mean) {
        a->mean = (float*)at;
        a->rstd = (float*)(at + gact::gn_align((size_t)a->B * a->H * sizeof(float)));
    }
    return GACT_OK;
}

}  // namespace

extern "C" {

size_t gact_group_norm_workspace_bytes(int64_t batch, int64_t pixels, int channels, int groups, gact_dtype dtype, int backward) {
    if (!norm_sizes_ok(batch, pixels, channels, groups) || !dtype_ok((int)dtype) || batch == 0 || pixels == 0) return 0;
    gact::GnArgs a{};
    norm_sizes(batch, pixels, channels, groups, (int)dtype, &a);
    const int whole = gact::plan_whole(&a, (int)dtype, backward != 0, false);
    return backward ? gact::gn_backward_bytes(a, whole) : gact::gn_forward_bytes(a, whole);
}

int gact_group_norm(const gact_channel_norm* h_norm, void* d_workspace, size_t workspace_bytes, void* stream) {
    gact::GnArgs a{};
    int bits = 0, whole = 0;
    if (const int rc = stage_norm(h_norm, false, d_workspace, workspace_bytes, &a, &bits, &whole)) return rc;
    if (a.B == 0) return GACT_OK;
    return gact_launch_group_norm(&a, h_norm->dtype, bits, h_norm->act, whole, stream) == 0 ? GACT_OK : GACT_E_HIP;
}

int gact_group_norm_backward(const gact_channel_norm* h_norm, void* d_workspace, size_t workspace_bytes, void* stream) {
    gact::GnArgs a{};
    int bits = 0, whole = 0;
    if (const int rc = stage_norm(h_norm, true, d_workspace, workspace_bytes, &a, &bits, &whole)) return rc;
    if (a.B == 0) {                                     // nothing to add: the sums are zero
        if (!a.dw && !a.db) return GACT_OK;
        return gact_launch_group_norm_zero(&a, stream) == 0 ? GACT_OK : GACT_E_HIP;
    }
    return gact_launch_group_norm_backward(&a, h_norm->dtype, bits, h_norm->act, whole, stream) == 0 ? GACT_OK : GACT_E_HIP;
}

size_t gact_linear_weight_grad_workspace_bytes(int64_t tokens, int64_t out_features, int64_t in_features, gact_dtype dtype) {
    if (!weight_sizes_ok(tokens, out_features, in_features) || !dtype_ok((int)dtype)) return 0;
    const uint64_t T = (uint64_t)tokens, N = (uint64_t)out_features, K = (uint64_t)in_features;
    if (N == 0) return 0;
    return gact::weight_workspace_bytes(gact::plan_weight(T, N, K, (int)dtype), N, K);
}

int gact_linear_weight_grad(const gact_linear_grad* h_grad, void* d_workspace, size_t workspace_bytes, void* stream) {
    if (!h_grad) return GACT_E_ARG;
    const gact_linear_grad& h = *h_grad;
    if (!bits_ok(h.bits)) return GACT_E_BITS;
    if (!group_ok(h.group_size)) return GACT_E_GROUP;
    if (!dtype_ok(h.dtype) || !dtype_ok(h.w_dtype) || !weight_sizes_ok(h.tokens, h.out_features, h.in_features)) return GACT_E_ARG;
    const uint64_t T = (uint64_t)h.tokens, N = (uint64_t)h.out_features, K = (uint64_t)h.in_features;
    if (N == 0 || (K == 0 && !h.db)) return GACT_OK;
    const size_t w_size = size_of(h.w_dtype);
    if (!aligned(h.db, w_size) || (K > 0 && (!h.dw || !aligned(h.dw, w_size) || h.dw == h.db))) return GACT_E_ARG;
    if (T > 0 && (!h.dy || !aligned(h.dy, size_of(h.dtype)) || h.dy == h.dw || h.dy == h.db)) return GACT_E_ARG;
    if (T * K > 0 && (!h.packed || !h.gmin || !h.gscale || !aligned(h.packed, 16) || !aligned(h.gmin, 4) || !aligned(h.gscale, 4)))
        return GACT_E_ARG;
    const gact::WeightPlan plan = gact::plan_weight(T, N, K, h.dtype);
    const gact::WeightTile tile = gact::weight_tile(h.dtype, plan.form);
    const uint64_t blocks = (uint64_t)plan.tiles_n * plan.tiles_k * plan.splits;
    if (!gact::launchable(blocks, (uint32_t)tile.threads) ||
        (plan.splits > 1 && !gact::launchable((N * K + N) * (uint64_t)gact::join_parts(plan.splits) / 1024 + 2, 256)))
        return GACT_E_ARG;
    const size_t need = gact::weight_workspace_bytes(plan, N, K);
    if (need > 0 && (!d_workspace || !aligned(d_workspace, 16) || workspace_bytes < need)) return GACT_E_ARG;
    gact::WeightArgs a{};
    a.dy = (const uint8_t*)h.dy;
    a.packed = (const uint8_t*)h.packed;
    a.gmin = h.gmin;
    a.gscale = h.gscale;
    a.dw = h.dw;
    a.db = h.db;
    if (plan.splits > 1) {
        a.partial = (float*)d_workspace;
        a.db_partial = (float*)((uint8_t*)d_workspace + gact::weight_partial_bytes(plan, N, K));
    }
    a.dy_stride = h.dy_stride;
    a.T = (uint32_t)T;
    a.N = (uint32_t)N;
    a.K = (uint32_t)K;
    const uint64_t words = (T * K * (uint64_t)h.bits + 127) / 128 * 4;
    a.last_word = words ? words - 1 : 0;
    a.last_group = T * K ? (uint32_t)((T * K - 1) / (uint64_t)h.group_size) : 0;
    a.group = (uint32_t)h.group_size;
    a.by_group = gact::divisor((uint32_t)h.group_size / 32);
    a.tiles_n = plan.tiles_n;
    a.tiles_k = plan.tiles_k;
    a.splits = plan.splits;
    a.chunks = plan.chunks;
    a.db_every = plan.db_every;
    const uint32_t BT = (uint32_t)tile.tokens;
    a.dy_chunk = BT * (uint32_t)h.dy_stride * (uint32_t)size_of(h.dtype);
    a.code_chunk = BT * a.K / 8 * (uint32_t)h.bits;
    a.group_chunk = BT * a.K / a.group * 4;
    a.w_f32 = h.w_dtype == GACT_F32;
    return gact_launch_weight(&a, plan.form, h.dtype, h.bits, stream) == 0 ? GACT_OK : GACT_E_HIP;
}

}  // extern "C"
