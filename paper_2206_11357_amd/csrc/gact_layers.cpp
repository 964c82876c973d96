// Entry points of layers whose context is read as codes (include/gact.h): argument checks and launch plans.  The kernels
// are in gact_weight.hip.
#include <hip/hip_runtime.h>

#include "gact.h"
#include "gact_device.h"
#include "gact_weight.h"

namespace {

bool bits_ok(int bits) { return bits == 1 || bits == 2 || bits == 4 || bits == 8; }
bool group_ok(int g) { return g >= 32 && g <= 1024 && g % 32 == 0; }
bool dtype_ok(int dt) { return dt == GACT_F32 || dt == GACT_BF16; }
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t size_of(int dt) { return dt == GACT_F32 ? 4 : 2; }

constexpr int64_t kMost = 0x7FFFFFFFll;

bool weight_sizes_ok(int64_t T, int64_t N, int64_t K) {
    if (T < 0 || N < 0 || K < 0 || T > kMost || N > kMost || K > kMost) return false;
    return (uint64_t)T * (uint64_t)K < 1ull << 35 && (uint64_t)N * (uint64_t)K < 1ull << 38;
}

}  // namespace

extern "C" {

size_t gact_linear_weight_grad_workspace_bytes(int64_t tokens, int64_t out_features, int64_t in_features, gact_dtype dtype) {
    if (!weight_sizes_ok(tokens, out_features, in_features) || !dtype_ok((int)dtype)) return 0;
    const uint64_t T = (uint64_t)tokens, N = (uint64_t)out_features, K = (uint64_t)in_features;
    if (N == 0) return 0;
    return gact::weight_workspace_bytes(gact::plan_weight(T, N, K, (int)dtype), N, K);
}

int gact_linear_weight_grad(const void* d_dy, int64_t dy_stride, gact_dtype dtype, int64_t tokens, int64_t out_features,
                            int64_t in_features, const void* d_packed, const float* d_gmin, const float* d_gscale,
                            int group_size, int bits, void* d_dw, void* d_db, gact_dtype w_dtype, void* d_workspace,
                            size_t workspace_bytes, void* stream) {
    if (!bits_ok(bits)) return GACT_E_BITS;
    if (!group_ok(group_size)) return GACT_E_GROUP;
    if (!dtype_ok((int)dtype) || !dtype_ok((int)w_dtype) || !weight_sizes_ok(tokens, out_features, in_features)) return GACT_E_ARG;
    const uint64_t T = (uint64_t)tokens, N = (uint64_t)out_features, K = (uint64_t)in_features;
    if (N == 0 || (K == 0 && !d_db)) return GACT_OK;
    const size_t w_size = size_of(w_dtype);
    if (!aligned(d_db, w_size) || (K > 0 && (!d_dw || !aligned(d_dw, w_size) || d_dw == d_db))) return GACT_E_ARG;
    if (T > 0 && (!d_dy || !aligned(d_dy, size_of(dtype)))) return GACT_E_ARG;
    if (T * K > 0 && (!d_packed || !d_gmin || !d_gscale || !aligned(d_packed, 16) || !aligned(d_gmin, 4) || !aligned(d_gscale, 4)))
        return GACT_E_ARG;
    const gact::WeightPlan plan = gact::plan_weight(T, N, K, (int)dtype);
    const uint64_t blocks = (uint64_t)plan.tiles_n * plan.tiles_k * plan.splits;
    if (!gact::launchable(blocks, gact::kWeightThreads)) return GACT_E_ARG;
    const size_t need = gact::weight_workspace_bytes(plan, N, K);
    if (need > 0 && (!d_workspace || !aligned(d_workspace, 16) || workspace_bytes < need)) return GACT_E_ARG;
    gact::WeightArgs a{};
    a.dy = (const uint8_t*)d_dy;
    a.packed = (const uint8_t*)d_packed;
    a.gmin = d_gmin;
    a.gscale = d_gscale;
    a.dw = d_dw;
    a.db = d_db;
    if (plan.splits > 1) {
        a.partial = (float*)d_workspace;
        a.db_partial = (float*)((uint8_t*)d_workspace + gact::weight_partial_bytes(plan, N, K));
    }
    a.dy_stride = dy_stride;
    a.T = (uint32_t)T;
    a.N = (uint32_t)N;
    a.K = (uint32_t)K;
    const uint64_t words = (T * K * (uint64_t)bits + 127) / 128 * 4;
    a.last_word = words ? words - 1 : 0;
    a.last_group = T * K ? (uint32_t)((T * K - 1) / (uint64_t)group_size) : 0;
    a.group = (uint32_t)group_size;
    a.by_group = gact::divisor((uint32_t)group_size / 32);
    a.tiles_n = plan.tiles_n;
    a.tiles_k = plan.tiles_k;
    a.splits = plan.splits;
    a.chunks = plan.chunks;
    a.db_every = plan.db_every;
    a.w_f32 = w_dtype == GACT_F32;
    return gact_launch_weight(&a, plan.which, (int)dtype, bits, stream) == 0 ? GACT_OK : GACT_E_HIP;
}

}  // extern "C"
