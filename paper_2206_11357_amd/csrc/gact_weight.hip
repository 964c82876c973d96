// Second launch of the weight gradient: the splits' sums (gact_weight_kernel.h has the first).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gact_codec.h"
#include "gact_device.h"
#include "gact_weight.h"

namespace gact {

typedef float wf4 __attribute__((ext_vector_type(4)));

// dW and db from the splits' sums.  A workgroup takes 1024 / PARTS neighbouring elements of dW, four a thread, and each
// PARTS-th of the splits goes to one of its PARTS parts, whose sums are added in their order; the workgroups behind them add db
// likewise, a thread an element.  Many splits are those of a small dW, whose elements alone would not fill the GPU.
constexpr int kJoinThreads = 256;
__device__ __forceinline__ void put_weight(void* p, int f32, size_t i, float v) {
    if (f32) ((float*)p)[i] = v;
    else ((uint16_t*)p)[i] = (uint16_t)bf16_pair_rne(v, 0.0f);
}
template <int PARTS>
__global__ __launch_bounds__(kJoinThreads) void weight_join_kernel(WeightArgs a, uint32_t dw_blocks) {
    constexpr uint32_t kEach = kJoinThreads / PARTS;
    __shared__ wf4 lds[PARTS][kEach];
    const uint32_t part = threadIdx.x / kEach, j = threadIdx.x % kEach;
    const bool of_db = blockIdx.x >= dw_blocks;
    const size_t n = of_db ? a.N : (size_t)a.N * a.K;
    const size_t i = ((size_t)(of_db ? blockIdx.x - dw_blocks : blockIdx.x) * kEach + j) * 4;
    const float* from = of_db ? a.db_partial : a.partial;
    const uint32_t terms = of_db ? a.splits * a.db_every : a.splits;
    wf4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (i < n) {
        if (n % 4 == 0) {
#pragma unroll 8
            for (uint32_t k = part; k < terms; k += PARTS) {
                const wf4 v = *(const wf4*)(from + k * n + i);
#pragma unroll
                for (int c = 0; c < 4; ++c) s[c] += v[c];
            }
        } else {
            for (uint32_t k = part; k < terms; k += PARTS)
#pragma unroll
                for (int c = 0; c < 4; ++c) s[c] += i + c < n ? from[k * n + i + c] : 0.0f;
        }
    }
    if (PARTS > 1) {
        lds[part][j] = s;
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int k = 1; k < PARTS; ++k)
#pragma unroll
            for (int c = 0; c < 4; ++c) s[c] += lds[k][j][c];
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (i + c < n) put_weight(of_db ? a.db : a.dw, a.w_f32, i + c, s[c]);
}

}  // namespace gact

extern "C" int gact_launch_weight(const gact::WeightArgs* a, int form, int dtype, int bits, void* stream) {
    const int rc = dtype == GACT_DT_F32 ? gact_launch_weight_f32(a, form, bits, stream) : gact_launch_weight_bf16(a, form, bits, stream);
    if (rc != 0) return rc;
    if (a->splits > 1) {
        const int parts = gact::join_parts(a->splits);
        const uint64_t n = (uint64_t)a->N * a->K, each = 4 * gact::kJoinThreads / parts;
        const uint32_t dw_blocks = (uint32_t)((n + each - 1) / each);
        const uint32_t db_blocks = a->db ? (uint32_t)((a->N + each - 1) / each) : 0;
        const dim3 grid(dw_blocks + db_blocks), block(gact::kJoinThreads);
        switch (parts) {
            case 1: hipLaunchKernelGGL(gact::weight_join_kernel<1>, grid, block, 0, (hipStream_t)stream, *a, dw_blocks); break;
            case 4: hipLaunchKernelGGL(gact::weight_join_kernel<4>, grid, block, 0, (hipStream_t)stream, *a, dw_blocks); break;
            default: hipLaunchKernelGGL(gact::weight_join_kernel<16>, grid, block, 0, (hipStream_t)stream, *a, dw_blocks); break;
        }
        if (hipGetLastError() != hipSuccess) return -1;
    }
    return 0;
}
