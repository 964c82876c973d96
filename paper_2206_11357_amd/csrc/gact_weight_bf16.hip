// The weight gradient's kernels for bf16 dy (gact_weight_kernel.h).
#include "gact_weight_kernel.h"

extern "C" int gact_launch_weight_bf16(const gact::WeightArgs* a, int form, int bits, void* stream) {
    return gact::launch_type<GACT_DT_BF16>(*a, form, bits, (hipStream_t)stream);
}
