// The weight gradient's kernels for fp32 dy (gact_weight_kernel.h).
#include "gact_weight_kernel.h"

extern "C" int gact_launch_weight_f32(const gact::WeightArgs* a, int form, int bits, void* stream) {
    return gact::launch_type<GACT_DT_F32>(*a, form, bits, (hipStream_t)stream);
}
