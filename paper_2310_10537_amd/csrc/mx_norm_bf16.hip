// RMS norm of bf16 rows, every output form (mx_norm_fwd.hpp).
#include "mx_norm_fwd.hpp"

namespace mx {

hipError_t launch_norm_bf16(const NormArgs &a, int out, hipStream_t st)
{
    switch (out) {
        case FP8_E4M3: return launch_norm_t<FP8_E4M3, DT_BF16>(a, st);
        case FP8_E5M2: return launch_norm_t<FP8_E5M2, DT_BF16>(a, st);
        case FP6_E3M2: return launch_norm_t<FP6_E3M2, DT_BF16>(a, st);
        case FP6_E2M3: return launch_norm_t<FP6_E2M3, DT_BF16>(a, st);
        case FP4_E2M1: return launch_norm_t<FP4_E2M1, DT_BF16>(a, st);
        case INT8: return launch_norm_t<INT8, DT_BF16>(a, st);
        case OUT_B128_E4M3: return launch_norm_t<OUT_B128_E4M3, DT_BF16>(a, st);
        case OUT_B128_E5M2: return launch_norm_t<OUT_B128_E5M2, DT_BF16>(a, st);
        default: return launch_norm_t<OUT_NONE, DT_BF16>(a, st);
    }
}

}  // namespace mx
