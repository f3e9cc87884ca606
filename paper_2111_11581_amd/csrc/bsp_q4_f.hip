// k_q4 for fp32 activations.
#include <hip/hip_runtime.h>

#include "bsp_q4_mm.h"

namespace bsp {
hipError_t q4_linear_f32(const Q4Args &a, hipStream_t st) { return q4_linear<float>(a, st); }
}  // namespace bsp
