// k_q4 for bf16 activations.
#include <hip/hip_runtime.h>

#include "bsp_q4_mm.h"

namespace bsp {
hipError_t q4_linear_bf16(const Q4Args &a, hipStream_t st) { return q4_linear<uint16_t>(a, st); }
}  // namespace bsp
