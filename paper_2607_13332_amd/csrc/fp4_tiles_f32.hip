// The 4-bit cache's tile kernel (and with it the rows kernel, where a batch has
// both) for queries and outputs in float32.
#include "fp4_attn_kernels.h"

namespace ssn {

hipError_t launch_fp4_tiles_f32(const Fp4AttnArgs& f, const AttnPlan& p, hipStream_t st) {
  if (f.a.D <= 64) return SSN_FP4_EXACT(launch_fp4_tiles, float, 64, 1);
  if (f.a.D <= 128) return SSN_FP4_EXACT(launch_fp4_tiles, float, 128, 1);
  return SSN_FP4_EXACT(launch_fp4_tiles, float, 256, 1);
}

}  // namespace ssn
