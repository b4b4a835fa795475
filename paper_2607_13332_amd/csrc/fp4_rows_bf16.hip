// The 4-bit cache's rows kernel for queries and outputs in bf16.
#include "fp4_attn_kernels.h"

namespace ssn {

hipError_t launch_fp4_rows_bf16(const Fp4AttnArgs& f, const AttnPlan& p, hipStream_t st) {
  const bool one = p.rows.blocks == 1;
  if (f.a.D <= 64)
    return one ? SSN_FP4_EXACT(launch_fp4_rows, uint16_t, 64, 1) : SSN_FP4_EXACT(launch_fp4_rows, uint16_t, 64, 2);
  if (f.a.D <= 128)
    return one ? SSN_FP4_EXACT(launch_fp4_rows, uint16_t, 128, 1) : SSN_FP4_EXACT(launch_fp4_rows, uint16_t, 128, 2);
  return SSN_FP4_EXACT(launch_fp4_rows, uint16_t, 256, 1);
}

}  // namespace ssn
