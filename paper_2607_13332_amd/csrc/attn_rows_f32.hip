// The paged attention's rows kernel for f32 storage.
#include "attn_kernels.h"

namespace ssn {

hipError_t launch_attn_rows_f32(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  const bool one = p.rows.blocks == 1;
  if (a.D <= 64) return one ? SSN_ATTN_EXACT(launch_rows, float, 64, 1) : SSN_ATTN_EXACT(launch_rows, float, 64, 2);
  if (a.D <= 128) return one ? SSN_ATTN_EXACT(launch_rows, float, 128, 1) : SSN_ATTN_EXACT(launch_rows, float, 128, 2);
  return SSN_ATTN_EXACT(launch_rows, float, 256, 1);
}

}  // namespace ssn
