// The paged attention's tile kernel (and with it the rows kernel, where a batch
// has both) for f32 storage.
#include "attn_kernels.h"

namespace ssn {

hipError_t launch_attn_tiles_f32(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  if (a.D <= 64) return SSN_ATTN_EXACT(launch_tiles, float, 64, 1);
  if (a.D <= 128) return SSN_ATTN_EXACT(launch_tiles, float, 128, 1);
  return SSN_ATTN_EXACT(launch_tiles, float, 256, 1);
}

}  // namespace ssn
