// The paged attention's rows kernel for f32 storage.
#include "attn_rows.h"

namespace ssn {

hipError_t launch_attn_rows_f32(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  const bool one = p.rows.blocks == 1;
  if (a.D <= 64) return one ? launch_rows<float, 64, 1>(a, p, st) : launch_rows<float, 64, 2>(a, p, st);
  if (a.D <= 128) return one ? launch_rows<float, 128, 1>(a, p, st) : launch_rows<float, 128, 2>(a, p, st);
  return launch_rows<float, 256, 1>(a, p, st);
}

}  // namespace ssn
