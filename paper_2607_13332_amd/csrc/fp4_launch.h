// Launchers of the 4-bit cache's kernels; the C ABI in fp4_api.hip validates
// arguments and then calls these.
#pragma once

#include "attn_launch.h"

namespace ssn {

constexpr int kFp4Group = 32;          // elements that share a scale

// Codes [npages, Hk, page_size, D / 2] and scales [npages, Hk, page_size, D / 32].
struct Fp4Cache {
  uint8_t *Kc, *Ks, *Vc, *Vs;
};

hipError_t launch_kv_append_fp4(int dtype, const PagedBatch& pb, const NormRope& nr, HeadRows q, HeadRows k,
                                HeadRows v, const void* wq, const void* wk, const Fp4Cache& c, HeadRows qo,
                                hipStream_t st);
// Rows k and v (outputs) from the cache.
hipError_t launch_kv_read_fp4(int dtype, const PagedBatch& pb, int D, const Fp4Cache& c, HeadRows k, HeadRows v,
                              hipStream_t st);

// (a.Kc and a.Vc are the codes)
struct Fp4AttnArgs {
  AttnArgs a;
  const uint8_t *Ks, *Vs;
};
// Bytes of workspace that allow every split (0: none).
size_t fp4_attention_workspace_bytes(int dtype, int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D,
                                     int64_t max_q, int64_t max_len);
hipError_t launch_fp4_rows_bf16(const Fp4AttnArgs& f, const AttnPlan& p, hipStream_t st);
hipError_t launch_fp4_rows_f32(const Fp4AttnArgs& f, const AttnPlan& p, hipStream_t st);
hipError_t launch_fp4_tiles_bf16(const Fp4AttnArgs& f, const AttnPlan& p, hipStream_t st);
hipError_t launch_fp4_tiles_f32(const Fp4AttnArgs& f, const AttnPlan& p, hipStream_t st);
hipError_t launch_paged_attention_fp4(int dtype, const Fp4AttnArgs& a, void* ws, size_t ws_bytes, hipStream_t st);

}  // namespace ssn
