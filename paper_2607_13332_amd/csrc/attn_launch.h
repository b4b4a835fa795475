// Launchers of the attention sublayer's kernels (norm and rotation of heads,
// cache appends, attention over the cache); the C ABI in attn_api.hip
// validates arguments and then calls these.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ssn {

// Rows of heads: row i, head h at p + i * ld + h * D (elements).
struct HeadRows {
  const void* p;
  int64_t ld;
  int H;
};

// x / d for 0 <= x < 2^31 as one multiplication: with s = ceil(log2 d) and
// m = floor(2^(31+s) / d) + 1, m d - 2^(31+s) lies in (0, d], d <= 2^s, so
// x (m d - 2^(31+s)) < 2^(31+s) and the quotient is exact.  m < 2^33; for
// d > 1 it is below 2^32 (d > 2^(s-1)), and d = 1 has s = 0, m = 2^31 + 1.
struct FastDiv {
  uint32_t m, s, d;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t s = 0;
  while (((uint64_t)1 << s) < d) ++s;
  return FastDiv{(uint32_t)((((uint64_t)1 << (31 + s)) / d) + 1), s, d};
}

// A batch of sequences over a paged cache (include/ssn.h).
struct PagedBatch {
  const int32_t* pages;
  const int32_t* starts;
  const int32_t* lens;
  int32_t width, npages, B, N;
  int32_t max_len;      // lengths are clamped to it (width * page_size at most)
  FastDiv page;         // page_size = page.d
};

struct NormRope {
  int D, R, P;
  int pairs;            // pairs (2i, 2i+1) are rotated, not (i, i + R/2)
  float eps;            // < 0: no norm
  const float* table;
};

hipError_t launch_rope_table(int64_t P, int64_t R, double theta, float* table, hipStream_t st);
// Out = rot(norm(In)) for the heads of q and k (H may be 0); wq / wk NULL: ones.
hipError_t launch_norm_rope(int dtype, int64_t N, const NormRope& nr, HeadRows q, HeadRows k,
                            const void* wq, const void* wk, const int32_t* pos, HeadRows qo,
                            HeadRows ko, hipStream_t st);
// Blocks whose partial weight gradients [2][D] float32 the backward stages.
int norm_rope_backward_blocks(int64_t N, int64_t heads);
hipError_t launch_norm_rope_backward(int dtype, int64_t N, const NormRope& nr, HeadRows q, HeadRows k,
                                     const void* wq, const void* wk, const int32_t* pos, HeadRows gq,
                                     HeadRows gk, HeadRows gqi, HeadRows gki, float* gwq, float* gwk,
                                     float* ws, hipStream_t st);
hipError_t launch_kv_append(int dtype, const PagedBatch& pb, const NormRope& nr, HeadRows q, HeadRows k,
                            HeadRows v, const void* wq, const void* wk, void* Kc, void* Vc, HeadRows qo,
                            hipStream_t st);

struct AttnArgs {
  PagedBatch pb;
  const void *Q, *Kc, *Vc;
  void* O;
  float* lse;           // NULL: not wanted
  int64_t ldq, ldo;
  int Hq, Hk, D, G;     // G = Hq / Hk
  int max_q;
  float scale;
};
// A sequence's rows of one key head are its new tokens times the G heads of
// the group: row r is token r / G, head r % G.  Sequences of up to `few` rows
// run the rows kernel, whose waves share the keys; the others the tile kernel,
// whose waves share the rows.  Each kernel splits the keys into ranges of
// `chunk`; where a sequence (rows kernel) or row tile (tile kernel) has more
// than one, partial results are staged and joined: O unnormalized and (m, l)
// of every row, range by range.
//
// Ranges that `keys` keys make, and the end of the one that begins at `begin`.
// (Not by a sum of keys and chunk: lengths reach 2^31 - 4097.)
__host__ __device__ inline int key_ranges(int keys, int chunk) { return keys > chunk ? (keys - 1) / chunk + 1 : 1; }
__host__ __device__ inline int range_end(int begin, int chunk, int keys) {
  return keys - begin < chunk ? keys : begin + chunk;
}
struct AttnPart {
  int blocks;           // 16-row blocks of a wave (0: kernel not launched)
  int chunk, ranges;    // keys of a range, ranges of the longest sequence
  float* o;             // [range][stage_rows][D]
  float* ml;            // [range][stage_rows][2]
  int64_t stage_rows;
};
struct AttnPlan {
  int few;
  AttnPart rows, tiles;
};
// Bytes of workspace that allow every split (0: none).
size_t attention_workspace_bytes(int dtype, int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D,
                                 int64_t max_q, int64_t max_len);
hipError_t launch_attn_rows_bf16(const AttnArgs& a, const AttnPlan& p, hipStream_t st);
hipError_t launch_attn_rows_f32(const AttnArgs& a, const AttnPlan& p, hipStream_t st);
hipError_t launch_attn_tiles_bf16(const AttnArgs& a, const AttnPlan& p, hipStream_t st);
hipError_t launch_attn_tiles_f32(const AttnArgs& a, const AttnPlan& p, hipStream_t st);
hipError_t launch_paged_attention(int dtype, const AttnArgs& a, void* ws, size_t ws_bytes, hipStream_t st);

}  // namespace ssn
