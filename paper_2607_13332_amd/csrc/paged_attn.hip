// Attention of new tokens over a paged cache: dispatch and the generic kernel.
//
//   O_i = sum_{t <= p_i} softmax_t(scale q_i . k_t) v_t
//
// in one pass over the keys with the running maximum m and sum l of the
// softmax: for a tile of scores s, m' = max(m, max s), and with a =
// exp(m - m'), l' = a l + sum exp(s - m'), O' = a O + sum exp(s - m') v; at
// the end O / l.
#include "attn_mma.h"
#include "ssn_launch.h"

namespace ssn {

// Generic kernel (any D up to 1024, any alignment): a wave owns one row and
// head.  64 keys at a time: lane l computes the score of key t0 + l, the query
// in LDS; then every lane owns the elements l, l + 64, .. of the output.
// Keys past the row's position are not read.
constexpr int kGenericD = 1024;

template <typename T>
__global__ __launch_bounds__(256) void paged_attn_generic(AttnArgs a) {
  __shared__ float qs[4][kGenericD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = a.D;
  const int64_t total = (int64_t)a.pb.N * a.Hq;
  for (int64_t j = blockIdx.x * 4LL + wave; j < total; j += gridDim.x * 4LL) {
    const int i = (int)(j / a.Hq), h = (int)(j - (int64_t)i * a.Hq);
    const int b = sequence_of_row(a.pb, i);
    if (b < 0) continue;
    const Sequence sq = sequence_of(a.pb, b);
    if (i >= sq.s1) continue;
    const int keys = sq.len - (sq.s1 - i) + 1;       // positions 0 .. keys - 1 are seen
    const T* q = (const T*)a.Q + i * a.ldq + (int64_t)h * D;
    wave_lds_order();
    for (int e = lane; e < D; e += kWave) qs[wave][e] = load_as_f32(q + e) * a.scale;
    wave_lds_order();
    float o[kGenericD / kWave] = {}, m = -__builtin_inff(), l = 0.f;
    for (int t0 = 0; t0 < keys; t0 += kWave) {
      const int t = t0 + lane;
      uint32_t row = 0;
      float s = -__builtin_inff();
      if (t < keys) {
        row = cache_row(a.pb, b, a.Hk, h / a.G, t);
        const T* kp = (const T*)a.Kc + (int64_t)row * D;
        s = 0.f;
        for (int e = 0; e < D; ++e) s += qs[wave][e] * load_as_f32(kp + e);
      }
      const float mn = fmaxf(m, wave_max(s));
      // scores of -inf so far: exp(-inf - 0) = 0 rather than exp(-inf + inf)
      const float base = mn == -__builtin_inff() ? 0.f : mn;
      const float p = t < keys ? expf(s - base) : 0.f, fade = expf(m - base);
      l = l * fade + wave_sum(p);
      m = mn;
#pragma unroll
      for (int c = 0; c < kGenericD / kWave; ++c) o[c] *= fade;
      const int n = keys - t0 < kWave ? keys - t0 : kWave;
      for (int u = 0; u < n; ++u) {
        const float pu = __shfl(p, u, kWave);
        const T* vp = (const T*)a.Vc + (int64_t)(uint32_t)__shfl((int)row, u, kWave) * D;
#pragma unroll
        for (int c = 0; c < kGenericD / kWave; ++c)
          if (lane + c * kWave < D) o[c] += pu * load_as_f32(vp + lane + c * kWave);
      }
    }
    T* out = (T*)a.O + i * a.ldo + (int64_t)h * D;
    const float inv = keys > 0 ? 1.f / l : 0.f;
#pragma unroll
    for (int c = 0; c < kGenericD / kWave; ++c)
      if (lane + c * kWave < D) store_from_f32(out + lane + c * kWave, o[c] * inv);
    if (a.lse && lane == 0) a.lse[(int64_t)i * a.Hq + h] = keys > 0 ? m + logf(l) : -__builtin_inff();
  }
}

// Joins the partial results of a row's ranges: with M the largest m, O = sum
// exp2(m - M) O_r / sum exp2(m - M) l_r, in a fixed order.  A wave owns a row:
// lane i the (m, l) of ranges i, i + 64, ..; then `lanes` lanes the row's
// elements, four each, the groups of them the ranges in turn.
constexpr int kMaxRanges = 256, kRangeChunks = kMaxRanges / kWave;

// Row r of sequence b and key head kh, its partial results at `at`.
struct JoinRow {
  int b, kh, r, ranges;
  int64_t at;
  Sequence sq;
};
// Line `line` of the rows kernel's stage, or of the batch's (token, head) pairs.
template <bool FEW>
__device__ __forceinline__ bool join_row(const AttnArgs& a, const AttnPart& p, int few, int line, JoinRow& j) {
  if constexpr (FEW) {
    const int per = 16 * p.blocks;
    j.r = line % per;
    j.kh = line / per % a.Hk;
    j.b = line / per / a.Hk;
  } else {
    const int token = line / a.Hq, head = line - token * a.Hq;
    j.b = sequence_of_row(a.pb, token);
    if (j.b < 0) return false;
    j.kh = head / a.G;
    j.r = (token - clampi(a.pb.starts[j.b], 0, a.pb.N)) * a.G + head % a.G;
  }
  j.sq = sequence_of(a.pb, j.b);
  const int n = j.sq.s1 - j.sq.s0, rows = n * a.G;
  if (j.r >= rows || (rows <= few) != FEW) return false;
  int keys = j.sq.len;
  if constexpr (!FEW) {
    const int bm = 64 * p.blocks, last = (j.r / bm + 1) * bm - 1;
    keys = j.sq.len - n + (last < rows ? last : rows - 1) / a.G + 1;
  }
  j.at = line;
  j.ranges = keys > p.chunk ? (keys + p.chunk - 1) / p.chunk : 1;
  return j.ranges > 1;
}

template <typename T, bool FEW>
__global__ __launch_bounds__(256) void paged_attn_join(AttnArgs a, AttnPart p, int few, int lines, int lanes) {
  const int lane = threadIdx.x & 63;
  for (int line = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6))); line < lines;
       line += gridDim.x * 4) {
    JoinRow j;
    if (!join_row<FEW>(a, p, few, line, j)) continue;
    float w[kRangeChunks], sum = 0.f, top = kNegInf;
#pragma unroll
    for (int c = 0; c < kRangeChunks; ++c) {
      w[c] = kNegInf;
      if (c * kWave + lane < j.ranges) w[c] = p.ml[2 * ((c * kWave + lane) * p.stage_rows + j.at)];
      top = fmaxf(top, w[c]);
    }
    top = wave_max(top);
#pragma unroll
    for (int c = 0; c < kRangeChunks; ++c)
      if (c * kWave + lane < j.ranges) {
        w[c] = __builtin_amdgcn_exp2f(w[c] - (top == kNegInf ? 0.f : top));
        sum += p.ml[2 * ((c * kWave + lane) * p.stage_rows + j.at) + 1] * w[c];
      }
    sum = wave_sum(sum);
    const int e = (lane & (lanes - 1)) * 4, groups = kWave / lanes;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < kRangeChunks; ++c) {
      const int n = j.ranges - c * kWave < kWave ? j.ranges - c * kWave : kWave;
#pragma unroll 4
      for (int g = 0; g < n; g += groups) {
        const int mine = g + lane / lanes;
        const float weight = __shfl(w[c], mine & 63, kWave);
        if (mine < n && e < a.D)
          o += *(const f32x4*)(p.o + ((c * kWave + mine) * p.stage_rows + j.at) * a.D + e) * weight;
      }
    }
    for (int m = lanes; m < kWave; m <<= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], m, kWave);
    const int64_t token = j.sq.s0 + j.r / a.G;
    const int head = j.kh * a.G + j.r % a.G;
    const bool sees = j.sq.len - (j.sq.s1 - (int)token) >= 0;
    if (lane < lanes && e < a.D)
      store4((T*)a.O + token * a.ldo + (int64_t)head * a.D + e, o * (sees ? 1.f / sum : 0.f));
    if (a.lse && lane == 0)
      a.lse[token * a.Hq + head] = sees ? (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f : kNegInf;
  }
}

template <bool FEW>
static hipError_t launch_join(int dtype, const AttnArgs& a, const AttnPart& p, int few, hipStream_t st) {
  if (p.blocks == 0 || p.ranges <= 1) return hipSuccess;
  int lanes = 1;
  while (lanes * 4 < a.D) lanes *= 2;
  const int lines = (int)p.stage_rows;
  const dim3 grid((unsigned)((lines + 3) / 4 < (1 << 20) ? (lines + 3) / 4 : (1 << 20)));
  if (dtype == kBF16)
    hipLaunchKernelGGL((paged_attn_join<uint16_t, FEW>), grid, dim3(256), 0, st, a, p, few, lines, lanes);
  else
    hipLaunchKernelGGL((paged_attn_join<float, FEW>), grid, dim3(256), 0, st, a, p, few, lines, lanes);
  return hipGetLastError();
}

// How a call is run.  ws: the workspace (NULL: as many bytes as it takes).
static size_t stage_bytes(const AttnPart& p, int64_t D) {
  return p.blocks && p.ranges > 1 ? (size_t)p.ranges * (size_t)p.stage_rows * (size_t)(D + 2) * 4 : 0;
}
// Ranges for about `want` of them, no more than `fit` bytes hold.
static void split_keys(AttnPart& p, int64_t want, int64_t unit, int64_t max_len, int64_t D, size_t fit) {
  const int64_t row_bytes = p.stage_rows * (D + 2) * 4;
  if (row_bytes > 0 && (size_t)want > fit / (size_t)row_bytes) want = (int64_t)(fit / (size_t)row_bytes);
  if (want > kMaxRanges) want = kMaxRanges;
  const int64_t len = max_len > 1 ? max_len : 1;
  int64_t chunk = want > 1 ? (len + want - 1) / want : len;
  chunk = (chunk + unit - 1) / unit * unit;
  p.chunk = (int)chunk;
  p.ranges = (int)((len + p.chunk - 1) / p.chunk);
}
static AttnPlan attention_plan(int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D, int64_t max_q,
                               int64_t max_len, size_t ws_bytes) {
  AttnPlan p = {};
  const int64_t G = Hq / Hk, most = max_q * G;
  const bool wide = D > 128;
  if (most <= 16 || (most <= 32 && !wide)) {
    p.few = most <= 16 ? 16 : 32;
  } else {
    // single tokens among longer chunks, unless all have max_q
    if (G <= 16 && N != B * max_q) p.few = 16;
    p.tiles.blocks = (most <= 64 || wide) ? 1 : 2;
  }
  p.rows.blocks = (p.few + 15) / 16;
  p.rows.stage_rows = B * Hk * 16 * p.rows.blocks;
  p.tiles.stage_rows = N * Hq;
  if (p.tiles.blocks) {
    // two blocks to a compute unit, where the rows alone do not give them
    const int64_t big = p.few ? (N - B + 1 > 1 ? N - B + 1 : 1) : N;
    const int64_t blocks = (big * G / (64 * p.tiles.blocks) + 1) * Hk;
    split_keys(p.tiles, blocks >= 512 ? 1 : 512 / blocks, 256, max_len, D, ws_bytes);
  }
  if (p.rows.blocks) {
    const size_t left = ws_bytes - stage_bytes(p.tiles, D);
    const int64_t pairs = B * Hk, full = 512 / pairs, want = (2048 + pairs - 1) / pairs;
    split_keys(p.rows, want > 64 && want > full ? (full > 64 ? full : 64) : want, 128, max_len, D, left);
  }
  return p;
}

size_t attention_workspace_bytes(int, int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D, int64_t max_q,
                                 int64_t max_len) {
  if (D > 256) return 0;
  const AttnPlan p = attention_plan(N, B, Hq, Hk, D, max_q, max_len, (size_t)1 << 60);
  return stage_bytes(p.tiles, D) + stage_bytes(p.rows, D);
}

// The matrix-core kernels read 16 bytes at a time.
static bool vector_access(int dtype, const AttnArgs& a) {
  const int64_t s = dtype == kBF16 ? 2 : 4;
  const uintptr_t p = (uintptr_t)a.Q | (uintptr_t)a.Kc | (uintptr_t)a.Vc | (uintptr_t)a.O;
  return a.D <= 256 && (a.D * s) % 16 == 0 && p % 16 == 0 && (a.ldq * s) % 16 == 0 && (a.ldo * s) % 16 == 0;
}

hipError_t launch_paged_attention(int dtype, const AttnArgs& a, void* ws, size_t ws_bytes, hipStream_t st) {
  if (!vector_access(dtype, a)) {
    const int64_t waves = (int64_t)a.pb.N * a.Hq, blocks = (waves + 3) / 4;
    const unsigned grid = (unsigned)(blocks > (1 << 20) ? (1 << 20) : blocks);
    if (dtype == kBF16)
      hipLaunchKernelGGL((paged_attn_generic<uint16_t>), dim3(grid), dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((paged_attn_generic<float>), dim3(grid), dim3(256), 0, st, a);
    return hipGetLastError();
  }
  AttnPlan p = attention_plan(a.pb.N, a.pb.B, a.Hq, a.Hk, a.D, a.max_q, a.pb.max_len, ws ? ws_bytes : 0);
  float* at = (float*)ws;
  for (AttnPart* x : {&p.tiles, &p.rows})
    if (stage_bytes(*x, a.D)) {
      x->o = at;
      x->ml = at + x->ranges * x->stage_rows * a.D;
      at = x->ml + x->ranges * x->stage_rows * 2;
    }
  hipError_t e = hipSuccess;
  if (p.tiles.blocks) e = dtype == kBF16 ? launch_attn_tiles_bf16(a, p, st) : launch_attn_tiles_f32(a, p, st);
  if (e == hipSuccess && p.rows.blocks)
    e = dtype == kBF16 ? launch_attn_rows_bf16(a, p, st) : launch_attn_rows_f32(a, p, st);
  if (e == hipSuccess) e = launch_join<false>(dtype, a, p.tiles, p.few, st);
  return e == hipSuccess ? launch_join<true>(dtype, a, p.rows, p.few, st) : e;
}

}  // namespace ssn
