// Attention of new tokens over a paged cache: dispatch, the join of ranges and the
// generic kernel (the matrix-core kernels: attn_tiles.h, attn_rows.h).
//
//   O_i = sum_{t <= p_i} softmax_t(scale q_i . k_t) v_t
//
// The generic kernel makes one pass over the keys with the running maximum m and
// sum l of the softmax: for a tile of scores s, m' = max(m, max s), and with a =
// exp(m - m'), l' = a l + sum exp(s - m'), O' = a O + sum exp(s - m') v; at
// the end O / l.
#include "attn_mma.h"
#include "attn_plan.h"

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
// exp2(m - M) O_r / sum exp2(m - M) l_r, in a fixed order.  `lanes` lanes of a
// wave own a row, four elements each; with up to `lanes` ranges every group of
// them takes a row of its own (of one token), with more the groups share one
// and take the ranges in turn.

// Row r of sequence b and key head kh, its partial results at `at`.
struct JoinRow {
  int b, kh, r, ranges;
  int64_t at;
  Sequence sq;
};
template <bool FEW>
__device__ __forceinline__ bool join_row(const AttnArgs& a, const AttnPart& p, int few, JoinRow& j) {
  j.sq = sequence_of(a.pb, j.b);
  const int n = j.sq.s1 - j.sq.s0, rows = n * a.G;
  if (j.r >= rows || (rows <= few) != FEW) return false;
  int keys = j.sq.len;
  if constexpr (!FEW) {
    const int bm = 64 * p.blocks, last = (j.r / bm + 1) * bm - 1;
    keys = j.sq.len - n + (last < rows ? last : rows - 1) / a.G + 1;
  }
  j.ranges = key_ranges(keys, p.chunk);
  return j.ranges > 1;
}

// One wave: `share` lanes to a row.
template <typename T>
__device__ __forceinline__ void join_line(const AttnArgs& a, const AttnPart& p, const JoinRow& j, bool mine,
                                          int lanes, int share) {
  const int lane = threadIdx.x & 63, at = lane & (share - 1);
  float top = kNegInf;
  for (int g = at; g < j.ranges; g += share) top = fmaxf(top, p.ml[2 * (g * p.stage_rows + j.at)]);
  for (int m = share / 2; m >= 1; m >>= 1) top = fmaxf(top, __shfl_xor(top, m, kWave));
  const float base = top == kNegInf ? 0.f : top;
  const int e = (lane & (lanes - 1)) * 4, groups = share / lanes;
  float sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int g0 = at / lanes; g0 < j.ranges; g0 += 8 * groups) {
    f32x4 x[8];
    f32x2 ml[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {          // eight ranges in flight
      const int g = g0 + u * groups;
      x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      ml[u] = f32x2{kNegInf, 0.f};
      if (g < j.ranges) {
        ml[u] = *(const f32x2*)(p.ml + 2 * (g * p.stage_rows + j.at));
        if (e < a.D) x[u] = *(const f32x4*)(p.o + (g * p.stage_rows + j.at) * a.D + e);
      }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float w = __builtin_amdgcn_exp2f(ml[u][0] - base);
      sum += ml[u][1] * w;
      o += x[u] * w;
    }
  }
  for (int m = lanes; m < share; m <<= 1) {
    sum += __shfl_xor(sum, m, kWave);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], m, kWave);
  }
  const int64_t token = j.sq.s0 + j.r / a.G;
  const int head = j.kh * a.G + j.r % a.G;
  const bool sees = j.sq.len - (j.sq.s1 - (int)token) >= 0;
  if (mine && at < lanes && e < a.D)
    store4((T*)a.O + token * a.ldo + (int64_t)head * a.D + e, o * (sees ? 1.f / sum : 0.f));
  if (mine && a.lse && at == 0)
    a.lse[token * a.Hq + head] = sees ? (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f : kNegInf;
}

// Units of the tiles' lines (a token and `pt` of its heads), then of the rows
// kernel's (a sequence, a key head and `pr` of its rows): one wave each, pt and
// pr 1 or 64 / lanes.
struct JoinShape {
  int lanes, pt, pr, tile_units, units;
};
template <typename T>
__global__ __launch_bounds__(256) void paged_attn_join(AttnArgs a, AttnPlan plan, JoinShape js) {
  const int lane = threadIdx.x & 63, sub = lane / js.lanes;
  for (int unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6))); unit < js.units;
       unit += gridDim.x * 4) {
    JoinRow j;
    if (unit < js.tile_units) {
      const int per = (a.Hq + js.pt - 1) / js.pt, token = unit / per, h0 = (unit - token * per) * js.pt;
      j.b = sequence_of_row(a.pb, token);
      if (j.b < 0) continue;
      const bool mine = js.pt == 1 || h0 + sub < a.Hq;
      const int head = js.pt == 1 ? h0 : (mine ? h0 + sub : h0);
      j.kh = head / a.G;
      j.r = (token - clampi(a.pb.starts[j.b], 0, a.pb.N)) * a.G + head % a.G;
      j.at = (int64_t)token * a.Hq + head;
      // (lanes of different rows may differ in the ranges of their tiles)
      if (join_row<false>(a, plan.tiles, plan.few, j))
        join_line<T>(a, plan.tiles, j, mine, js.lanes, js.pt == 1 ? kWave : js.lanes);
    } else {
      const int rows = 16 * plan.rows.blocks, per = rows / js.pr, i = unit - js.tile_units;
      const int r0 = i % per * js.pr;
      j.kh = i / per % a.Hk;
      j.b = i / per / a.Hk;
      j.r = r0 + (js.pr == 1 ? 0 : sub);
      j.at = ((int64_t)j.b * a.Hk + j.kh) * rows + j.r;
      if (join_row<true>(a, plan.rows, plan.few, j))
        join_line<T>(a, plan.rows, j, true, js.lanes, js.pr == 1 ? kWave : js.lanes);
    }
  }
}

static hipError_t launch_join(int dtype, const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  JoinShape js;
  js.lanes = 1;
  while (js.lanes * 4 < a.D) js.lanes *= 2;
  js.pt = p.tiles.ranges <= js.lanes ? kWave / js.lanes : 1;
  js.pr = p.rows.ranges <= js.lanes ? kWave / js.lanes : 1;
  if (js.pr > 16) js.pr = 16;
  const int64_t tiles = p.tiles.blocks && p.tiles.ranges > 1 ? a.pb.N * (int64_t)((a.Hq + js.pt - 1) / js.pt) : 0;
  const int64_t rows = p.rows.blocks && p.rows.ranges > 1 ? p.rows.stage_rows / js.pr : 0;
  if (tiles + rows == 0) return hipSuccess;
  js.tile_units = (int)tiles;
  js.units = (int)(tiles + rows);
  const int64_t blocks = (tiles + rows + 3) / 4;
  const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)));
  if (dtype == kBF16)
    hipLaunchKernelGGL((paged_attn_join<uint16_t>), grid, dim3(256), 0, st, a, p, js);
  else
    hipLaunchKernelGGL((paged_attn_join<float>), grid, dim3(256), 0, st, a, p, js);
  return hipGetLastError();
}

// How a call is run: attn_plan.h.
size_t attention_workspace_bytes(int dtype, int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D, int64_t max_q,
                                 int64_t max_len) {
  if (D > 256) return 0;
  const AttnPlan p = attention_plan(dtype, N, B, Hq, Hk, D, max_q, max_len, (size_t)1 << 60);
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
  AttnPlan p = attention_plan(dtype, a.pb.N, a.pb.B, a.Hq, a.Hk, a.D, a.max_q, a.pb.max_len, ws ? ws_bytes : 0);
  char* at = (char*)ws;
  for (AttnPart* x : {&p.tiles, &p.rows})
    if (const size_t bytes = stage_bytes(*x, a.D)) {
      x->o = (float*)at;
      x->ml = x->o + x->ranges * x->stage_rows * a.D;
      at += bytes;
    }
  hipError_t e;
  if (p.tiles.blocks) e = dtype == kBF16 ? launch_attn_tiles_bf16(a, p, st) : launch_attn_tiles_f32(a, p, st);
  else e = dtype == kBF16 ? launch_attn_rows_bf16(a, p, st) : launch_attn_rows_f32(a, p, st);
  return e == hipSuccess ? launch_join(dtype, a, p, st) : e;
}

}  // namespace ssn
