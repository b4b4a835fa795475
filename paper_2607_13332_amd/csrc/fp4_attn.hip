// Attention of new tokens over a paged cache held in 4 bits: dispatch and the
// generic kernel.
//
//   O_i = sum_{t <= p_i} softmax_t(scale q_i . k_t) v_t
//
// with k and v the values that the cache stands for.  The generic kernel makes one
// pass over the keys with the running maximum m and sum l of the softmax: for a
// tile of scores s, m' = max(m, max s), and with a = exp(m - m'), l' = a l + sum
// exp(s - m'), O' = a O + sum exp(s - m') v; at the end O / l.
#include "fp4.h"
#include "fp4_plan.h"

namespace ssn {

// Any D up to 1024, any alignment: a wave owns one row and head.  64 keys at a
// time: lane l computes the score of key t0 + l, the query in LDS; then every lane
// owns the elements 2 l, 2 l + 1, 2 l + 128, .. of the output.  Keys past the
// row's position are not read.
constexpr int kFp4GenericD = 1024;

template <typename T>
__global__ __launch_bounds__(256) void paged_attn_fp4_generic(Fp4AttnArgs fa) {
  __shared__ float qs[4][kFp4GenericD];
  const AttnArgs& a = fa.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = a.D, groups = D / kFp4Group;
  const uint8_t *kc = (const uint8_t*)a.Kc, *vc = (const uint8_t*)a.Vc;
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
    constexpr int kPairs = kFp4GenericD / 2 / kWave;
    f32x2 o[kPairs];
#pragma unroll
    for (int c = 0; c < kPairs; ++c) o[c] = f32x2{0.f, 0.f};
    float m = -__builtin_inff(), l = 0.f;
    for (int t0 = 0; t0 < keys; t0 += kWave) {
      const int t = t0 + lane;
      uint32_t row = 0;
      float s = -__builtin_inff();
      if (t < keys) {
        row = cache_row(a.pb, b, a.Hk, h / a.G, t);
        const uint8_t* codes = kc + (int64_t)row * (D / 2);
        const uint8_t* scales = fa.Ks + (int64_t)row * groups;
        s = 0.f;
        for (int g = 0; g < groups; ++g) {
          const float scale = fp4_scale(scales[g]);
          for (int e = g * kFp4Group; e < (g + 1) * kFp4Group; e += 2) {
            const f32x2 x = fp4_f32x2<0>(codes[e >> 1], scale);
            s += qs[wave][e] * x[0];
            s += qs[wave][e + 1] * x[1];
          }
        }
      }
      const float mn = fmaxf(m, wave_max(s));
      // scores of -inf so far: exp(-inf - 0) = 0 rather than exp(-inf + inf)
      const float base = mn == -__builtin_inff() ? 0.f : mn;
      const float p = t < keys ? expf(s - base) : 0.f, fade = expf(m - base);
      l = l * fade + wave_sum(p);
      m = mn;
#pragma unroll
      for (int c = 0; c < kPairs; ++c) o[c] *= fade;
      const int n = keys - t0 < kWave ? keys - t0 : kWave;
      for (int u = 0; u < n; ++u) {
        const float pu = __shfl(p, u, kWave);
        const int64_t at = (uint32_t)__shfl((int)row, u, kWave);
#pragma unroll
        for (int c = 0; c < kPairs; ++c) {
          const int e = 2 * lane + c * 2 * kWave;
          if (e < D) o[c] += pu * fp4_f32x2<0>(vc[at * (D / 2) + (e >> 1)], fp4_scale(fa.Vs[at * groups + e / kFp4Group]));
        }
      }
    }
    T* out = (T*)a.O + i * a.ldo + (int64_t)h * D;
    const float inv = keys > 0 ? 1.f / l : 0.f;
#pragma unroll
    for (int c = 0; c < kPairs; ++c) {
      const int e = 2 * lane + c * 2 * kWave;
      if (e < D) {
        store_from_f32(out + e, o[c][0] * inv);
        store_from_f32(out + e + 1, o[c][1] * inv);
      }
    }
    if (a.lse && lane == 0) a.lse[(int64_t)i * a.Hq + h] = keys > 0 ? m + logf(l) : -__builtin_inff();
  }
}

// How a call is run: fp4_plan.h.
size_t fp4_attention_workspace_bytes(int dtype, int64_t N, int64_t B, int64_t Hq, int64_t Hk, int64_t D,
                                     int64_t max_q, int64_t max_len) {
  if (D > 256) return 0;
  const AttnPlan p = attention_plan(dtype, N, B, Hq, Hk, D, max_q, max_len, (size_t)1 << 60, kFp4Tuning);
  return stage_bytes(p.tiles, D) + stage_bytes(p.rows, D);
}

// The matrix-core kernels read 16 bytes at a time (8 of heads up to 64).
static bool fp4_vector_access(int dtype, const AttnArgs& a) {
  const int64_t s = dtype == kBF16 ? 2 : 4;
  const uintptr_t p = (uintptr_t)a.Q | (uintptr_t)a.Kc | (uintptr_t)a.Vc | (uintptr_t)a.O;
  return a.D <= 256 && p % 16 == 0 && (a.ldq * s) % 16 == 0 && (a.ldo * s) % 16 == 0;
}

hipError_t launch_paged_attention_fp4(int dtype, const Fp4AttnArgs& f, void* ws, size_t ws_bytes, hipStream_t st) {
  const AttnArgs& a = f.a;
  if (!fp4_vector_access(dtype, a)) {
    const int64_t waves = (int64_t)a.pb.N * a.Hq, blocks = (waves + 3) / 4;
    const unsigned grid = (unsigned)(blocks > (1 << 20) ? (1 << 20) : blocks);
    if (dtype == kBF16)
      hipLaunchKernelGGL((paged_attn_fp4_generic<uint16_t>), dim3(grid), dim3(256), 0, st, f);
    else
      hipLaunchKernelGGL((paged_attn_fp4_generic<float>), dim3(grid), dim3(256), 0, st, f);
    return hipGetLastError();
  }
  AttnPlan p = attention_plan(dtype, a.pb.N, a.pb.B, a.Hq, a.Hk, a.D, a.max_q, a.pb.max_len, ws ? ws_bytes : 0, kFp4Tuning);
  char* at = (char*)ws;
  for (AttnPart* x : {&p.tiles, &p.rows})
    if (const size_t bytes = stage_bytes(*x, a.D)) {
      x->o = (float*)at;
      x->ml = x->o + x->ranges * x->stage_rows * a.D;
      at += bytes;
    }
  hipError_t e;
  if (p.tiles.blocks) e = dtype == kBF16 ? launch_fp4_tiles_bf16(f, p, st) : launch_fp4_tiles_f32(f, p, st);
  else e = dtype == kBF16 ? launch_fp4_rows_bf16(f, p, st) : launch_fp4_rows_f32(f, p, st);
  return e == hipSuccess ? launch_attn_join(dtype, a, p, st) : e;
}

}  // namespace ssn
