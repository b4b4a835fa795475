// Attention of new tokens over a paged cache: dispatch and the generic kernel.
//
//   O_i = sum_{t <= p_i} softmax_t(scale q_i . k_t) v_t
//
// in one pass over the keys with the running maximum m and sum l of the
// softmax: for a tile of scores s, m' = max(m, max s), and with a =
// exp(m - m'), l' = a l + sum exp(s - m'), O' = a O + sum exp(s - m') v; at
// the end O / l.
#include "attn_device.h"
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

size_t attention_workspace_bytes(int, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t) {
  return 0;
}

hipError_t launch_paged_attention(int dtype, const AttnArgs& a, void*, size_t, hipStream_t st) {
  const int64_t waves = (int64_t)a.pb.N * a.Hq, blocks = (waves + 3) / 4;
  const unsigned grid = (unsigned)(blocks > (1 << 20) ? (1 << 20) : blocks);
  if (dtype == kBF16)
    hipLaunchKernelGGL((paged_attn_generic<uint16_t>), dim3(grid), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((paged_attn_generic<float>), dim3(grid), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace ssn
