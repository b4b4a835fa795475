// Appends to a cache held in 4 bits, and reading it back.
#include "fp4.h"
#include "norm_rope.h"

namespace ssn {

// ---------------------------------------------------------------------------
// Generic kernels (any D up to 1024, any R, any alignment): a wave owns one
// head, lane l its elements l, l + 64, ...; half a wave holds a group.
// ---------------------------------------------------------------------------

// Element e of a head is v, in every lane of the half wave: to codes and scales.
__device__ __forceinline__ void put_fp4(int e, float v, uint8_t* codes, uint8_t* scales) {
  uint32_t top = abs_bits(v);
#pragma unroll
  for (int m = 16; m >= 1; m >>= 1) top = umax(top, (uint32_t)__shfl_xor((int)top, m, kWave));
  const uint32_t s = fp4_scale_byte(top);
  const float next = __shfl_xor(v, 1, kWave);
  if (!(e & 1)) codes[e >> 1] = s == kNanScale ? 0 : (uint8_t)fp4_pack<0>(0, v, next, fp4_scale(s));
  if (e % kFp4Group == 0) scales[e / kFp4Group] = (uint8_t)s;
}

template <typename T>
__global__ __launch_bounds__(256) void kv_append_fp4_generic(PagedBatch pb, NormRope nr, HeadRows q, HeadRows k,
                                                             HeadRows v, const T* wq, const T* wk, Fp4Cache c,
                                                             HeadRows qo) {
  const int lane = threadIdx.x & 63, heads = q.H + 2 * k.H, D = nr.D;
  const int64_t total = (int64_t)pb.N * heads;
  for (int64_t j = blockIdx.x * 4LL + (threadIdx.x >> 6); j < total; j += gridDim.x * 4LL) {
    const int i = (int)(j / heads), h = (int)(j - (int64_t)i * heads);
    const int b = sequence_of_row(pb, i);
    if (b < 0) continue;
    const Sequence sq = sequence_of(pb, b);
    const int p = sq.len - (sq.s1 - i);
    if (i >= sq.s1 || p < 0) continue;
    const float* row = nr.R ? nr.table + (int64_t)clampi(p, 0, nr.P - 1) * nr.R : nullptr;
    if (h < q.H) {
      norm_rope_head(nr, head_ptr<T>(q, i, h, D), wq, row, (T*)head_ptr<T>(qo, i, h, D), lane);
    } else if (h < q.H + k.H) {
      const int64_t at = cache_row(pb, b, k.H, h - q.H, p);
      norm_rope_each(nr, head_ptr<T>(k, i, h - q.H, D), wk, row, lane, [&](int e, float x) {
        put_fp4(e, x, c.Kc + at * (D / 2), c.Ks + at * (D / kFp4Group));
      });
    } else {
      const T* x = head_ptr<T>(v, i, h - q.H - k.H, D);
      const int64_t at = cache_row(pb, b, k.H, h - q.H - k.H, p);
      for (int e = lane; e < D; e += kWave)
        put_fp4(e, load_as_f32(x + e), c.Vc + at * (D / 2), c.Vs + at * (D / kFp4Group));
    }
  }
}

hipError_t launch_kv_append_fp4(int dtype, const PagedBatch& pb, const NormRope& nr, HeadRows q, HeadRows k,
                                HeadRows v, const void* wq, const void* wk, const Fp4Cache& c, HeadRows qo,
                                hipStream_t st) {
  const unsigned blocks = wave_blocks((int64_t)pb.N * (q.H + 2 * k.H));
  if (dtype == kBF16)
    hipLaunchKernelGGL((kv_append_fp4_generic<uint16_t>), dim3(blocks), dim3(256), 0, st, pb, nr, q, k, v,
                       (const uint16_t*)wq, (const uint16_t*)wk, c, qo);
  else
    hipLaunchKernelGGL((kv_append_fp4_generic<float>), dim3(blocks), dim3(256), 0, st, pb, nr, q, k, v,
                       (const float*)wq, (const float*)wk, c, qo);
  return hipGetLastError();
}

// Reading back, any alignment of the rows: a wave owns one head, a lane two
// elements of every 128.
template <typename T>
__global__ __launch_bounds__(256) void kv_read_fp4_generic(PagedBatch pb, int D, Fp4Cache c, HeadRows k,
                                                           HeadRows v) {
  const int lane = threadIdx.x & 63, heads = 2 * k.H;
  const int64_t total = (int64_t)pb.N * heads;
  for (int64_t j = blockIdx.x * 4LL + (threadIdx.x >> 6); j < total; j += gridDim.x * 4LL) {
    const int i = (int)(j / heads), h = (int)(j - (int64_t)i * heads);
    const int b = sequence_of_row(pb, i);
    if (b < 0) continue;
    const Sequence sq = sequence_of(pb, b);
    const int p = sq.len - (sq.s1 - i);
    if (i >= sq.s1 || p < 0) continue;
    const bool isv = h >= k.H;
    const int64_t at = cache_row(pb, b, k.H, isv ? h - k.H : h, p);
    const uint8_t* codes = (isv ? c.Vc : c.Kc) + at * (D / 2);
    const uint8_t* scales = (isv ? c.Vs : c.Ks) + at * (D / kFp4Group);
    T* y = (T*)(isv ? head_ptr<T>(v, i, h - k.H, D) : head_ptr<T>(k, i, h, D));
    for (int e = 2 * lane; e < D; e += 2 * kWave) {
      const f32x2 x = fp4_f32x2<0>(codes[e >> 1], fp4_scale(scales[e / kFp4Group]));
      store_from_f32(y + e, x[0]);
      store_from_f32(y + e + 1, x[1]);
    }
  }
}

hipError_t launch_kv_read_fp4(int dtype, const PagedBatch& pb, int D, const Fp4Cache& c, HeadRows k, HeadRows v,
                              hipStream_t st) {
  const unsigned blocks = wave_blocks((int64_t)pb.N * 2 * k.H);
  if (dtype == kBF16)
    hipLaunchKernelGGL((kv_read_fp4_generic<uint16_t>), dim3(blocks), dim3(256), 0, st, pb, D, c, k, v);
  else
    hipLaunchKernelGGL((kv_read_fp4_generic<float>), dim3(blocks), dim3(256), 0, st, pb, D, c, k, v);
  return hipGetLastError();
}

}  // namespace ssn
