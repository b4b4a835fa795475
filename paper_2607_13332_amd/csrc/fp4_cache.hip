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

// ---------------------------------------------------------------------------
// Fast kernels (16-byte aligned rows, 4-byte aligned codes).  Memory bounds them:
// rows are read (or written) once, 4.25 bits an element the other way.  12676 tokens of
// 8 + 8 heads of 128 are appended in 17 us and read back in 16 (66 MB each, 3.9 and 4.1
// TB/s; with norm, rotation and 40 heads of queries 58 us, 6 TB/s); one token takes 2
// us each way, the latency of three loads one after the other.
// ---------------------------------------------------------------------------

// Where a lane's 8 elements of a token's keys and values are: chunk `chunk` of 2 Hk
// D / 8, keys first, then values.
struct KvChunk {
  bool any, isv;
  int h, e;             // head and its element
  __device__ __forceinline__ KvChunk(int chunk, int Hk, int D) {
    const int per = D / 8, half = Hk * per;
    any = chunk < 2 * half;
    isv = chunk >= half;
    const int c = any ? (isv ? chunk - half : chunk) : 0;
    h = c / per;
    e = (c - h * per) * 8;
  }
};
// The batch's sequences as a wave looks rows up in them.  Of up to 64 a lane has one,
// all loaded at once, and a lookup waits for nothing; of more every lookup searches
// memory.
struct Sequences {
  int s0, s1, len;      // of sequence `lane`
  __device__ __forceinline__ void load(const PagedBatch& pb) {
    const int lane = threadIdx.x & 63, b = lane < pb.B ? lane : pb.B - 1;
    if (pb.B > kWave) return;
    s0 = pb.starts[b];
    s1 = pb.starts[b + 1];
    len = pb.lens[b];
  }
  // The sequence of row i, its number b; -1 before the first.
  __device__ __forceinline__ Sequence find(const PagedBatch& pb, int i, int& b) const {
    if (pb.B > kWave) {
      b = sequence_of_row(pb, i);
      return b < 0 ? Sequence{0, 0, 0} : sequence_of(pb, b);
    }
    const int lane = threadIdx.x & 63;
    b = __popcll(__ballot(lane < pb.B && s0 <= i)) - 1;
    Sequence sq = {0, 0, 0};
    if (b >= 0) {
      sq.s0 = clampi(__builtin_amdgcn_readlane(s0, b), 0, pb.N);
      sq.s1 = clampi(__builtin_amdgcn_readlane(s1, b), sq.s0, pb.N);
      sq.len = clampi(__builtin_amdgcn_readlane(len, b), 0, pb.max_len);
    }
    return sq;
  }
};

// The cache rows of head h at the positions of U consecutive rows from i on; -1:
// a row has none.  Rows of one sequence follow from the first.
template <int U>
__device__ __forceinline__ void find_rows(const PagedBatch& pb, const Sequences& seqs, int i, int Hk, int h,
                                          int64_t (&row)[U]) {
  int b;
  Sequence sq = seqs.find(pb, i, b);
  bool has[U];
  Slot slot[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u && i + u < pb.N && (b < 0 || i + u >= sq.s1)) sq = seqs.find(pb, i + u, b);
    const int p = sq.len - (sq.s1 - (i + u));
    has[u] = b >= 0 && i + u < sq.s1 && p >= 0;
    slot[u] = Slot{0, 0};
    if (has[u]) slot[u] = find_slot(pb, b, p);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) row[u] = has[u] ? (int64_t)slot_row(pb, slot[u], Hk, h) : -1;
}

// Keys and values that are quantised as they are: a wave takes 64 chunks of U
// consecutive tokens, four lanes a group, and keeps to its chunks from token to
// token.
template <typename T, int U>
__global__ __launch_bounds__(256) void kv_append_fp4_plain(Spread sp, PagedBatch pb, int D, HeadRows k, HeadRows v,
                                                           Fp4Cache c) {
  const int lane = threadIdx.x & 63;
  const int id = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (id >= sp.waves()) return;
  const KvChunk at(id % sp.passes * kWave + lane, k.H, D);
  const HeadRows in = at.isv ? v : k;
  const T* src = (const T*)in.p + at.h * D + at.e;
  uint8_t *codes = at.isv ? c.Vc : c.Kc, *scales = at.isv ? c.Vs : c.Ks;
  Sequences seqs;
  seqs.load(pb);
  for (int64_t i = (int64_t)(id / sp.passes) * U; i < pb.N; i += (int64_t)sp.slots * U) {
    Chunk<uint16_t> x[U];               // 8 elements of either type
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool any = at.any && i + u < pb.N;
      const T* from = src + (i + u) * in.ld;
      if constexpr (sizeof(T) == 2) {
        x[u].set(any ? __builtin_nontemporal_load((const u32x4*)from) : u32x4{0, 0, 0, 0});
      } else {
#pragma unroll
        for (int z = 0; z < 2; ++z)
          *(f32x4*)(x[u].v + 4 * z) = any ? __builtin_nontemporal_load((const f32x4*)(from + 4 * z)) : f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
    int64_t row[U];
    find_rows<U>(pb, seqs, (int)i, k.H, at.h, row);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t s;
      const uint32_t w = fp4_quantise<8>(x[u].v, s);
      if (row[u] >= 0 && at.any) {
        *(uint32_t*)(codes + row[u] * (D / 2) + at.e / 2) = w;
        if (at.e % kFp4Group == 0) scales[row[u] * (D / kFp4Group) + at.e / kFp4Group] = (uint8_t)s;
      }
    }
  }
}

// With norm or rotation, or with queries: as the append to a bf16 or float32 cache
// (heads of 64, 128 or 256, all rotated or none of it), a group in the lanes of one
// chunk of 16 bytes each.
template <typename T, int D, int ROT>
__global__ __launch_bounds__(256) void kv_append_fp4_rows(Spread sp, NormRope nr, HeadRows q, HeadRows k, HeadRows v,
                                                          const T* __restrict__ wq, const T* __restrict__ wk,
                                                          HeadRows qo, PagedBatch pb, Fp4Cache c) {
  constexpr int E = Chunk<T>::E, LPH = D / (2 * E);
  const int lane = threadIdx.x & 63;
  const int id = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (id >= sp.waves()) return;
  const int pass = id % sp.passes, j = lane % LPH, head = pass * (kWave / LPH) + lane / LPH;
  const bool isq = head < q.H, isk = !isq && head < q.H + k.H;
  const bool isv = !isq && !isk && head < q.H + 2 * k.H, any = isq || isk || isv;
  const HeadRows in = isq ? q : (isv ? v : k);
  const int h = isq ? head : (isv ? head - q.H - k.H : head - q.H);
  const T* src = (const T*)in.p + h * D + E * j;
  Chunk<T> wa, wb;
  wa.ones();
  wb.ones();
  const T* w = isq ? wq : wk;
  if (any && !isv && w) {
    wa.set(*(const u32x4*)(w + E * j));
    wb.set(*(const u32x4*)(w + D / 2 + E * j));
  }
  Sequences seqs;
  seqs.load(pb);
  for (int i = id / sp.passes; i < pb.N; i += sp.slots) {
    int b;
    const Sequence sq = seqs.find(pb, i, b);
    const int p = sq.len - (sq.s1 - i);
    if (b < 0 || i >= sq.s1 || p < 0) continue;
    u32x4 xa = {0, 0, 0, 0}, xb = {0, 0, 0, 0};
    if (any) {
      xa = __builtin_nontemporal_load((const u32x4*)(src + i * in.ld));
      xb = __builtin_nontemporal_load((const u32x4*)(src + i * in.ld + D / 2));
    }
    Turn<T, D, ROT> turn;
    if constexpr (ROT != kNoRotation) turn.load(nr.table + (int64_t)clampi(p, 0, nr.P - 1) * D, j);
    Chunk<T> x, y;
    x.set(xa);
    y.set(xb);
    if (!isv) {
      if (nr.eps >= 0.f) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) ss += x.v[e] * x.v[e] + y.v[e] * y.v[e];
        const float r = rsqrtf(head_sum<LPH>(ss) * (1.f / D) + nr.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          x.v[e] *= r * wa.v[e];
          y.v[e] *= r * wb.v[e];
        }
      }
      turn.apply(x, y, 1.f);
    }
    uint32_t sx, sy;
    const uint32_t cx = fp4_quantise<E>(x.v, sx), cy = fp4_quantise<E>(y.v, sy);
    if (isq) {
      T* dst = (T*)qo.p + i * qo.ld + h * D + E * j;
      *(u32x4*)dst = x.get();
      *(u32x4*)(dst + D / 2) = y.get();
    } else if (any) {
      const int64_t row = cache_row(pb, b, k.H, h, p);
      uint8_t* codes = (isv ? c.Vc : c.Kc) + row * (D / 2) + E * j / 2;
      uint8_t* scales = (isv ? c.Vs : c.Ks) + row * (D / kFp4Group) + E * j / kFp4Group;
      if constexpr (E == 8) {
        *(uint32_t*)codes = cx;
        *(uint32_t*)(codes + D / 4) = cy;
      } else {
        *(uint16_t*)codes = (uint16_t)cx;
        *(uint16_t*)(codes + D / 4) = (uint16_t)cy;
      }
      if (E * j % kFp4Group == 0) {
        scales[0] = (uint8_t)sx;
        scales[D / 2 / kFp4Group] = (uint8_t)sy;
      }
    }
  }
}

// Reading back: a wave takes 64 chunks of 8 elements of U consecutive tokens.
template <typename T, int U>
__global__ __launch_bounds__(256) void kv_read_fp4_rows(Spread sp, PagedBatch pb, int D, Fp4Cache c, HeadRows k,
                                                        HeadRows v) {
  const int lane = threadIdx.x & 63;
  const int id = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (id >= sp.waves()) return;
  const KvChunk at(id % sp.passes * kWave + lane, k.H, D);
  const HeadRows out = at.isv ? v : k;
  T* dst = (T*)out.p + at.h * D + at.e;
  const uint8_t *codes = at.isv ? c.Vc : c.Kc, *scales = at.isv ? c.Vs : c.Ks;
  Sequences seqs;
  seqs.load(pb);
  for (int64_t i = (int64_t)(id / sp.passes) * U; i < pb.N; i += (int64_t)sp.slots * U) {
    int64_t row[U];
    find_rows<U>(pb, seqs, (int)i, k.H, at.h, row);
    uint32_t w[U], e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      w[u] = e[u] = 0;
      if (row[u] >= 0 && at.any) {
        w[u] = __builtin_nontemporal_load((const uint32_t*)(codes + row[u] * (D / 2) + at.e / 2));
        e[u] = scales[row[u] * (D / kFp4Group) + at.e / kFp4Group];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (row[u] < 0 || !at.any) continue;
      const float scale = fp4_scale(e[u]);
      T* to = dst + (i + u) * out.ld;
      if constexpr (sizeof(T) == 2) {
        __builtin_nontemporal_store(fp4_bf16x8(w[u], scale), (u32x4*)to);
      } else {
        const f32x2 a = fp4_f32x2<0>(w[u], scale), b = fp4_f32x2<1>(w[u], scale), x = fp4_f32x2<2>(w[u], scale),
                    y = fp4_f32x2<3>(w[u], scale);
        __builtin_nontemporal_store(f32x4{a[0], a[1], b[0], b[1]}, (f32x4*)to);
        __builtin_nontemporal_store(f32x4{x[0], x[1], y[0], y[1]}, (f32x4*)(to + 4));
      }
    }
  }
}

static bool codes_aligned(const Fp4Cache& c) { return ((uintptr_t)c.Kc | (uintptr_t)c.Vc) % 4 == 0; }
// Tokens that a wave has at a time, one where there would be too few waves.  29.5k
// tokens of 8 heads of 128 are read back in 42 / 38 / 36 us with 2 / 4 / 8, 131072 in
// 178 / 159 / 138 (4.9 TB/s, the rate of a large copy); appends gain 1 % from more
// than 4.  (69 us with one and a search in memory for each, 41 with four of those.)
constexpr int kAppendTokens = 4, kReadTokens = 8;
static bool many_tokens(const PagedBatch& pb, int Hk, int D) { return (int64_t)pb.N * Hk * D >= kForwardWaves * 256; }
static Spread spread_chunks(int64_t tokens, int Hk, int D) {
  return spread_tokens(tokens, 2 * Hk * (D / 8), kWave, kForwardWaves);
}
static dim3 grid_of(const Spread& sp) { return dim3((unsigned)((sp.waves() + 3) / 4)); }

struct Fp4Append {
  PagedBatch pb;
  NormRope nr;
  HeadRows q, k, v;
  const void *wq, *wk;
  Fp4Cache c;
  HeadRows qo;
  hipStream_t st;
};
template <typename T, int D, int ROT>
static hipError_t append_rows(const Fp4Append& a) {
  const Spread sp = spread_tokens(a.pb.N, a.q.H + 2 * a.k.H, kWave * 2 * Chunk<T>::E / D, kForwardWaves);
  hipLaunchKernelGGL((kv_append_fp4_rows<T, D, ROT>), grid_of(sp), dim3(256), 0, a.st, sp, a.nr, a.q, a.k, a.v,
                     (const T*)a.wq, (const T*)a.wk, a.qo, a.pb, a.c);
  return hipGetLastError();
}
template <typename T, int D>
static hipError_t append_rot(const Fp4Append& a) {
  if (!a.nr.R) return append_rows<T, D, kNoRotation>(a);
  return a.nr.pairs ? append_rows<T, D, kPairs>(a) : append_rows<T, D, kHalves>(a);
}
template <typename T>
static hipError_t append(const Fp4Append& a) {
  constexpr int kType = sizeof(T) == 2 ? kBF16 : kF32;
  const bool codes = codes_aligned(a.c);
  if (codes && a.q.H == 0 && a.nr.eps < 0.f && a.nr.R == 0 && aligned16(a.k, sizeof(T)) && aligned16(a.v, sizeof(T))) {
    if (many_tokens(a.pb, a.k.H, a.nr.D)) {
      const Spread sp = spread_chunks((a.pb.N + kAppendTokens - 1) / kAppendTokens, a.k.H, a.nr.D);
      hipLaunchKernelGGL((kv_append_fp4_plain<T, kAppendTokens>), grid_of(sp), dim3(256), 0, a.st, sp, a.pb, a.nr.D, a.k, a.v, a.c);
    } else {
      const Spread sp = spread_chunks(a.pb.N, a.k.H, a.nr.D);
      hipLaunchKernelGGL((kv_append_fp4_plain<T, 1>), grid_of(sp), dim3(256), 0, a.st, sp, a.pb, a.nr.D, a.k, a.v, a.c);
    }
    return hipGetLastError();
  }
  if (codes && fast_heads(kType, a.nr, {a.q, a.k, a.v, a.qo}, {a.wq, a.wk})) {
    if (a.nr.D == 64) return append_rot<T, 64>(a);
    return a.nr.D == 128 ? append_rot<T, 128>(a) : append_rot<T, 256>(a);
  }
  hipLaunchKernelGGL((kv_append_fp4_generic<T>), dim3(wave_blocks((int64_t)a.pb.N * (a.q.H + 2 * a.k.H))), dim3(256),
                     0, a.st, a.pb, a.nr, a.q, a.k, a.v, (const T*)a.wq, (const T*)a.wk, a.c, a.qo);
  return hipGetLastError();
}

hipError_t launch_kv_append_fp4(int dtype, const PagedBatch& pb, const NormRope& nr, HeadRows q, HeadRows k,
                                HeadRows v, const void* wq, const void* wk, const Fp4Cache& c, HeadRows qo,
                                hipStream_t st) {
  const Fp4Append a = {pb, nr, q, k, v, wq, wk, c, qo, st};
  return dtype == kBF16 ? append<uint16_t>(a) : append<float>(a);
}

template <typename T>
static hipError_t read_back(const PagedBatch& pb, int D, const Fp4Cache& c, HeadRows k, HeadRows v, hipStream_t st) {
  if (codes_aligned(c) && aligned16(k, sizeof(T)) && aligned16(v, sizeof(T))) {
    if (many_tokens(pb, k.H, D)) {
      const Spread sp = spread_chunks((pb.N + kReadTokens - 1) / kReadTokens, k.H, D);
      hipLaunchKernelGGL((kv_read_fp4_rows<T, kReadTokens>), grid_of(sp), dim3(256), 0, st, sp, pb, D, c, k, v);
    } else {
      const Spread sp = spread_chunks(pb.N, k.H, D);
      hipLaunchKernelGGL((kv_read_fp4_rows<T, 1>), grid_of(sp), dim3(256), 0, st, sp, pb, D, c, k, v);
    }
  } else {
    hipLaunchKernelGGL((kv_read_fp4_generic<T>), dim3(wave_blocks((int64_t)pb.N * 2 * k.H)), dim3(256), 0, st, pb, D, c,
                       k, v);
  }
  return hipGetLastError();
}

hipError_t launch_kv_read_fp4(int dtype, const PagedBatch& pb, int D, const Fp4Cache& c, HeadRows k, HeadRows v,
                              hipStream_t st) {
  return dtype == kBF16 ? read_back<uint16_t>(pb, D, c, k, v, st) : read_back<float>(pb, D, c, k, v, st);
}

}  // namespace ssn
