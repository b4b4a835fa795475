// Attention of few rows over a 4-bit cache: a block of 4 waves owns a range of the
// keys of one sequence and key head; its waves take the range's tiles of 64 keys in
// turn, all with the same 16 QB rows, and join their results in LDS at the end.
#pragma once

#include "attn_rows.h"
#include "fp4_attn_mma.h"

namespace ssn {

constexpr int kFp4Keys = 64;           // of a wave's tile
template <int DT, int QB>
constexpr int fp4_rows_lds() {
  const int tiles = 4 * 32 * DT * 2, join = 2 * (DT / 16 * QB * kWave * 16);
  return (tiles > join ? tiles : join) + 4 * QB * kWave * 4;         // and m, l of two waves
}

template <typename T, int DT, int QB, bool EXACT>
__device__ __forceinline__ void fp4_rows_block(const Fp4AttnArgs& fa, const AttnPart& part, int few, int id, char* lds) {
  using Tag = OverFp4<T>;
  using M = Mma<Tag>;
  constexpr int RB = DT * 2, TK = kFp4Keys, NKB = TK / 16, NC = DT / 32, DT16 = DT / 16, PARTS = M::kRowsParts;
  // A key's lanes 16 g + its number hold the g-th quarter of its head, UW dwords
  // of codes and SC scales: 16 bytes of one group where the head has 128 elements.
  constexpr int UE = DT / 4, UW = UE / 8, SC = UE > kFp4Group ? UE / kFp4Group : 1, kTile = 32 * RB;
  const AttnArgs& a = fa.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kh = id % a.Hk, rest = id / a.Hk, b = rest % a.pb.B, range = rest / a.pb.B;
  const Sequence sq = sequence_of(a.pb, b);
  const int n = sq.s1 - sq.s0, rows = n * a.G, keys = sq.len;
  if (rows == 0 || rows > few) return;
  const int ranges = key_ranges(keys, part.chunk);
  if (range >= ranges) return;
  const int before = sq.len - n, groups = a.D / kFp4Group;
  const int k_begin = range * part.chunk, k_end = range_end(k_begin, part.chunk, keys);
  const int g = lane >> 4, e0 = g * UE;

  int row[QB], seen[QB];
  u32x4 qf[QB][NC][M::kQueries];
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    row[q] = q * 16 + (lane & 15);
    const int r = row[q] < rows ? row[q] : rows - 1, token = r / a.G;
    seen[q] = before + token;
    const T* p = (const T*)a.Q + (sq.s0 + token) * a.ldq + (int64_t)(kh * a.G + r % a.G) * a.D;
#pragma unroll
    for (int ch = 0; ch < NC; ++ch) {
#pragma unroll
      for (int m = 0; m < M::kQueries; ++m) qf[q][ch][m] = u32x4{0, 0, 0, 0};
      if (a.scale != 0.f && (EXACT || e0 + 8 * ch < a.D)) query_parts<T>(p + e0 + 8 * ch, sign_bits<T>(a.scale), qf[q][ch]);
    }
  }
  const float c = (a.scale == 0.f ? 1.f : fabsf(a.scale)) * kLog2e;

  char* vl = lds + wave * kTile;
  uint32_t kreg[NKB][UW], vreg[NKB][UW];
  uint8_t ks[NKB][SC], vs[NKB][SC];
  auto rows_of = [&](int t) {
    const int key = t + lane;
    return find_slot(a.pb, b, key < keys ? key : keys - 1);
  };
  auto load = [&](const uint8_t* codes, const uint8_t* scales, uint32_t r, uint32_t (&w)[UW], uint8_t (&s)[SC]) {
    constexpr int V = UW < 4 ? UW : 4;
    typedef uint32_t piece __attribute__((ext_vector_type(V)));
#pragma unroll
    for (int i = 0; i < UW; i += V) {
      piece x = {};
      if (EXACT || e0 + 8 * i < a.D)
        x = __builtin_nontemporal_load((const piece*)(codes + (int64_t)r * (a.D / 2) + e0 / 2 + 4 * i));
#pragma unroll
      for (int j = 0; j < V; ++j) w[i + j] = x[j];
    }
#pragma unroll
    for (int i = 0; i < SC; ++i) {
      s[i] = 0;
      if (EXACT || e0 + 32 * i < a.D) s[i] = scales[(int64_t)r * groups + e0 / kFp4Group + i];
    }
  };
  auto fetch_key = [&](uint32_t mine, int k) {
    load((const uint8_t*)a.Kc, fa.Ks, (uint32_t)__shfl((int)mine, 16 * k + (lane & 15), kWave), kreg[k], ks[k]);
  };
  auto fetch_value = [&](uint32_t mine, int k) {
    load((const uint8_t*)a.Vc, fa.Vs, (uint32_t)__shfl((int)mine, 16 * k + value_key<RB>(lane & 15), kWave), vreg[k], vs[k]);
  };
  const uint32_t vb[1] = {M::template vbase<RB>(lane, 0)};

  RowState<DT16, QB> rs;
  rs.clear();
  int t = k_begin + wave * TK;
  uint32_t odd = 0;
  Slot next = {0, 0};
  if (t < k_end) {
    const uint32_t mine = slot_row(a.pb, rows_of(t), a.Hk, kh);
#pragma unroll
    for (int k = 0; k < NKB; ++k) fetch_key(mine, k);
#pragma unroll
    for (int k = 0; k < NKB; ++k) fetch_value(mine, k);
    if (t + 4 * TK < k_end) next = rows_of(t + 4 * TK);
  }
  for (; t < k_end; t += 4 * TK) {
    const bool masked = t + TK - 1 > before, more = t + 4 * TK < k_end;
    f32x4 s[NKB][QB];
#pragma unroll
    for (int k = 0; k < NKB; ++k) {
#pragma unroll
      for (int q = 0; q < QB; ++q) s[k][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ch = 0; ch < NC; ++ch) {
        const u32x4 kf = fp4_bf16x8(kreg[k][ch], fp4_scale(ks[k][8 * ch / kFp4Group]));
#pragma unroll
        for (int q = 0; q < QB; ++q)
#pragma unroll
          for (int m = M::kQueries - 1; m >= 0; --m) s[k][q] = M::mma(kf, qf[q][ch][m], s[k][q]);
      }
    }
    uint32_t mine = 0;
    if (more) {
      mine = slot_row(a.pb, next, a.Hk, kh);
#pragma unroll
      for (int k = 0; k < NKB; ++k) fetch_key(mine, k);
      if (t + 8 * TK < k_end) next = rows_of(t + 8 * TK);
    }
    if (masked) {
#pragma unroll
      for (int q = 0; q < QB; ++q)
#pragma unroll
        for (int k = 0; k < NKB; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * k + 4 * (lane >> 4) + i > seen[q] - t) s[k][q][i] = kNegInf;
    }
    u32x4 p[PARTS][NKB / 2][QB];
    softmax_step<Tag, PARTS>(s, rs, c, p);
    // 32 keys' values at a time through the wave's part of LDS
#pragma unroll
    for (int half = 0; half < NKB / 2; ++half) {
      wave_lds_order();
#pragma unroll
      for (int k = 2 * half; k < 2 * half + 2; ++k) {
        const int key = 16 * (k & 1) + value_key<RB>(lane & 15);
#pragma unroll
        for (int ch = 0; ch < NC; ++ch)
          *(u32x4*)(vl + key * RB + (((uint32_t)(g * NC + ch) ^ swizzle_values<RB>(key)) << 4)) =
              fp4_bf16x8(vreg[k][ch], fp4_scale(vs[k][8 * ch / kFp4Group]));
        if (more) fetch_value(mine, k);
      }
      wave_lds_order();
      u32x4 ph[PARTS][1][QB];
#pragma unroll
      for (int m = 0; m < PARTS; ++m)
#pragma unroll
        for (int q = 0; q < QB; ++q) ph[m][0][q] = p[m][half][q];
      if (masked) weigh<Tag, RB, true>(vl, vb, ph, rs, odd);
      else weigh<Tag, RB, false>(vl, vb, ph, rs, odd);
    }
  }
  if (__any(odd != 0)) {
    // the keys of this wave's masked tiles
#pragma unroll 1
    for (int k = k_begin + wave * TK; k < k_end; k += 4 * TK)
#pragma unroll 1
      for (int u = k; u < k + TK && u < k_end && k + TK - 1 > before; ++u) {
        bool sees[QB];
#pragma unroll
        for (int q = 0; q < QB; ++q) sees[q] = u <= seen[q];
        add_nan_groups(fa.Vs + (int64_t)cache_row(a.pb, b, a.Hk, kh, u) * groups, a.D, sees, rs);
      }
  }
  join_waves<DT16, QB>(rs, lds, fp4_rows_lds<DT, QB>(), wave, lane, c);
  if (wave == 0)
    finish_rows<T, DT, QB, EXACT>(a, part, rs, row, seen, rows, sq.s0, kh, range,
                                  ((int64_t)b * a.Hk + kh) * (16 * QB), ranges == 1, c, lane);
}

}  // namespace ssn
