// Paged attention of few rows (a sequence's next token, or a few): a block of
// 4 waves owns a range of the keys of one sequence and key head; its waves take
// the range's tiles in turn, all with the same 16 QB rows, and join their
// results in LDS at the end.
//
// What bounds it: reading the cache.  64 single tokens over caches of 1 to 4096
// keys (40 / 8 heads of 128, bf16) take 100 us (5.5 TB/s), four over 100000 to
// 131072 keys 316 us (6.7 TB/s; a large copy moves 4.6), and the join 7 to 10 us
// more.  The matrix cores are used with 16 rows where a group has 4 or 5 heads:
// they are busy 6 % of the time, and each key is read once for the group.
//
// bf16 probabilities are multiplied in two parts (their rounding and what it left),
// which the matrix cores have room for: single tokens with heads of 64 and 128 take
// the same time with one part (64 caches 107 us, four long ones 325), 30 rows of
// heads of 128 over 16 caches of up to 8192 keys 128 us for 119, 7 rows of heads
// of 256 136 for 129.  Of the outputs' error against float64 only their own
// rounding is left (0.0017; with one part up to 0.0023).
#pragma once

#include "attn_tiles.h"

namespace ssn {

template <typename T, int DT, int QB>
constexpr int rows_join() { return DT / 16 * QB * kWave * 16; }      // bytes of a wave's O
template <typename T, int DT, int QB>
constexpr int rows_lds() {
  const int tiles = 4 * Mma<T>::kKeys * DT * (int)sizeof(T), join = 2 * rows_join<T, DT, QB>();
  return (tiles > join ? tiles : join) + 4 * QB * kWave * 4;         // and m, l of two waves
}

template <typename T, int DT, int QB, bool EXACT>
__device__ __forceinline__ void rows_block(const AttnArgs& a, const AttnPart& part, int few, int id, char* lds) {
  using M = Mma<T>;
  constexpr int RB = DT * (int)sizeof(T), TK = M::kKeys, NKB = TK / 16, NC = RB / 64, DT16 = DT / 16;
  constexpr int CH = RB / 16, RPI = kWave / CH, NI = TK / RPI;
  constexpr int kTile = TK * RB, kJoin = rows_join<T, DT, QB>();
  float(*joint)[2][QB][kWave] = (float(*)[2][QB][kWave])(lds + rows_lds<T, DT, QB>() - 4 * QB * kWave * 4);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kh = id % a.Hk, rest = id / a.Hk, b = rest % a.pb.B, range = rest / a.pb.B;
  const Sequence sq = sequence_of(a.pb, b);
  const int n = sq.s1 - sq.s0, rows = n * a.G, keys = sq.len;
  if (rows == 0 || rows > few) return;
  const int ranges = key_ranges(keys, part.chunk);
  if (range >= ranges) return;
  const int bytes = a.D * (int)sizeof(T), before = sq.len - n;
  const int k_begin = range * part.chunk;
  const int k_end = range_end(k_begin, part.chunk, keys);

  int row[QB], seen[QB];
  u32x4 qf[QB][NC];
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    row[q] = q * 16 + (lane & 15);
    const int r = row[q] < rows ? row[q] : rows - 1, token = r / a.G;
    seen[q] = before + token;
    load_query<NC, EXACT>((const char*)a.Q + ((sq.s0 + token) * a.ldq + (int64_t)(kh * a.G + r % a.G) * a.D) * (int)sizeof(T),
                          bytes, lane, sign_bits<T>(a.scale), a.scale == 0.f, qf[q]);
  }
  const float c = (a.scale == 0.f ? 1.f : fabsf(a.scale)) * kLog2e;

  // A tile's keys go straight to registers as A operands (16 rows x 64 bytes
  // an instruction); its values whole rows at a time, through the wave's part
  // of LDS.  The next tile's loads are issued as soon as this one's registers
  // are free, and the blocks of a compute unit cover each other's waits.  A key
  // is read once by one block: without a place in the caches (non-temporal loads)
  // four caches of 131072 keys take 323 us (6.5 TB/s) instead of 366.
  char* vl = lds + wave * kTile;
  u32x4 kreg[NKB][NC], vreg[NI];
  auto key_slot = [&](int t) {
    const int key = t + (lane & (TK - 1));
    return find_slot(a.pb, b, key < keys ? key : keys - 1);
  };
  auto fetch = [&](const Slot& s) {
    const uint32_t mine = slot_row(a.pb, s, a.Hk, kh);
#pragma unroll
    for (int k = 0; k < NKB; ++k) {
      const char* p = (const char*)a.Kc + (int64_t)(uint32_t)__shfl((int)mine, 16 * k + (lane & 15), kWave) * bytes;
#pragma unroll
      for (int ch = 0; ch < NC; ++ch) {
        const int at = ch * 64 + (lane >> 4) * 16;
        kreg[k][ch] = u32x4{0, 0, 0, 0};
        if (EXACT || at < bytes) kreg[k][ch] = __builtin_nontemporal_load((const u32x4*)(p + at));
      }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int at = (lane % CH) * 16;
      const char* p = (const char*)a.Vc + (int64_t)(uint32_t)__shfl((int)mine, i * RPI + lane / CH, kWave) * bytes;
      vreg[i] = u32x4{0, 0, 0, 0};
      if (EXACT || at < bytes) vreg[i] = __builtin_nontemporal_load((const u32x4*)(p + at));
    }
  };
  uint32_t vb[M::kBases];
#pragma unroll
  for (int i = 0; i < M::kBases; ++i) vb[i] = M::template vbase<RB>(lane, i);

  RowState<DT16, QB> rs;
  rs.clear();
  int t = k_begin + wave * TK;
  uint32_t odd = 0;
  Slot next = {0, 0};
  if (t < k_end) {
    fetch(key_slot(t));
    if (t + 4 * TK < k_end) next = key_slot(t + 4 * TK);
  }
  for (; t < k_end; t += 4 * TK) {
    const bool masked = t + TK - 1 > before;           // row 0 does not see it all
    wave_lds_order();
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int r = i * RPI + lane / CH;
      *(u32x4*)(vl + r * RB + (((uint32_t)(lane % CH) ^ swizzle_values<RB>(r)) << 4)) = vreg[i];
    }
    wave_lds_order();
    f32x4 s[NKB][QB];
#pragma unroll
    for (int k = 0; k < NKB; ++k)
#pragma unroll
      for (int q = 0; q < QB; ++q) {
        s[k][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ch = 0; ch < NC; ++ch) s[k][q] = M::mma(kreg[k][ch], qf[q][ch], s[k][q]);
      }
    if (t + 4 * TK < k_end) {
      fetch(next);
      if (t + 8 * TK < k_end) next = key_slot(t + 8 * TK);
    }
    u32x4 p[M::kParts][NKB / M::kTiles][QB];
    if (masked) {
#pragma unroll
      for (int q = 0; q < QB; ++q)
#pragma unroll
        for (int k = 0; k < NKB; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * k + 4 * (lane >> 4) + i > seen[q] - t) s[k][q][i] = kNegInf;
      softmax_step<T, M::kParts>(s, rs, c, p);
      weigh<T, RB, true>(vl, vb, p, rs, odd);
    } else {
      softmax_step<T, M::kParts>(s, rs, c, p);
      weigh<T, RB, false>(vl, vb, p, rs, odd);
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
        add_not_finite<T, DT16, QB>((const T*)a.Vc + (int64_t)cache_row(a.pb, b, a.Hk, kh, u) * a.D, a.D, sees, rs);
      }
  }

  // Join the waves: 2 and 3 into 0 and 1, then 1 into 0.
#pragma unroll
  for (int step = 2; step >= 1; step >>= 1) {
    __syncthreads();
    if (wave >= step && wave < 2 * step) {
#pragma unroll
      for (int q = 0; q < QB; ++q) {
        joint[wave - step][0][q][lane] = rs.m[q];
        joint[wave - step][1][q][lane] = rs.l[q];
#pragma unroll
        for (int d = 0; d < DT16; ++d)
          *(f32x4*)(lds + (wave - step) * kJoin + ((d * QB + q) * kWave + lane) * 16) = rs.o[d][q];
      }
    }
    __syncthreads();
    if (wave < step) {
#pragma unroll
      for (int q = 0; q < QB; ++q) {
        const float m2 = joint[wave][0][q][lane], l2 = joint[wave][1][q][lane];
        const float m = fmaxf(rs.m[q], m2), base = m == kNegInf ? 0.f : m;
        const float w1 = __builtin_amdgcn_exp2f((rs.m[q] - base) * c), w2 = __builtin_amdgcn_exp2f((m2 - base) * c);
        rs.m[q] = m;
        rs.l[q] = rs.l[q] * w1 + l2 * w2;
#pragma unroll
        for (int d = 0; d < DT16; ++d)
          rs.o[d][q] = rs.o[d][q] * w1 + *(const f32x4*)(lds + wave * kJoin + ((d * QB + q) * kWave + lane) * 16) * w2;
      }
    }
  }
  if (wave == 0)
    finish_rows<T, DT, QB, EXACT>(a, part, rs, row, seen, rows, sq.s0, kh, range,
                                  ((int64_t)b * a.Hk + kh) * (16 * QB), ranges == 1, c, lane);
}

}  // namespace ssn
