// Paged attention of many rows: a block of 4 waves owns a tile of rows of one
// sequence and key head (64 QB rows, 16 QB to a wave) and walks the keys the
// tile sees, 64 (or 32) at a time through LDS, double buffered.  Rows of all the
// heads of a group share the tile, so a key is read once for the group.
//
// What bounds it: the compute.  A prompt of 4096 tokens (40 / 8 heads of 128, bf16)
// takes 171 us, 1010 TFLOP/s where a large matrix product reaches 1260 to 1365, and
// four of them 680 us, 1010.  Of that the matrix cores are busy 40 %, the vector
// units issue 45 %; without the tile loads it would take 12 % less, without the
// exponentials 4 %, without barriers the same: the rest is the latency of
// LDS reads, products and probabilities one after the other in a wave, two waves
// to a SIMD.  Measured and not kept: scores a step ahead of the probabilities (+-5
// %), values read before the scores (+-2 %), 32-key tiles with three blocks to a
// compute unit (spills), blocks of 8 waves (1 to 5 % faster at 4096 tokens and
// more, 10 % slower below).
//
// bf16 probabilities are rounded once for the product with V.  What the rounding
// leaves as a second product, as the rows kernel has it, costs more here than it
// gives: prompts of 1024 / 2048 / 4096 tokens take 37 / 89 / 256 us with it and 29 /
// 60 / 178 without, 512 tokens over 32768 keys 531 and 370.  The outputs' error
// against float64 is 0.0022 (4096 tokens), 0.0016 with it, which is their own rounding.
#pragma once

#include "attn_mma.h"

namespace ssn {

// 16 bytes of every active lane, from its own address to LDS: lane i's to `to` +
// 16 i (`to` the same in the wave).  In assembly, because the compiler waits for
// all such loads before the next ds_read_b64_tr_b16, also where that reads
// another buffer (2048-token prompt 62 -> 59 us, 4 of 4096 686 -> 674); there is
// no output register.  Readers wait for vmcnt and pass a barrier.
__device__ __forceinline__ void load_to_lds(const char* from, const char* to) {
  const uint32_t at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)to;
  // (one wait state between a scalar write of m0 and its use by the load)
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "{m0}"(at) : "memory");
}

// The launch's row tiles by their place in their sequence, the last places first:
// of prompts without cached keys before them, those that see the most keys.  (What
// is cached before a chunk is not looked at.)  Up to kCounted sequences every block
// counts the tiles of each (four a lane) and ranks them over all; past that
// sequence b has the numbers from starts[b] * G / BM + b on, which leaves ceil(rows
// / BM) to each, some numbers name none, and the last goes first.
constexpr int kCounted = 256;
__device__ __forceinline__ int first_slot(const PagedBatch& pb, int b, int G, int BM) {
  return (int)((int64_t)clampi(pb.starts[b], 0, pb.N) * G / BM) + b;
}
__device__ __forceinline__ int tiles_of(const PagedBatch& pb, int b, int G, int BM, int few) {
  if (b >= pb.B) return 0;
  const int s0 = clampi(pb.starts[b], 0, pb.N), rows = (clampi(pb.starts[b + 1], s0, pb.N) - s0) * G;
  return rows > few ? (rows + BM - 1) / BM : 0;
}
struct TileCount {
  int mine[kCounted / kWave];     // tiles of sequence 64 c + lane
  int total, most;
  // The sum over a wave of values below 2^bits, in scalar registers: bit by bit,
  // by the lanes that have it.
  __device__ __forceinline__ static int wave_total(int v, int bits) {
    int n = 0;
    for (int k = 0; k < bits; ++k) n += __popcll(__ballot((v >> k) & 1)) << k;
    return n;
  }
  __device__ __forceinline__ static int bits_of(int v) { return 32 - __clz(v); }
  __device__ __forceinline__ void count(const PagedBatch& pb, int G, int BM, int few, int slots) {
    total = slots;
    if (pb.B > kCounted) return;
    if (pb.B == 1) {
      total = tiles_of(pb, 0, G, BM, few);
      return;
    }
#pragma unroll
    for (int c = 0; c < kCounted / kWave; ++c)
      mine[c] = 64 * c < pb.B ? tiles_of(pb, 64 * c + (threadIdx.x & 63), G, BM, few) : 0;
    most = 0;
    for (int k = bits_of(slots) - 1; k >= 0; --k) {
      const int up = (most | (1 << k)) >> k;
      bool has = false;
#pragma unroll
      for (int c = 0; c < kCounted / kWave; ++c) has |= (mine[c] >> k) == up;
      if (__any(has)) most |= 1 << k;
    }
    // contents past the contract may count more than the grid has
    const int n = from_level(0);
    total = n < slots ? n : slots;
  }
  // Tiles that are number `level` or later of their sequence.
  __device__ __forceinline__ int from_level(int level) const {
    int n = 0;
#pragma unroll
    for (int c = 0; c < kCounted / kWave; ++c) n += mine[c] > level ? mine[c] - level : 0;
    return wave_total(n, bits_of(most) + 2);
  }
  // Sequence and tile of rank i < total; false: none.
  __device__ __forceinline__ bool find(const PagedBatch& pb, int G, int BM, int few, int i, int& b, int& tile) const {
    if (pb.B > kCounted) {
      const int slot = total - 1 - i;
      b = last_at_most(pb.B, slot, [&](int x) { return first_slot(pb, x, G, BM); });
      tile = slot - first_slot(pb, b, G, BM);
      return tile >= 0 && tile < tiles_of(pb, b, G, BM, few);
    }
    if (pb.B == 1) {
      b = 0;
      tile = total - 1 - i;
      return true;
    }
    int lo = 0, hi = most;          // from_level(lo) > i >= from_level(hi)
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (from_level(mid) > i) lo = mid;
      else hi = mid;
    }
    tile = lo;
    int nth = i - from_level(lo + 1);
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int c = 0; c < kCounted / kWave; ++c) {
      const uint64_t has = __ballot(mine[c] > lo);
      const int n = __popcll(has), rank = __popcll(has & (((uint64_t)1 << lane) - 1));
      if (nth < n) {
        b = 64 * c + __ffsll((unsigned long long)__ballot(mine[c] > lo && rank == nth)) - 1;
        return true;
      }
      nth -= n;
    }
    return false;
  }
};

// A compute unit gets one block of the first round and one of the second: a
// long and a short one.
constexpr int kUnits = 256;
__device__ __forceinline__ int balanced_order(int i, int slots, int Hk) {
  const int round = kUnits / Hk;
  if (i < round || i >= 2 * round || slots < 2 * round) return i;
  return 3 * round - 1 - i;
}

// What a wave does with its rows when its keys are done: the result, or its
// part of it.  Row r of the sequence's rows is token r / G, head r % G.
template <typename T, int DT, int QB, bool EXACT>
__device__ __forceinline__ void finish_rows(const AttnArgs& a, const AttnPart& part, RowState<DT / 16, QB>& rs,
                                            const int (&row)[QB], const int (&seen)[QB], int rows, int s0,
                                            int kh, int range, int64_t stage0, bool whole, float c, int lane) {
  const int h4 = 4 * (lane >> 4);
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    const float l = column_sum(rs.l[q]);
    if (row[q] >= rows) continue;
    const int token = s0 + row[q] / a.G, head = kh * a.G + row[q] % a.G;
    const int64_t at = (int64_t)token * a.Hq + head;
    if (whole) {
      // 0 / 0 where every score a row sees is -inf; a row that sees nothing is zero
      const float inv = seen[q] < 0 ? 0.f : 1.f / l;
      T* out = (T*)a.O + token * a.ldo + (int64_t)head * a.D;
#pragma unroll
      for (int d = 0; d < DT / 16; ++d)
        if (EXACT || 16 * d + h4 < a.D) store4(out + 16 * d + h4, rs.o[d][q] * inv);
      if (a.lse && lane < 16)
        a.lse[at] = seen[q] < 0 ? kNegInf : (rs.m[q] * c + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
    } else {
      // (stage0 < 0: rows staged by token and head, else from there in row order)
      const int64_t to = range * part.stage_rows + (stage0 < 0 ? at : stage0 + row[q]);
      float* out = part.o + to * a.D;
#pragma unroll
      for (int d = 0; d < DT / 16; ++d)
        if (EXACT || 16 * d + h4 < a.D) *(f32x4*)(out + 16 * d + h4) = rs.o[d][q];
      if (lane < 16) {
        float* ml = part.ml + 2 * to;
        ml[0] = rs.m[q] * c;
        ml[1] = l;
      }
    }
  }
}

// Q^T of 16 rows as B operands: lane's row is lane % 16, chunk c of 64 bytes
// at lane / 16.  `flip`: the sign bits of a negative scale.
template <int NC, bool EXACT>
__device__ __forceinline__ void load_query(const char* p, int bytes, int lane, uint32_t flip, bool zero,
                                           u32x4 (&q)[NC]) {
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int at = c * 64 + (lane >> 4) * 16;
    u32x4 v = {0, 0, 0, 0};
    if (!zero && (EXACT || at < bytes)) v = *(const u32x4*)(p + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) q[c][i] = v[i] ^ flip;
  }
}
template <typename T>
__device__ __forceinline__ uint32_t sign_bits(float scale) {
  return scale < 0.f ? (sizeof(T) == 2 ? 0x80008000u : 0x80000000u) : 0u;
}

template <typename T, int DT>
constexpr int tile_keys() { return DT * (int)sizeof(T) <= 256 ? 64 : 32; }
template <typename T, int DT>
constexpr int tiles_lds() { return 4 * tile_keys<T, DT>() * DT * (int)sizeof(T); }

template <typename T, int DT, int QB, bool EXACT>
__device__ __forceinline__ void tiles_block(const AttnArgs& a, const AttnPart& part, int few, const TileCount& count,
                                            int id, char* mem) {
  using M = Mma<T>;
  constexpr int RB = DT * (int)sizeof(T), TK = tile_keys<T, DT>(), NC = RB / 64;
  // keys whose scores are held at a time
  constexpr int SK = 32, NKB = SK / 16;
  constexpr int CH = RB / 16, RPI = kWave / CH, NI = TK / RPI / 4, BM = 64 * QB;
  char(*lds)[2][TK * RB] = (char(*)[2][TK * RB])mem;      // [buffer][K, V]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kh = id % a.Hk, rest = id / a.Hk;
  if (count.total <= 0) return;
  const int range = rest / count.total;
  int b, tile;
  if (range >= part.ranges ||
      !count.find(a.pb, a.G, BM, few, balanced_order(rest % count.total, count.total, a.Hk), b, tile))
    return;
  const Sequence sq = sequence_of(a.pb, b);
  const int n = sq.s1 - sq.s0, rows = n * a.G, r0 = tile * BM;
  const int before = sq.len - n;                           // position of the sequence's token 0
  const int last = r0 + BM < rows ? r0 + BM - 1 : rows - 1;
  const int keys = before + last / a.G + 1;                // that the tile sees
  const int ranges = key_ranges(keys, part.chunk);
  if (range >= ranges) return;

  const int bytes = a.D * (int)sizeof(T);
  int row[QB], seen[QB];
  u32x4 qf[QB][NC];
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    row[q] = r0 + wave * (16 * QB) + q * 16 + (lane & 15);
    const int r = row[q] < rows ? row[q] : rows - 1, token = r / a.G;
    seen[q] = before + token;
    load_query<NC, EXACT>((const char*)a.Q + ((sq.s0 + token) * a.ldq + (int64_t)(kh * a.G + r % a.G) * a.D) * (int)sizeof(T),
                          bytes, lane, sign_bits<T>(a.scale), a.scale == 0.f, qf[q]);
  }
  // a scale of zero: zero queries, any other scale
  const float c = (a.scale == 0.f ? 1.f : fabsf(a.scale)) * kLog2e;
  const int wave_last = r0 + (wave + 1) * (16 * QB) - 1;
  const int seen_hi = before + (wave_last < rows ? wave_last : rows - 1) / a.G;

  const int t0 = range * (part.chunk / TK);
  const int all = (keys + TK - 1) / TK, t1 = all < t0 + part.chunk / TK ? all : t0 + part.chunk / TK;

  // Loads of a tile: straight to LDS, 16 bytes a lane, RPI rows to an
  // instruction; the chunk a lane fetches is the one its position holds.  Rows
  // past the last key repeat it (their scores are masked).
  auto key_slot = [&](int t) {
    const int key = t * TK + (lane & (TK - 1));
    return find_slot(a.pb, b, key < keys ? key : keys - 1);
  };
  auto fetch = [&](const Slot& s, int buf) {
    const uint32_t mine = slot_row(a.pb, s, a.Hk, kh);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int base = (i * 4 + wave) * RPI, r = base + lane / CH;
      const uint32_t kc = (uint32_t)(lane % CH) ^ swizzle_keys<RB>(r), vc = (uint32_t)(lane % CH) ^ swizzle_values<RB>(r);
      const int64_t src = (int64_t)(uint32_t)__shfl((int)mine, r, kWave) * bytes;
      if (EXACT || (int)kc * 16 < bytes)
        load_to_lds((const char*)a.Kc + src + kc * 16, &lds[buf][0][base * RB]);
      if (EXACT || (int)vc * 16 < bytes)
        load_to_lds((const char*)a.Vc + src + vc * 16, &lds[buf][1][base * RB]);
    }
  };
  if constexpr (!EXACT) {
    // chunks past a row's end are never loaded: zero once
    for (int i = threadIdx.x * 16; i < tiles_lds<T, DT>(); i += 256 * 16) *(u32x4*)(mem + i) = u32x4{0, 0, 0, 0};
    __syncthreads();
  }

  uint32_t vb[M::kBases];
#pragma unroll
  for (int i = 0; i < M::kBases; ++i) vb[i] = M::template vbase<RB>(lane, i);
  const uint32_t kb0 = (lane & 15) * RB + (((uint32_t)(lane >> 4) ^ swizzle_keys<RB>(lane & 15)) << 4);

  RowState<DT / 16, QB> rs;
  rs.clear();
  uint32_t odd = 0;
  Slot next = {0, 0};
  if (t0 < t1) {
    fetch(key_slot(t0), 0);
    if (t0 + 1 < t1) next = key_slot(t0 + 1);
  }
  auto arrive = [&](int t) {
    // this wave's part of tile t has arrived; past the barrier everyone's has,
    // and everyone is done with tile t - 1
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (t + 1 < t1) fetch(next, (t + 1 - t0) & 1);
    if (t + 2 < t1) next = key_slot(t + 2);
  };
  // The widest tiles ask for the matrix cores first (s_setprio), so that of a
  // SIMD's two waves one multiplies while the other exponentiates: 4 % at 192
  // rows (8192-token prompt 698 -> 679 us), nothing below.
  constexpr bool kFirst = QB == 3;
  auto scores = [&](const char* kl, f32x4 (&s)[NKB][QB]) {
#pragma unroll
    for (int k = 0; k < NKB; ++k) {
#pragma unroll
      for (int q = 0; q < QB; ++q) s[k][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ch = 0; ch < NC; ++ch) {
        const u32x4 kf = *(const u32x4*)(kl + (kb0 ^ (uint32_t)(ch * 64)) + k * 16 * RB);
#pragma unroll
        for (int q = 0; q < QB; ++q) s[k][q] = M::mma(kf, qf[q][ch], s[k][q]);
      }
    }
  };
  // Tiles that every row of the block sees, then the others.  (Two loops: one
  // with both cases keeps O in two sets of registers.)
  const int open = (before + r0 / a.G + 1) / TK, t_open = open < t0 ? t0 : (open < t1 ? open : t1);
  int t = t0;
  for (; t < t_open; ++t) {
    arrive(t);
    const char *kl = lds[(t - t0) & 1][0], *vl = lds[(t - t0) & 1][1];
#pragma unroll
    for (int u = 0; u < TK; u += SK) {
      f32x4 s[NKB][QB];
      if constexpr (kFirst) __builtin_amdgcn_s_setprio(1);
      scores(kl + u * RB, s);
      if constexpr (kFirst) __builtin_amdgcn_s_setprio(0);
      u32x4 p[1][NKB / M::kTiles][QB];
      softmax_step<T, 1>(s, rs, c, p);
      if constexpr (kFirst) __builtin_amdgcn_s_setprio(1);
      weigh<T, RB, false>(vl + u * RB, vb, p, rs, odd);
      if constexpr (kFirst) __builtin_amdgcn_s_setprio(0);
    }
  }
  for (; t < t1; ++t) {
    arrive(t);
    const char *kl = lds[(t - t0) & 1][0], *vl = lds[(t - t0) & 1][1];
#pragma unroll 1
    for (int u = 0; u < TK; u += SK) {
      const int k0 = t * TK + u;
      if (k0 > seen_hi) break;
      f32x4 s[NKB][QB];
      scores(kl + u * RB, s);
#pragma unroll
      for (int q = 0; q < QB; ++q)
#pragma unroll
        for (int k = 0; k < NKB; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * k + 4 * (lane >> 4) + i > seen[q] - k0) s[k][q][i] = kNegInf;
      u32x4 p[1][NKB / M::kTiles][QB];
      softmax_step<T, 1>(s, rs, c, p);
      weigh<T, RB, true>(vl + u * RB, vb, p, rs, odd);
    }
  }
  if (__any(odd != 0)) {
    // the keys of the masked tiles
#pragma unroll 1
    for (int k = t_open * TK; k < t1 * TK && k <= seen_hi; ++k) {
      bool sees[QB];
#pragma unroll
      for (int q = 0; q < QB; ++q) sees[q] = k <= seen[q];
      add_not_finite<T, DT / 16, QB>((const T*)a.Vc + (int64_t)cache_row(a.pb, b, a.Hk, kh, k) * a.D, a.D, sees, rs);
    }
  }
  finish_rows<T, DT, QB, EXACT>(a, part, rs, row, seen, rows, sq.s0, kh, range, -1, ranges == 1, c, lane);
}

}  // namespace ssn
