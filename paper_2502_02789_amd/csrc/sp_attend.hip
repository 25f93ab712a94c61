// sp_attend: attention of new tokens over a (paged, bf16, E4M3 or MXFP4) cache, the keys of a shared prefix read once for a group.
//
// One launch takes every piece of the plan (sp_attend_plan.h), a workgroup of eight waves (d = 128: one on a compute unit; four
// and three of them, d = 64) a stretch of pieces for one KV head.  Two forms:
//   few rows (<= 32: single tokens or several, their heads)   bound by reading keys and values.  Each wave walks over 32-key tiles of
//     its own through LDS, with one or two 16x16 tiles of logits twice; nothing is shared before the end, and every wave has its next
//     tile of keys and of values in flight.  64 sequences of 4096 bf16 keys, H_kv 8, d 128: 177 us, 6.1 TB/s; in 8 bits 104 us, 5.2 TB/s:
//     there the waves wait for more than half of their time, the LDS is busy for 41 % (half of it the banks that the widened chunks meet in), the
//     vector ALUs for 20 %.  Two tiles of rows instead of a large block, whose matrix tiles they would fill to a tenth: 14 to 27 % less
//     time; 32 sequences of 1K-3K keys and 2 to 8 tokens of 4 heads: 62 us, 4.5 TB/s.
//     4-bit caches have a form of their own (below, few rows, 4-bit keys and values): 64-key tiles, keys from registers to the matrix cores without LDS.
//     64 sequences of 1K-4K keys 44 us, 128K keys 31 us (H 64), join and launches, 6 to 7 us, among them; the kernel alone reads 3.8 and 5.3 TB/s.  Loads alone,
//     with the same start and join, take 36 and 29 us, 3.6 of the 36 for the scales.
//   many rows (<= 256, d = 64 128: prompts, prefixes of groups)  bound by the matrix cores and the vector work between their products.
//     The waves share 64-key tiles in LDS (two buffers, one barrier a tile; a second tile on its way in registers), each has 32 rows.
//     6592 tokens, H 64, d 128, causal: 690-720 us, 1.0 PFLOP/s (matrix cores busy for 48 % of the clocks, vector ALUs for 43 %, at 1.93 GHz); eight
//     prompts of 300-3000 tokens, H 32, d 64: 119 us, 0.6 (28 and 58 %).
//     (Blocks of at most 128 rows with the waves' halves on alternate tiles and their sums added at the end: 5 % slower, and single tokens
//     3 % by the mere size of the kernel.)
// Both compute S^T = K Q^T, so that a lane has the logits of one row, turn the weights exp2(s - m) into bf16 in place -- the order
// of keys in a matrix product's sum is free, and is chosen so that a lane's logits are its own operand of O^T = V^T P^T -- and read
// V^T out of row-major LDS tiles with the transposing LDS read.  Logits, maxima, sums and O are fp32.  A weight is rounded to bf16, by 2^-8 of
// itself at most, because a product of the matrix cores takes both operands of one type and the values are bf16; a second product with what the
// rounding left would make that error 2^-16 and half as many products again.  The sum of weights is that of the unrounded ones, so that the lse keeps the
// accuracy of fp32; out is off by the mean of the weights' roundings: 0.0023 of its size in all for 64 sequences of 1K-4K keys, where its own
// rounding to bf16 makes 0.0017.  The running maximum m follows the logits only
// where one exceeds it by more than 8 (weights stay below 2^8), so sums are rarely rescaled.
// Compiled on the assumption that there are no NaNs; those that mark invalid rows are written as bit patterns.
// (Nothing here may need scratch memory: workgroups that do are dispatched later, 64 single tokens 5 % slower with 20 bytes of it.)
#include "sp_attend_internal.h"
#include "sp_lds.h"

#include <type_traits>

namespace sp {

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr uint32_t kNanF32 = 0x7fc00000u;
constexpr int kNanBf16 = 0x7fc0;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kSlack = 8.f;   // logits (log2) may exceed the running maximum by this much
constexpr int kTileKeys = 64;   // many rows
constexpr int kAhead = 6;       // operands that are read before the first product that takes one

// kinds of instructions, for __builtin_amdgcn_sched_group_barrier
constexpr int kSchedValu = 0x2, kSchedMfma = 0x8, kSchedLdsRead = 0x100;

// Place of 16-byte chunk c of row r in a tile of rows of C chunks, permuted so that neither the operand reads (16 or 32 rows,
// one or two chunks) nor the transposing reads (4 or 8 rows, 2 or 4 chunks) meet in a bank more often than they must.
template <int C>
__device__ __forceinline__ int swizzled(int r, int c) {
  if constexpr (C == 16) return c ^ (((r & 3) << 2) | ((r >> 2) & 3));
  else return c ^ ((((r >> 1) & 1) << 2) | ((r >> 2) & 3));
}

__device__ __forceinline__ s16x4 lds_read_tr(const char* at) {
  typedef __attribute__((address_space(3))) s16x4 lds_t;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)at);
}
__device__ __forceinline__ bf16x8 join8(s16x4 a, s16x4 b) {
  typedef __attribute__((ext_vector_type(8))) short s16x8;
  const s16x8 v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, v);
}

// 16 E4M3 codes -> 16 bf16 values (exact)
__device__ __forceinline__ void widen_e4m3(const u32x4 w, u32x4& lo, u32x4& hi) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    lo[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, false));
    lo[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, true));
    hi[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 + i], 1.0f, false));
    hi[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 + i], 1.0f, true));
  }
}

// 2 N E2M1 codes and their E8M0 scale -> as many bf16 values (exact)
template <int N>
__device__ __forceinline__ void widen_e2m1(const uint32_t (&w)[N / 4], uint32_t scale, uint32_t (&out)[N]) {
  const float s = __uint_as_float(scale << 23);
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    out[4 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 0));
    out[4 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 1));
    out[4 * i + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 2));
    out[4 * i + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], s, 3));
  }
}

// Where the rows of a piece's keys lie.  Tiles start at multiples of 8 keys and pages hold multiples of 8, so the 8 keys of an
// octet lie at one stride from one base, formed in scalar registers, once for all lanes of a wave.  The page numbers of a tile's
// keys come in a vector register, a lane each, requested a tile ahead and before that tile's loads, so that nothing waits for them
// that does not wait for older loads anyway.  (Scalar loads share a counter with the LDS reads, whose waits then wait for both:
// 3 % slower for 64 new tokens behind 128K keys.  64 pages at a time, asked for when needed, instead of a tile's: 4 % slower
// for 64 sequences of 4096 8-bit keys.)
template <bool PAGED>
struct KeyRows {
  const int32_t* table;
  int lg_page, first, last_key, lane;
  uint32_t last, pages;
  int32_t ts;
  int64_t ps;
  // tile: the first that will be asked for
  __device__ __forceinline__ KeyRows(const AttendDev& p, const AttendUnit& u, int l, int tile) {
    ts = p.c_ts; ps = p.c_ps; lg_page = p.lg_page; last_key = u.k1 - 1; lane = l;
    first = PAGED ? 0 : u.seq;
    last = PAGED ? p.last_page : p.last_row;
    table = PAGED ? p.table + (int64_t)u.seq * p.blocks_per_seq : nullptr;
    if (u.k0 < u.k1) ahead(tile);
  }
  // asks for the pages of the tile that begins at `tile`
  __device__ __forceinline__ void ahead(int tile) {
    if constexpr (PAGED) pages = (uint32_t)table[min(tile + lane, last_key) >> lg_page];
  }
  // first key of the octet that row r (wave-uniform) of a tile lies in, no further than the last key's
  __device__ __forceinline__ int octet(int tile, int r) const { return min(tile + r, last_key) & ~7; }
  // byte offset of that key.  Nothing outside the pool is addressed, a bad page is noted.
  __device__ __forceinline__ int64_t base(int octet, int r, uint32_t& bad) const {
    if constexpr (PAGED) {
      const uint32_t entry = (uint32_t)__builtin_amdgcn_readlane((int)pages, r & ~7);
      bad |= entry > last;
      return (int64_t)min(entry, last) * ps + (int64_t)(octet & ((1 << lg_page) - 1)) * ts;
    } else {
      return (int64_t)min((uint32_t)(first + octet), last) * ts;
    }
  }
  // ... of `key` behind the octet's first: of the last key, where it lies beyond that (its weight is zero there, and it is finite)
  __device__ __forceinline__ uint32_t within(int octet, int key) const {
    if constexpr (PAGED) return (uint32_t)(min(key, last_key) - octet) * (uint32_t)ts;
    else return (min((uint32_t)(first + min(key, last_key)), last) - min((uint32_t)(first + octet), last)) * (uint32_t)ts;
  }
};

// The logits' factor: its magnitude; its sign, or a zero, goes into the queries, so that maxima in front of it stay right
__device__ __forceinline__ float key_factor(const AttendDev& p, int g, uint32_t& flip, uint32_t& keep) {
  float c = p.k_scale ? p.scale_log2 * p.k_scale[g] : p.scale_log2;
  flip = c < 0.f ? 0x80008000u : 0u;
  keep = c == 0.f ? 0u : 0xffffffffu;
  return c == 0.f ? 1.f : fabsf(c);
}

// threadIdx.x, as a value of its own for every piece: what is computed from it is not kept in registers across the loop over pieces
__device__ __forceinline__ int thread_of_piece() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

struct RowPlace { int token, h; };
__device__ __forceinline__ RowPlace row_place(const AttendDev& p, int flat, int g) {
  RowPlace r;
  r.token = flat / p.G;
  r.h = g * p.G + flat - r.token * p.G;
  return r;
}

// index of row r of a piece among all rows of the workspace
__device__ __forceinline__ int64_t slot_row(const AttendDev& p, int slot, int r, int g) {
  return ((int64_t)(slot + r / kSlotRows) * p.H_kv + g) * kSlotRows + r % kSlotRows;
}

// (the sum of an invalid row is a NaN, as a bit pattern: the compiler takes it that no float is one)
__device__ __forceinline__ void store_stats(const AttendDev& p, int64_t place, float top, float sum, int bad) {
  *reinterpret_cast<uint2*>(p.stats + place) = make_uint2(__float_as_uint(top), bad ? kNanF32 : __float_as_uint(sum));
}

__device__ __forceinline__ void store_values(uint16_t* dst, f32x4 x, bool bad) {  // four of a row
  const uint32_t nan2 = kNanBf16 * 0x10001u;
  const uint2 v = make_uint2(pack_bf16_pair(x[0], x[1]), pack_bf16_pair(x[2], x[3]));
  *reinterpret_cast<uint2*>(dst) = bad ? make_uint2(nan2, nan2) : v;
}
__device__ __forceinline__ void store_lse(const AttendDev& p, int token, int h, float top, float sum, bool bad) {
  const float lse = sum == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
  reinterpret_cast<uint32_t*>(p.lse)[(int64_t)token * p.H + h] = bad ? kNanF32 : __float_as_uint(lse);
}

// ---------------------------------------------------------------- few rows
// One wave's 32-key tile of keys or values on its way from memory to LDS.  A load instruction covers whole rows (256 bytes of
// each of 4 keys, bf16 and d = 128), so that every request is for a whole line.
template <int D, bool FP8>
struct FewTile {
  static constexpr int C = FP8 ? D / 16 : D / 8;  // 16-byte chunks of a stored row
  static constexpr int R = 64 / C;                // rows of a load
  static constexpr int N = 32 / R;                // loads of a tile
  u32x4 x[N];
  __device__ __forceinline__ void load(const char* base, const int64_t (&at)[N], const uint32_t (&in)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(base + at[i] + in[i]));
  }
  __device__ __forceinline__ void store(char* tile, int l) const {  // as bf16
    const int ch = l % C;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = l / C + R * i;
      char* row = tile + r * (D * 2);
      if constexpr (FP8) {
        u32x4 lo, hi;
        widen_e4m3(x[i], lo, hi);
        *reinterpret_cast<u32x4*>(row + swizzled<D / 8>(r, 2 * ch) * 16) = lo;
        *reinterpret_cast<u32x4*>(row + swizzled<D / 8>(r, 2 * ch + 1) * 16) = hi;
      } else {
        *reinterpret_cast<u32x4*>(row + swizzled<D / 8>(r, ch) * 16) = x[i];
      }
    }
  }
};

// The end of a piece of few rows: the sums of its W waves become one.  A lane has, of rows (l & 15) + 16 n, values 16 i + 4 quad .. + 3 of O in
// o[n][i], the maximum and its own part of the sum of weights.
template <int D, int NR>
__device__ __forceinline__ void finish_few(const AttendDev& p, const AttendUnit& u, int g, int W, char* lds, int w, int turn, int l, int tid, uint32_t bad,
                                           const f32x4 (&o)[NR][D / 16], const float (&m)[NR], float (&sum)[NR]) {
  constexpr int DB = D / 16, NW = attend_waves(D);
  const int row = l & 15, quad = l >> 4;
  // every wave's sums in what was its own tile, 16-byte chunks of a row permuted (rows begin in one bank), then one barrier
  constexpr int ROWS = 16 * NR;
  float* const tops = reinterpret_cast<float*>(lds + NW * (2 * 32 * D * 2));  // [wave][ROWS], sums of weights, bad pages
  float* const sums = tops + NW * ROWS;
  uint32_t* const bads = reinterpret_cast<uint32_t*>(sums + NW * ROWS);
  float* const parts = reinterpret_cast<float*>(lds);
  auto chunk_at = [](int r, int ch) { return r * D + 4 * (ch ^ (r & (D / 4 - 1))); };
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    sum[n] += __shfl_xor(sum[n], 16, kWave);
    sum[n] += __shfl_xor(sum[n], 32, kWave);
    const int r = row + 16 * n;
#pragma unroll
    for (int i = 0; i < DB; ++i) *reinterpret_cast<f32x4*>(parts + w * (32 * D) + chunk_at(r, 4 * i + quad)) = o[n][i];
    if (quad == 0) {
      tops[w * ROWS + r] = m[n];
      sums[w * ROWS + r] = sum[n];
    }
  }
  if (l == 0) bads[w] = bad;
  __syncthreads();
  // the piece's waves join them, in their order, 16 lanes to a row
  constexpr int V = D / 16;
  const int w0 = w - turn, lane = tid & 15;
  for (int r = (turn * 64 + l) >> 4; r < u.nr; r += 4 * W) {
    float acc[V], l_all = 0.f, top = tops[w0 * ROWS + r];
    uint32_t any_bad = bads[w0];
    for (int x = w0 + 1; x < w0 + W; ++x) {
      top = fmaxf(top, tops[x * ROWS + r]);
      any_bad |= bads[x];
    }
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
#pragma unroll 2
    for (int x = w0; x < w0 + W; ++x) {
      const float f = fast_exp2(tops[x * ROWS + r] - base);
      l_all += sums[x * ROWS + r] * f;
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const f32x4 part = *reinterpret_cast<const f32x4*>(parts + x * (32 * D) + chunk_at(r, lane * (V / 4) + i / 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i + e] += part[e] * f;
      }
    }
    if (u.slot >= 0) {
      const int64_t place = slot_row(p, u.slot, r, g);
      float* dst = p.sums + place * D + lane * V;
#pragma unroll
      for (int i = 0; i < V; i += 4) *reinterpret_cast<f32x4*>(dst + i) = f32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
      if (lane == 0) store_stats(p, place, top, l_all, any_bad);
      continue;
    }
    const RowPlace to = row_place(p, u.r0 + r, g);
    const float mul = (l_all == 0.f ? 0.f : 1.f / l_all) * (p.v_scale ? p.v_scale[g] : 1.f);
    uint16_t* dst = p.out + to.token * p.o_ts + to.h * p.o_hs + lane * V;
#pragma unroll
    for (int i = 0; i < V; i += 4) store_values(dst + i, f32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]} * mul, any_bad);
    if (lane == 0 && p.lse) store_lse(p, to.token, to.h, top, l_all, any_bad);
  }
}

// NR tiles of 16 rows.  W waves (a power of two of those of the workgroup, side by side) take the piece; the others take others at the
// same time, and all meet at one barrier.
template <int D, bool FP8, bool PAGED, int NR>
__device__ __forceinline__ void attend_few(const AttendDev& p, const AttendUnit& u, int g, int W, char* lds) {
  constexpr int KS = D / 32;          // steps of the product with the queries
  constexpr int DB = D / 16;          // blocks of values
  constexpr int C = D / 8;            // 16-byte chunks of a bf16 row
  using Tile = FewTile<D, FP8>;
  const int tid = thread_of_piece(), w = __builtin_amdgcn_readfirstlane(tid >> 6), turn = w & (W - 1), l = tid & 63, row = l & 15, quad = l >> 4;
  bool mine[NR];
  RowPlace at[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    mine[n] = row + 16 * n < u.nr;
    at[n] = row_place(p, u.r0 + (mine[n] ? row + 16 * n : 0), g);
  }

  int tile = u.k0 < u.k1 ? (u.k0 & ~31) + 32 * turn : u.k1;
  KeyRows<PAGED> rows(p, u, l, tile);
  const char* const kb = p.k + (int64_t)g * p.c_hs;
  const char* const vb = p.v + (int64_t)g * p.c_hs;
  char* const kd = lds + w * (2 * 32 * D * 2);
  char* const vd = kd + 32 * D * 2;
  const int lane_row = l / Tile::C, lane_chunk = (l % Tile::C) * 16;
  uint32_t bad = 0;
  Tile kt, vl;
  int64_t oct_at[Tile::N];
  uint32_t in[Tile::N];
  auto place = [&](int tile) {
    int64_t bases[4];
    int octs[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      octs[j] = rows.octet(tile, 8 * j);
      bases[j] = rows.base(octs[j], 8 * j, bad);
    }
#pragma unroll
    for (int i = 0; i < Tile::N; ++i) {
      constexpr int R = Tile::R;
      const int j = R * i / 8;
      const bool second = R > 8 && lane_row >= 8;  // (a load may cover two octets)
      oct_at[i] = second ? bases[(j + 1) & 3] : bases[j];
      in[i] = rows.within(second ? octs[(j + 1) & 3] : octs[j], tile + R * i + lane_row) + lane_chunk;
    }
    rows.ahead(tile + 32 * W);
  };
  if (tile < u.k1) {
    place(tile);
    kt.load(kb, oct_at, in);
    vl.load(vb, oct_at, in);
  }

  // the queries
  uint32_t flip, keep;
  const float c = key_factor(p, g, flip, keep);
  bf16x8 qf[NR][KS];
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 x = {0, 0, 0, 0};
      if (mine[n]) x = *reinterpret_cast<const u32x4*>(p.q + at[n].token * p.q_ts + at[n].h * p.q_hs + s * 32 + quad * 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = (x[i] ^ flip) & keep;
      qf[n][s] = __builtin_bit_cast(bf16x8, x);
    }
  int limit[NR], least = u.k1;
#pragma unroll
  for (int n = 0; n < NR; ++n) limit[n] = u.k1;
  if (u.off != kNoLimit) {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      if (mine[n]) limit[n] = min(u.k1, at[n].token + u.off);
      least = min(least, limit[n]);
    }
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) least = min(least, __shfl_xor(least, off, kWave));
    least = __builtin_amdgcn_readfirstlane(least);
  }
  f32x4 o[NR][DB];
  float m[NR], sum[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
#pragma unroll
    for (int i = 0; i < DB; ++i) o[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[n] = -INFINITY;
    sum[n] = 0.f;
  }

  for (; tile < u.k1; tile += 32 * W) {
    const bool more = tile + 32 * W < u.k1;
    kt.store(kd, l);
    if (more) {
      place(tile + 32 * W);
      kt.load(kb, oct_at, in);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    f32x4 s[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) s[n][0] = s[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const char* at0 = kd + row * (D * 2) + swizzled<C>(row, 4 * i + quad) * 16;  // (rows 16 apart are permuted alike)
      const bf16x8 k0 = *reinterpret_cast<const bf16x8*>(at0), k1 = *reinterpret_cast<const bf16x8*>(at0 + 16 * D * 2);
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        s[n][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[n][i], s[n][0], 0, 0, 0);
        s[n][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[n][i], s[n][1], 0, 0, 0);
      }
    }
    vl.store(vd, l);
    if (more) vl.load(vb, oct_at, in);

    bf16x8 pf[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[i] = s[n][0][i] * c; x[4 + i] = s[n][1][i] * c; }
      if (tile + 32 > least || tile < u.k0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int key = tile + 16 * (i >> 2) + 4 * quad + (i & 3);
          if (key >= limit[n] || key < u.k0) x[i] = -INFINITY;
        }
      }
      float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      if (__builtin_amdgcn_ballot_w64(top > m[n] + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const float next = fmaxf(m[n], top);
        const float f = next == -INFINITY ? 1.f : fast_exp2(m[n] - next);
        m[n] = next;
        sum[n] *= f;
#pragma unroll
        for (int i = 0; i < DB; ++i) o[n][i] *= f;
      }
      const float base_m = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
      for (int i = 0; i < 8; ++i) { x[i] = fast_exp2(x[i] - base_m); sum[n] += x[i]; }
      const u32x4 pw = {pack_bf16_pair(x[0], x[1]), pack_bf16_pair(x[2], x[3]), pack_bf16_pair(x[4], x[5]), pack_bf16_pair(x[6], x[7])};
      pf[n] = __builtin_bit_cast(bf16x8, pw);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int vr = 4 * quad + ((l & 15) >> 2);  // row of the tile that this lane reads from (and 16 + that)
#pragma unroll
    for (int i = 0; i < DB; ++i) {
      const int ch = 2 * i + ((l & 3) >> 1);
      const char* at0 = vd + vr * (D * 2) + swizzled<C>(vr, ch) * 16 + (l & 1) * 8;
      const bf16x8 vf = join8(lds_read_tr(at0), lds_read_tr(at0 + 16 * D * 2));
#pragma unroll
      for (int n = 0; n < NR; ++n) o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n], o[n][i], 0, 0, 0);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }

  finish_few<D, NR>(p, u, g, W, lds, w, turn, l, tid, bad, o, m, sum);
}

// ---------------------------------------------------------------- few rows, 4-bit keys and values
// Where the keys of a 64-key tile lie, a key to a lane: byte offsets of their codes (a sixteenth of that: of their scales).  Loads whose lanes take
// other keys get theirs by lane permutes.  Pages as in KeyRows: requested a tile ahead of their use and before other loads.
template <bool PAGED>
struct KeyOffsets {
  const int32_t* table;
  int lg_page, first, last_key, lane;
  uint32_t last, pages, ts;
  int64_t ps, head;
  __device__ __forceinline__ KeyOffsets(const AttendDev& p, const AttendUnit& u, int l, int g, int tile) {
    ts = (uint32_t)p.c_ts; ps = p.c_ps; lg_page = p.lg_page; last_key = u.k1 - 1; lane = l;
    head = (int64_t)g * p.c_hs;
    first = PAGED ? 0 : u.seq;
    last = PAGED ? p.last_page : p.last_row;
    table = PAGED ? p.table + (int64_t)u.seq * p.blocks_per_seq : nullptr;
    if (u.k0 < u.k1) ahead(tile);
  }
  __device__ __forceinline__ void ahead(int tile) {
    if constexpr (PAGED) pages = (uint32_t)table[min(tile + lane, last_key) >> lg_page];
  }
  // (behind the last key: the last key's, whose weight is zero there.  Nothing outside the pool is addressed, a bad page is noted.)
  __device__ __forceinline__ uint64_t at(int tile, bool& bad) const {
    const int key = min(tile + lane, last_key);
    if constexpr (PAGED) {
      bad |= pages > last;
      return (uint64_t)min(pages, last) * (uint64_t)ps + (uint64_t)((uint32_t)(key & ((1 << lg_page) - 1))) * ts + (uint64_t)head;
    } else {
      return (uint64_t)min((uint32_t)(first + key), last) * ts + (uint64_t)head;
    }
  }
};

__device__ __forceinline__ uint64_t of_lane(uint64_t v, int lane4) {  // lane4: four times the lane
  const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute(lane4, (int)(uint32_t)v), hi = (uint32_t)__builtin_amdgcn_ds_bpermute(lane4, (int)(uint32_t)(v >> 32));
  return (uint64_t)hi << 32 | lo;
}

// As swizzled(), for rows whose chunks are written four at a time by lanes of their own: of 16 lanes, four (d = 64: eight) rows times every fourth chunk.
template <int C>
__device__ __forceinline__ int swizzled_blocks(int r, int c) {
  if constexpr (C == 16) return c ^ ((r & 3) | (r & 1) << 2 | (r >> 2 & 1) << 3);
  else return c ^ ((r >> 1 & 3) | (r >> 1 & 1) << 2);
}

// A wave's 64-key tile on its way, one to a wave (two, in registers: 64 single tokens 50.5 us instead of 44.8).  Keys need no LDS: lane (key l & 15, quad l >> 4) holds D/4 consecutive elements of a key, and as the order of
// elements inside a product's sum is free, it hands them to the matrix cores as they are, turned into bf16, eight to a step; the
// queries are laid out alike.  Values come by whole rows, become bf16 on their way into LDS, and are transposed there.
template <int D>
struct FourBitTile {
  static constexpr int KW = D / 32;    // 32-bit words of a lane's part of a key
  static constexpr int C = D / 32;     // 16-byte chunks of a stored row, a block each
  static constexpr int R = 64 / C;     // rows of a load of values
  static constexpr int N = 64 / R;     // loads of a tile of values
  uint32_t k[4][KW], v[N][4];
  uint32_t ks, vs;                     // the scales of key number `lane` of the tile, a byte to a block
  __device__ __forceinline__ static uint32_t load_scales(const uint8_t* scales, uint64_t at) {
    if constexpr (D == 128) return *reinterpret_cast<const uint32_t*>(scales + (at >> 4));
    else return *reinterpret_cast<const uint16_t*>(scales + (at >> 4));
  }
  // (Of d = 64 four rows share a cache line: left in the L2 for the other heads, where these are innermost, 64 sequences take 35 us instead of 43, and
  // otherwise no longer.  Of d = 128, heads outermost, non-temporal loads make 44 us of 46 and 31 of 35 for 128K keys.)
  template <typename T>
  __device__ __forceinline__ static T codes_at(const char* at) {
    if constexpr (D == 64) return *reinterpret_cast<const T*>(at);
    else return __builtin_nontemporal_load(reinterpret_cast<const T*>(at));
  }
  __device__ __forceinline__ void load_keys(const AttendDev& p, uint64_t at, int l) {
    ks = load_scales(p.k_block_scale, at);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const char* codes = p.k + of_lane(at, 4 * (16 * x + (l & 15))) + (l >> 4) * (4 * KW);
      if constexpr (KW == 4) {
        const u32x4 w = codes_at<u32x4>(codes);
#pragma unroll
        for (int i = 0; i < 4; ++i) k[x][i] = w[i];
      } else {
        typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
        const u32x2 w = codes_at<u32x2>(codes);
        k[x][0] = w[0];
        k[x][1] = w[1];
      }
    }
  }
  __device__ __forceinline__ void place_values(uint64_t at, int l, uint64_t (&v_at)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) v_at[i] = of_lane(at, 4 * (R * i + l / C));
  }
  __device__ __forceinline__ void load_values(const AttendDev& p, uint64_t at, const uint64_t (&v_at)[N], int l) {
    vs = load_scales(p.v_block_scale, at);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const u32x4 w = codes_at<u32x4>(p.v + v_at[i] + l % C * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i][j] = w[j];
    }
  }
  // 16 keys as operands, eight elements to each
  __device__ __forceinline__ void keys(int x, int l, bf16x8 (&out)[KW]) const {
    const uint32_t scales = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (16 * x + (l & 15)), (int)ks);
    uint32_t w[4 * KW];
    widen_e2m1<4 * KW>(k[x], scales >> ((l >> 4) * KW / 4 * 8) & 0xff, w);
#pragma unroll
    for (int i = 0; i < KW; ++i) out[i] = __builtin_bit_cast(bf16x8, u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]});
  }
  __device__ __forceinline__ void store_values(char* tile, int l) const {  // as bf16
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = l / C + R * i, ch = 4 * (l % C);
      const uint32_t scales = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * r, (int)vs);
      uint32_t w[16];
      widen_e2m1<16>(v[i], scales >> (l % C * 8) & 0xff, w);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<u32x4*>(tile + r * (D * 2) + swizzled_blocks<D / 8>(r, ch + j) * 16) = u32x4{w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]};
    }
  }
};

template <int D, bool PAGED, int NR>
__device__ __forceinline__ void attend_few_4bit(const AttendDev& p, const AttendUnit& u, int g, int W, char* lds) {
  constexpr int KS = D / 32;          // steps of the product with the queries
  constexpr int DB = D / 16;          // blocks of values
  constexpr int C = D / 8;            // 16-byte chunks of a bf16 row
  const int tid = thread_of_piece(), w = __builtin_amdgcn_readfirstlane(tid >> 6), turn = w & (W - 1), l = tid & 63, row = l & 15, quad = l >> 4;
  bool mine[NR];
  RowPlace at[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    mine[n] = row + 16 * n < u.nr;
    at[n] = row_place(p, u.r0 + (mine[n] ? row + 16 * n : 0), g);
  }
  int tile = u.k0 < u.k1 ? (u.k0 & ~63) + 64 * turn : u.k1;
  KeyOffsets<PAGED> offsets(p, u, l, g, tile);
  char* const vd = lds + w * (64 * D * 2);
  bool bad = false;
  FourBitTile<D> x;
  uint64_t at_keys, v_at[FourBitTile<D>::N];
  const auto load_keys = [&](int tile) {
    at_keys = offsets.at(tile, bad);
    offsets.ahead(tile + 64 * W);
    x.load_keys(p, at_keys, l);
    x.place_values(at_keys, l, v_at);
  };
  if (tile < u.k1) {
    load_keys(tile);
    x.load_values(p, at_keys, v_at, l);
  }

  // the queries, in the order of the keys' elements
  bf16x8 qf[NR][KS];
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 x = {0, 0, 0, 0};
      if (mine[n]) x = *reinterpret_cast<const u32x4*>(p.q + at[n].token * p.q_ts + at[n].h * p.q_hs + quad * (D / 4) + s * 8);
      qf[n][s] = __builtin_bit_cast(bf16x8, x);
    }
  const float c = p.scale_log2;  // (positive)
  int limit[NR], least = u.k1;
#pragma unroll
  for (int n = 0; n < NR; ++n) limit[n] = u.k1;
  if (u.off != kNoLimit) {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      if (mine[n]) limit[n] = min(u.k1, at[n].token + u.off);
      least = min(least, limit[n]);
    }
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) least = min(least, __shfl_xor(least, off, kWave));
    least = __builtin_amdgcn_readfirstlane(least);
  }
  f32x4 o[NR][DB];
  float m[NR], sum[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
#pragma unroll
    for (int i = 0; i < DB; ++i) o[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[n] = -INFINITY;
    sum[n] = 0.f;
  }

  for (; tile < u.k1; tile += 64 * W) {
    const bool more = tile + 64 * W < u.k1;
    __builtin_amdgcn_s_setprio(1);
    f32x4 s[NR][4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      bf16x8 kf[KS];
      x.keys(y, l, kf);
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        s[n][y] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KS; ++i) s[n][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i], qf[n][i], s[n][y], 0, 0, 0);
      }
    }
    // (the lanes' exchange of offsets in front of the stores to LDS, behind which it would wait; with two tiles of rows registers do not do for that)
    if (NR == 1 && more) load_keys(tile + 64 * W);
    x.store_values(vd, l);
    if (NR == 2 && more) load_keys(tile + 64 * W);
    if (more) x.load_values(p, at_keys, v_at, l);
    __builtin_amdgcn_s_setprio(0);
    bf16x8 pf[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      if (tile + 64 > least || tile < u.k0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = tile + 16 * (i >> 2) + 4 * quad + (i & 3);
          if (key >= limit[n] || key < u.k0) s[n][i >> 2][i & 3] = -INFINITY;
        }
      }
      float top = s[n][0][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[n][i >> 2][i & 3]);
      top *= c;
      if (__builtin_amdgcn_ballot_w64(top > m[n] + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const float next = fmaxf(m[n], top);
        const float f = next == -INFINITY ? 1.f : fast_exp2(m[n] - next);
        m[n] = next;
        sum[n] *= f;
#pragma unroll
        for (int i = 0; i < DB; ++i) o[n][i] *= f;
      }
      const float base_m = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          e[i] = fast_exp2(__builtin_fmaf(s[n][2 * y + (i >> 2)][i & 3], c, -base_m));
          sum[n] += e[i];
        }
        const u32x4 pw = {pack_bf16_pair(e[0], e[1]), pack_bf16_pair(e[2], e[3]), pack_bf16_pair(e[4], e[5]), pack_bf16_pair(e[6], e[7])};
        pf[n][y] = __builtin_bit_cast(bf16x8, pw);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int l2 = l;
    if (NR == 2) asm volatile("" : "+v"(l2));
    const int vr = (l2 >> 4) * 4 + ((l2 & 15) >> 2);  // row of the tile that this lane reads from (and 16, 32, 48 + that)
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        const int ch = 2 * i + ((l2 & 3) >> 1);
        const char* at0 = vd + (vr + 32 * y) * (D * 2) + swizzled_blocks<C>(vr, ch) * 16 + (l2 & 1) * 8;
        const bf16x8 vf = join8(lds_read_tr(at0), lds_read_tr(at0 + 16 * D * 2));
#pragma unroll
        for (int n = 0; n < NR; ++n) o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n][y], o[n][i], 0, 0, 0);
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  finish_few<D, NR>(p, u, g, W, lds, w, turn, l, tid, __builtin_amdgcn_ballot_w64(bad) != 0, o, m, sum);
}

// ---------------------------------------------------------------- many rows
// one lane's share of a 64-key tile of keys or values that T threads load: chunks tid + T i of the tile's 16-byte chunks
template <int D, int KIND, int T>
struct ManyTile {
  static constexpr bool FP8 = KIND == SP_K_FP8_E4M3;
  static constexpr int CB = 16;                            // bytes of a chunk
  static constexpr int C = FP8 ? D / 16 : D / 8;           // 16-byte chunks of a stored row
  static constexpr int N = kTileKeys * C / T;
  static constexpr int STEP = T / C;                       // rows between a lane's chunks
  u32x4 x[N];
  __device__ __forceinline__ void load(const char* base, const uint8_t*, const int64_t (&at)[N], const uint32_t (&in)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = *reinterpret_cast<const u32x4*>(base + at[i] + in[i]);
  }
  __device__ __forceinline__ void store(char* tile, int tid) const {
    const int ch = tid % C;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = tid / C + STEP * i;
      char* row = tile + r * (D * 2);
      if constexpr (FP8) {
        u32x4 lo, hi;
        widen_e4m3(x[i], lo, hi);
        *reinterpret_cast<u32x4*>(row + swizzled<D / 8>(r, 2 * ch) * 16) = lo;
        *reinterpret_cast<u32x4*>(row + swizzled<D / 8>(r, 2 * ch + 1) * 16) = hi;
      } else {
        *reinterpret_cast<u32x4*>(row + swizzled<D / 8>(r, ch) * 16) = x[i];
      }
    }
  }
};
// ... of 4-bit codes: half a block, 8 bytes, to a lane, so that all lanes load
template <int D, int T>
struct ManyTile<D, SP_K_MXFP4, T> {
  static constexpr int CB = 8, C = D / 16, N = 1, STEP = kTileKeys;
  static_assert(kTileKeys * C == T, "a chunk to a thread");
  uint2 x;
  uint32_t scale;
  __device__ __forceinline__ void load(const char* base, const uint8_t* scales, const int64_t (&at)[N], const uint32_t (&in)[N]) {
    x = *reinterpret_cast<const uint2*>(base + at[0] + in[0]);
    scale = scales[(at[0] + in[0]) >> 4];
  }
  __device__ __forceinline__ void store(char* tile, int tid) const {
    const int ch = 2 * (tid % C), r = tid / C;
    char* row = tile + r * (D * 2);
    const uint32_t codes[2] = {x.x, x.y};
    uint32_t w[8];
    widen_e2m1<8>(codes, scale, w);
    *reinterpret_cast<u32x4*>(row + swizzled<D / 8>(r, ch) * 16) = u32x4{w[0], w[1], w[2], w[3]};
    *reinterpret_cast<u32x4*>(row + swizzled<D / 8>(r, ch + 1) * 16) = u32x4{w[4], w[5], w[6], w[7]};
  }
};

template <int D, int KIND, bool PAGED>
__device__ __forceinline__ void attend_many(const AttendDev& p, const AttendUnit& u, int g, char* lds) {
  constexpr int NW = attend_waves(D);
  constexpr int SETS = NW == 8 ? 2 : 1;  // tiles on their way from memory
  constexpr int KS = D / 16;   // steps of the product with the queries
  constexpr int DB = D / 32;   // blocks of values
  constexpr int C = D / 8;
  constexpr int TILE = kTileKeys * D * 2;  // bytes of a tile of keys or of values
  using Tile = ManyTile<D, KIND, 64 * NW>;
  const int tid = thread_of_piece(), w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, half = l >> 5;
  const int row = w * 32 + (l & 31);
  const bool mine = row < u.nr;
  const RowPlace at = row_place(p, u.r0 + (mine ? row : 0), g);
  uint32_t flip, keep;
  const float c = key_factor(p, g, flip, keep);
  bf16x8 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    u32x4 x = {0, 0, 0, 0};
    if (mine) x = *reinterpret_cast<const u32x4*>(p.q + at.token * p.q_ts + at.h * p.q_hs + s * 16 + half * 8);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (x[i] ^ flip) & keep;
    qf[s] = __builtin_bit_cast(bf16x8, x);
  }
  // the keys that the wave's rows see: all see those below `least`, none those from `most` on
  int limit = mine ? u.k1 : u.k0;
  if (mine && u.off != kNoLimit) limit = min(u.k1, at.token + u.off);
  int least = mine ? limit : u.k1, most = limit;
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) {
    least = min(least, __shfl_xor(least, off, kWave));
    most = max(most, __shfl_xor(most, off, kWave));
  }
  least = __builtin_amdgcn_readfirstlane(least);
  most = __builtin_amdgcn_readfirstlane(most);

  const int first_tile = u.k0 < u.k1 ? u.k0 & ~(kTileKeys - 1) : u.k1;
  KeyRows<PAGED> rows(p, u, l, first_tile);
  const char* const kb = p.k + (int64_t)g * p.c_hs;
  const char* const vb = p.v + (int64_t)g * p.c_hs;
  const uint8_t* const kb_scale = KIND == SP_K_MXFP4 ? p.k_block_scale + (int64_t)g * p.c_hs / 16 : nullptr;
  const uint8_t* const vb_scale = KIND == SP_K_MXFP4 ? p.v_block_scale + (int64_t)g * p.c_hs / 16 : nullptr;
  const int lane_row = l / Tile::C, lane_chunk = (l % Tile::C) * Tile::CB;
  uint32_t bad = 0;

  f32x16 o[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  float m = -INFINITY, sum = 0.f;

  // addresses of the operands in a tile
  int k_at[KS], v_at[DB][2];
#pragma unroll
  for (int s = 0; s < KS; ++s) k_at[s] = (l & 31) * (D * 2) + swizzled<C>(l & 31, 2 * s + half) * 16;
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int vr = 8 * x + 4 * half + ((l & 15) >> 2);
      v_at[i][x] = vr * (D * 2) + swizzled<C>(vr, 4 * i + 2 * ((l >> 4) & 1) + ((l & 3) >> 1)) * 16 + (l & 1) * 8;
    }

  // the wave's loads cover rows w R + STEP i of a tile, R <= 8 of one octet or R = 16 of two
  constexpr int R = 64 / Tile::C;
  Tile kt[SETS], vl[SETS];
  auto load = [&](int tile, Tile& kt, Tile& vl) {
    int64_t at[Tile::N];
    uint32_t in[Tile::N];
#pragma unroll
    for (int i = 0; i < Tile::N; ++i) {
      const int r = R * w + Tile::STEP * i;
      int oct = rows.octet(tile, r);
      at[i] = rows.base(oct, r, bad);
      if constexpr (R > 8) {
        const int oct1 = rows.octet(tile, r + 8);
        const int64_t at1 = rows.base(oct1, r + 8, bad);
        if (lane_row >= 8) { at[i] = at1; oct = oct1; }
      }
      in[i] = rows.within(oct, tile + r + lane_row) + lane_chunk;
    }
    rows.ahead(tile + kTileKeys);
    kt.load(kb, kb_scale, at, in);
    vl.load(vb, vb_scale, at, in);
  };
  if (first_tile < u.k1) load(first_tile, kt[0], vl[0]);
  if (SETS == 2 && first_tile + kTileKeys < u.k1) load(first_tile + kTileKeys, kt[SETS - 1], vl[SETS - 1]);
  // One tile out of buffer BUF (a constant, so that the operands' addresses are too).  The compiler is told how to mix reads, products and
  // the rest: operands are read several products ahead, and the weights of the next 16 keys are formed while the
  // matrix cores work on these.
  auto step = [&](auto buf, int tile) {
    constexpr int SET = decltype(buf)::value % SETS;
    char* const kd = lds + decltype(buf)::value * 2 * TILE;
    char* const vd = kd + TILE;
    kt[SET].store(kd, tid);
    vl[SET].store(vd, tid);
    __syncthreads();
    if (tile + SETS * kTileKeys < u.k1) load(tile + SETS * kTileKeys, kt[SET], vl[SET]);
    if (tile >= most) return;  // (the wave's rows see none of these keys)
    __builtin_amdgcn_s_setprio(1);  // products first: the other wave's other instructions fill the gaps
    f32x16 s[2];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int j = 0; j < 16; ++j) s[x][j] = 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kd + k_at[i] + x * 32 * (D * 2));
        s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[i], s[x], 0, 0, 0);
      }
    __builtin_amdgcn_sched_group_barrier(kSchedLdsRead, kAhead, 0);
#pragma unroll
    for (int i = 0; i < 2 * KS - kAhead; ++i) {
      __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kSchedLdsRead, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kSchedMfma, kAhead, 0);
    __builtin_amdgcn_s_setprio(0);
    if (tile + kTileKeys > least || tile < u.k0) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int key = tile + 32 * x + 8 * (j >> 2) + 4 * half + (j & 3);
          if (key >= limit || key < u.k0) s[x][j] = -INFINITY;
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int j = 0; j < 16; ++j) top = fmaxf(top, s[x][j]);
    top *= c;
    if (__builtin_amdgcn_ballot_w64(top > m + kSlack)) {
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float next = fmaxf(m, top);
      const float f = next == -INFINITY ? 1.f : fast_exp2(m - next);
      m = next;
      sum *= f;
#pragma unroll
      for (int i = 0; i < DB; ++i) o[i] *= f;
    }
    const float base = m == -INFINITY ? 0.f : m;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float x[8], part = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = fast_exp2(__builtin_fmaf(s[e >> 1][8 * (e & 1) + j], c, -base));
        part += x[j];
      }
      sum += part;
      const u32x4 pw = {pack_bf16_pair(x[0], x[1]), pack_bf16_pair(x[2], x[3]), pack_bf16_pair(x[4], x[5]), pack_bf16_pair(x[6], x[7])};
      const bf16x8 pf = __builtin_bit_cast(bf16x8, pw);
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        const bf16x8 vf = join8(lds_read_tr(vd + v_at[i][0] + e * 16 * (D * 2)), lds_read_tr(vd + v_at[i][1] + e * 16 * (D * 2)));
        o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[i], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_group_barrier(kSchedLdsRead, 2 * DB, 0);
    __builtin_amdgcn_sched_group_barrier(kSchedValu, 28, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
        if (e < 3) {
          __builtin_amdgcn_sched_group_barrier(kSchedLdsRead, 2, 0);
          __builtin_amdgcn_sched_group_barrier(kSchedValu, 28 / DB, 0);
        }
      }
    __builtin_amdgcn_s_setprio(0);
  };
  for (int tile = first_tile; tile < u.k1; tile += 2 * kTileKeys) {
    step(std::integral_constant<int, 0>(), tile);
    if (tile + kTileKeys < u.k1) step(std::integral_constant<int, 1>(), tile + kTileKeys);
  }

  // the waves' bad pages (`bad` is the same in all lanes), behind the tiles
  uint32_t* const bads = reinterpret_cast<uint32_t*>(lds + 4 * TILE);
  if (l == 0) bads[w] = bad;
  __syncthreads();
  uint32_t any_bad = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) any_bad |= bads[i];
  sum += __shfl_xor(sum, 32, kWave);
  // (formed again: nothing of it is kept in registers over the loop)
  const int end_tid = thread_of_piece(), end_row = (end_tid >> 6) * 32 + (end_tid & 31), end_half = (end_tid >> 5) & 1;
  if (end_row >= u.nr) return;
  if (u.slot >= 0) {
    const int64_t place = slot_row(p, u.slot, end_row, g);
    float* dst = p.sums + place * D + 4 * end_half;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4*>(dst + 32 * i + 8 * j) = f32x4{o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]};
    if (end_half == 0) store_stats(p, place, m, sum, any_bad);
    return;
  }
  const float mul = (sum == 0.f ? 0.f : 1.f / sum) * (p.v_scale ? p.v_scale[g] : 1.f);
  const RowPlace to = row_place(p, u.r0 + end_row, g);
  uint16_t* dst = p.out + to.token * p.o_ts + to.h * p.o_hs + 4 * end_half;
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      store_values(dst + 32 * i + 8 * j, f32x4{o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]} * mul, any_bad);
    }
  if (end_half == 0 && p.lse) store_lse(p, to.token, to.h, m, sum, any_bad);
}

// every row of the call, or of one piece and KV head, becomes NaN
__device__ __forceinline__ void nan_rows(const AttendDev& p, int d, int64_t r0, int64_t nr, int heads, int h0, int64_t first, int64_t stride) {
  const int vec = d / 8;
  const uint32_t nan2 = kNanBf16 * 0x10001u;
  for (int64_t x = first; x < nr * vec; x += stride) {
    const int64_t flat = r0 + x / vec, token = flat / heads;
    const int h = h0 + (int)(flat % heads);
    *reinterpret_cast<u32x4*>(p.out + token * p.o_ts + h * p.o_hs + x % vec * 8) = u32x4{nan2, nan2, nan2, nan2};
    if (x % vec == 0 && p.lse) reinterpret_cast<uint32_t*>(p.lse)[token * p.H + h] = kNanF32;
  }
}

}  // namespace

template <int D, int KIND, bool PAGED>
__global__ __launch_bounds__(64 * attend_waves(D), D == 64 ? 3 : 2) void attend_kernel(const AttendDev p) {
  constexpr int T = 64 * attend_waves(D);
  __shared__ __align__(16) char lds[attend_waves(D) * (64 * D * 2 + 2 * kFewRows * 4 + 4)];  // tiles: 16 KB a wave (8, d = 64), and few rows' statistics
  // The KV heads of a piece are neighbours: with eight of them, each has the L2 of one XCD, which the rows of a
  // block share, as workgroups go to the XCDs in turn.
  // Where rows of several heads share a cache line, the heads of a piece go to one XCD instead, eight pieces side by side: no line is read by two.
  int n = (int)(blockIdx.x / (uint32_t)p.H_kv), g = (int)(blockIdx.x % (uint32_t)p.H_kv);
  if (KIND == SP_K_MXFP4 && p.heads_together) {
    const uint32_t group = blockIdx.x / (8u * (uint32_t)p.H_kv), in = blockIdx.x - group * (8u * (uint32_t)p.H_kv);
    const uint32_t side = min(8u, gridDim.x / (uint32_t)p.H_kv - 8u * group);
    n = (int)(8u * group + in % side);
    g = (int)(in / side);
  }
  // the plan through the scalar cache; header, stretch and its first piece together (the list has room for every workgroup's index)
  const auto header = reinterpret_cast<const __attribute__((address_space(4))) AttendHeader*>(reinterpret_cast<uintptr_t>(p.header));
  typedef const __attribute__((address_space(4))) AttendStretch* StretchPtr;
  typedef const __attribute__((address_space(4))) AttendUnit* UnitPtr;
  const auto stretch = reinterpret_cast<StretchPtr>(reinterpret_cast<uintptr_t>(p.stretches + n));
  auto read = [&](UnitPtr x) {
    AttendUnit u;
    u.r0 = x->r0; u.nr = x->nr; u.seq = x->seq; u.k0 = x->k0;
    u.k1 = x->k1; u.off = x->off; u.slot = x->slot; u.run = x->run;
    return u;
  };
  const uint64_t print = header->print;
  const int n_stretches = header->n_stretches;
  int x = stretch->first;
  const int end = stretch->end;
  AttendUnit u = read(&stretch->unit);
  if (print != p.print) {
    nan_rows(p, D, 0, (int64_t)p.T_new * p.H, p.H, 0, (int64_t)blockIdx.x * T + threadIdx.x, (int64_t)gridDim.x * T);
    return;
  }
  if (n >= n_stretches || x >= end) return;
  const auto unit_at = [&](int i) { return reinterpret_cast<UnitPtr>(reinterpret_cast<uintptr_t>(p.units + i)); };
  for (;;) {
    if (u.run != kBadUnit && u.nr <= kFewRows) {
      // one piece, or several short ones side by side
      const int run = u.run > 1 ? u.run : 1;
      int W = attend_waves(D);
      while (W > 1 && run * W > attend_waves(D)) W >>= 1;
      const int mine = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / W;
      AttendUnit v = u;
      if (mine > 0 && mine < run) v = read(unit_at(x + mine));
      if (mine >= run) v.nr = v.k0 = v.k1 = 0;
      if constexpr (KIND == SP_K_MXFP4) {
        if (u.nr <= kTileRows) attend_few_4bit<D, PAGED, 1>(p, v, g, W, lds);
        else attend_few_4bit<D, PAGED, 2>(p, v, g, W, lds);
      } else {
        constexpr bool FP8 = KIND == SP_K_FP8_E4M3;
        if (u.nr <= kTileRows) attend_few<D, FP8, PAGED, 1>(p, v, g, W, lds);
        else attend_few<D, FP8, PAGED, 2>(p, v, g, W, lds);
      }
      x += run;
    } else {
      if (u.run == kBadUnit) nan_rows(p, D, u.r0, u.nr, p.G, g * p.G, thread_of_piece(), T);
      else attend_many<D, KIND, PAGED>(p, u, g, lds);
      ++x;
    }
    if (x >= end) return;
    u = read(unit_at(x));
    __syncthreads();  // (the next piece uses the same LDS)
  }
}

namespace {

sp_status check_attend(const sp_attend_args* a) {
  const sp_status st = check_attend_plan_args(a);
  if (st != SP_OK) return st;
  if (!finite_f32(a->scale * kLog2e) || a->scale <= 0.f) return SP_EINVAL;
  const bool fp8 = a->cache_dtype == SP_K_FP8_E4M3, fp4 = a->cache_dtype == SP_K_MXFP4;
  if (!fp8 && (a->d_k_scale || a->d_v_scale)) return SP_EINVAL;
  if (!fp4 && (a->d_k_block_scale || a->d_v_block_scale)) return SP_EINVAL;
  if (a->cache_token_stride >= INT64_C(1) << 26) return SP_EINVAL;
  if ((a->T_new > 0 && (!a->d_q || !a->d_out)) || !a->d_k_cache || !a->d_v_cache) return SP_ENULL;
  if (fp4 && (!a->d_k_block_scale || !a->d_v_block_scale)) return SP_ENULL;
  const int64_t row[] = {a->q_token_stride, a->q_head_stride, a->out_token_stride, a->out_head_stride};
  const int64_t cache[] = {a->cache_token_stride, a->cache_head_stride, a->d_block_table ? a->cache_page_stride : 0};
  for (int64_t s : row) if (s < 0) return SP_EINVAL;
  for (int64_t s : cache) if (s < 0) return SP_EINVAL;
  if ((a->H > 1 && a->out_head_stride < a->d) || (a->T_new > 1 && a->out_token_stride < a->d)) return SP_EINVAL;  // rows of out that lie in one another
  for (int64_t s : row) if (s & 7) return SP_EALIGN;
  for (int64_t s : cache) if (s & (cache_stride_unit(a->cache_dtype, a->d) - 1)) return SP_EALIGN;
  if (!aligned_scales(a->d_k_block_scale, a->d) || !aligned_scales(a->d_v_block_scale, a->d)) return SP_EALIGN;
  if (!aligned16(a->d_q) || !aligned16(a->d_k_cache) || !aligned16(a->d_v_cache) || !aligned16(a->d_out)) return SP_EALIGN;
  if (!a->d_workspace || a->workspace_bytes < sp_attend_workspace_bytes(a)) return SP_EWORKSPACE;
  if (reinterpret_cast<uintptr_t>(a->d_workspace) & 255u) return SP_EALIGN;
  return SP_OK;
}

template <int D, int KIND>
void launch_attend(const AttendDev& p, bool paged, uint32_t grid, hipStream_t stream) {
  if (paged) hipLaunchKernelGGL((attend_kernel<D, KIND, true>), dim3(grid), dim3(64 * attend_waves(D)), 0, stream, p);
  else hipLaunchKernelGGL((attend_kernel<D, KIND, false>), dim3(grid), dim3(64 * attend_waves(D)), 0, stream, p);
}
template <int D>
void launch_attend(const AttendDev& p, int dtype, bool paged, uint32_t grid, hipStream_t stream) {
  if (dtype == SP_K_MXFP4) launch_attend<D, SP_K_MXFP4>(p, paged, grid, stream);
  else if (dtype == SP_K_FP8_E4M3) launch_attend<D, SP_K_FP8_E4M3>(p, paged, grid, stream);
  else launch_attend<D, SP_K_BF16>(p, paged, grid, stream);
}

}  // namespace

}  // namespace sp

extern "C" size_t sp_attend_workspace_bytes(const sp_attend_args* a) {
  return sp::check_attend_shape(a) == SP_OK ? sp::attend_workspace(a) : 0;
}

extern "C" sp_status sp_attend(const sp_attend_args* a, void* hip_stream) {
  using namespace sp;
  const sp_status st = check_attend(a);
  if (st != SP_OK) return st;
  if (a->T_new == 0) return SP_OK;
  const AttendCaps caps = attend_caps(a);
  const AttendPlanLayout l = attend_plan_layout(a);
  const char* base = static_cast<const char*>(a->d_plan);
  const bool paged = a->d_block_table != nullptr;
  const auto bytes = [&](int64_t elements) { return a->cache_dtype == SP_K_MXFP4 ? elements / 2 : a->cache_dtype == SP_K_FP8_E4M3 ? elements : 2 * elements; };
  AttendDev p;
  p.H = a->H; p.H_kv = a->H_kv; p.G = a->H / a->H_kv; p.T_new = (int)a->T_new;
  p.lg_page = 0;
  while (paged && (1 << p.lg_page) < a->page_size) ++p.lg_page;
  p.blocks_per_seq = a->blocks_per_seq;
  p.last_page = paged ? (uint32_t)(a->n_rows / a->page_size - 1) : 0;
  p.last_row = (uint32_t)(a->n_rows - 1);
  p.most_items = (uint32_t)(caps.rows * a->H_kv);  // (no more than T_new * H)
  p.scale_log2 = a->scale * kLog2e;
  p.q_ts = a->q_token_stride; p.q_hs = a->q_head_stride;
  p.o_ts = a->out_token_stride; p.o_hs = a->out_head_stride;
  p.c_ts = (int32_t)bytes(a->cache_token_stride); p.c_hs = bytes(a->cache_head_stride); p.c_ps = bytes(a->cache_page_stride);
  p.print = attend_print(a);
  p.header = reinterpret_cast<const AttendHeader*>(base);
  p.units = reinterpret_cast<const AttendUnit*>(base + l.units);
  p.stretches = reinterpret_cast<const AttendStretch*>(base + l.stretches);
  p.rows = reinterpret_cast<const AttendRow*>(base + l.rows);
  p.table = a->d_block_table;
  p.q = static_cast<const uint16_t*>(a->d_q);
  p.k = static_cast<const char*>(a->d_k_cache); p.v = static_cast<const char*>(a->d_v_cache);
  p.k_scale = a->d_k_scale; p.v_scale = a->d_v_scale;
  p.k_block_scale = a->d_k_block_scale; p.v_block_scale = a->d_v_block_scale;
  p.heads_together = a->H_kv > 1 && p.c_hs < 128;
  p.out = static_cast<uint16_t*>(a->d_out); p.lse = a->d_lse;
  p.sums = static_cast<float*>(a->d_workspace);
  p.stats = reinterpret_cast<float2*>(static_cast<char*>(a->d_workspace) + attend_sums_bytes(a));
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const uint32_t grid = (uint32_t)(most_stretches(a) * a->H_kv);
  if (a->d == 128) launch_attend<128>(p, a->cache_dtype, paged, grid, stream);
  else launch_attend<64>(p, a->cache_dtype, paged, grid, stream);
  launch_attend_join(p, a->d, stream);
  return launch_status();
}
