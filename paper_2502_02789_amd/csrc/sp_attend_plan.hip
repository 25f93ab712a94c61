// sp_attend_plan: the list of pieces of work of an attention call, made on the device from the lengths (which only the
// device knows, so that a captured graph follows them), and the kernel that joins the pieces' sums.  The cut itself is in sp_attend_plan.h.
// The plan is bound by its chain of dependent reads and barriers and by fetching its own code (one workgroup): 14 us for one sequence,
// 20 for 64, 25 for 64 that share a prefix, 9 for a long prompt whose blocks are not laid end to end; a step makes it once for all layers.
#include "sp_attend_internal.h"

namespace sp {

namespace {

constexpr int kPlanThreads = 512;  // (1024, whose registers do not do: twice the time for one sequence, 1.2 times for 64 that share a prefix; 256: a
                                   // twentieth less for one, 1.3 times for 64 that share a prefix)

struct PlanSeq { int32_t t0, n, len, shared; };                 // len -1: invalid
struct PlanGroup { int32_t shared, active, t0, tokens, slot, pieces, pad[2]; };

struct PlanDev {
  sp_attend_args a;   // (host pointers in it are not used)
  int G;
  int64_t cap_blocks, cap_units, cap_joins, cap_rows, cap_slots;
  uint64_t print;
  AttendHeader* header;
  AttendUnit* units;
  AttendStretch* stretches;
  AttendJoin* joins;
  AttendRow* rows;
  int32_t* seg_start;
  PlanSeq* seqs;
  PlanGroup* groups;
};

__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

__device__ __forceinline__ int group_of(const int32_t* cu_group, int n, int b) {
  if (n == 0 || b < cu_group[0] || b >= cu_group[n]) return -1;
  return upper_segment(cu_group, n, b);
}

// exclusive prefixes of N numbers over the workgroup's threads, and their sums over all of them (most waves have nothing to add)
template <int N>
__device__ __forceinline__ void block_exclusive(int64_t (&v)[N], int64_t (&total)[N]) {
  __shared__ int64_t waves[kPlanThreads / 64][N];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  bool any = false;
#pragma unroll
  for (int i = 0; i < N; ++i) any |= v[i] != 0;
  if (__ballot(any)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int64_t x = v[i];
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int64_t y = __shfl_up(x, off, kWave);
        if (l >= off) x += y;
      }
      if (l == 63) waves[w][i] = x;
      v[i] = x - v[i];
    }
  } else if (l < N) {
    waves[w][l] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    total[i] = 0;
#pragma unroll
    for (int x = 0; x < kPlanThreads / 64; ++x) {
      if (x == w) v[i] += total[i];
      total[i] += waves[x][i];
    }
  }
  __syncthreads();
}

struct Block {       // a block of rows
  int seg, i;        // segment (prefixes first, then sequences), block of it
  int rows;          // of the segment
  int m, nr;         // rows of a whole block, of this one
  int first, keys;   // its keys are [first, first + keys)
  int steps, cost;   // ... and a step's cost
  int extra;         // what the block costs besides
};

// largest i in [0, n) with table[i] <= x (table[0] <= x)
template <typename T>
__device__ __forceinline__ int last_at_most(const T* table, int n, T x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (table[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

constexpr int kLdsSeqs = 512;        // sequences and segments that are kept in LDS
constexpr int kMostStretches = 768;  // (attend_items())

}  // namespace

__global__ __launch_bounds__(kPlanThreads) void attend_plan_kernel(const PlanDev p) {
  __shared__ int most_pieces;
  __shared__ PlanSeq lds_seqs[kLdsSeqs];
  __shared__ PlanGroup lds_groups[kLdsSeqs];
  __shared__ int32_t lds_cu_group[kStagedOffsets];
  __shared__ int32_t lds_seg[2 * kLdsSeqs + 1];
  __shared__ int64_t start[kMostStretchBlocks + 1];   // by stretches: the blocks laid end to end
  __shared__ int64_t cuts[kMostStretches + 1];        // (block, step) that each stretch begins at
  __shared__ int32_t first_unit[kMostStretches + 1];
  __shared__ int32_t slot_of[kMostStretchBlocks];
  __shared__ uint8_t alone[kMostStretchBlocks + kMostStretches];  // pieces that are short: how many tiles of rows they have
  PlanSeq* const seqs = p.a.B <= kLdsSeqs ? lds_seqs : p.seqs;
  PlanGroup* const groups = p.a.B <= kLdsSeqs ? lds_groups : p.groups;  // (no more groups than sequences)
  int32_t* const seg_start = p.a.B <= kLdsSeqs ? lds_seg : p.seg_start;
  const int tid = threadIdx.x, B = p.a.B, n_groups = p.a.n_groups, G = p.G, T = (int)p.a.T_new;
  if (tid == 0) {
    p.header->print = 0;
    most_pieces = 0;
  }

  const int32_t* const cu_group = n_groups > 0 ? staged_offsets(p.a.d_cu_group, n_groups, lds_cu_group) : nullptr;

  // the sequences' new tokens and lengths, as far as they are valid
  for (int b = tid; b < B; b += kPlanThreads) {
    PlanSeq s;
    s.t0 = clamp_int(p.a.d_cu_new[b], 0, T);
    s.n = clamp_int(p.a.d_cu_new[b + 1], s.t0, T) - s.t0;
    s.len = p.a.d_kv_len[b];
    s.shared = 0;
    int64_t room;
    if (p.a.d_block_table) {
      room = (int64_t)p.a.blocks_per_seq * p.a.page_size;
    } else {
      const int64_t first = p.a.d_cu_cache[b], end = min((int64_t)p.a.d_cu_cache[b + 1], p.a.n_rows);
      room = first < 0 ? -1 : end - first;
    }
    if (s.len < 0 || s.len > room) s.len = -1;
    seqs[b] = s;
  }
  for (int g = tid; g < n_groups; g += kPlanThreads) {
    PlanGroup x = {};
    const int b0 = clamp_int(cu_group[g], 0, B), b1 = clamp_int(cu_group[g + 1], b0, B);
    x.shared = max(p.a.d_prefix_len[g], 0);
    x.t0 = clamp_int(p.a.d_cu_new[b0], 0, T);
    x.tokens = clamp_int(p.a.d_cu_new[b1], x.t0, T) - x.t0;
    groups[g] = x;
  }
  __syncthreads();
  // a prefix is cut to what all queries of the group see
  if (n_groups > 0) {
    for (int b = tid; b < B; b += kPlanThreads) {
      const int g = group_of(cu_group, n_groups, b);
      if (g < 0) continue;
      const PlanSeq s = seqs[b];
      if (s.n > 0) {
        atomicMin(&groups[g].shared, s.len < 0 ? 0 : max(s.len - s.n, 0));
        atomicAdd(&groups[g].active, 1);
      }
    }
    __syncthreads();
    for (int g = tid; g < n_groups; g += kPlanThreads) {  // (atomics are done in L2: read there)
      const int active = __hip_atomic_load(&groups[g].active, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      // (no more than the sequence has whose pages are read, whatever the offsets are)
      const int shared = min(__hip_atomic_load(&groups[g].shared, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), max(seqs[clamp_int(cu_group[g], 0, B - 1)].len, 0));
      groups[g].shared = prefix_pays(groups[g].tokens * G, active, shared, p.a.d, p.a.cache_dtype) ? shared : 0;
    }
    __syncthreads();
    for (int b = tid; b < B; b += kPlanThreads) {
      const int g = group_of(cu_group, n_groups, b);
      if (g >= 0) seqs[b].shared = groups[g].shared;
    }
    __syncthreads();
  }
  {  // the segments' first blocks
    const int n_seg = n_groups + B, per = (n_seg + kPlanThreads - 1) / kPlanThreads, s0 = min(n_seg, tid * per), s1 = min(n_seg, s0 + per);
    auto blocks_of = [&](int s) {
      const int tokens = s < n_groups ? (groups[s].shared > 0 ? groups[s].tokens : 0) : seqs[s - n_groups].n;
      return tokens > 0 ? segment_blocks(tokens * G, p.a.d) : 0;
    };
    int64_t count[1] = {0}, all[1];
    for (int s = s0; s < s1; ++s) count[0] += blocks_of(s);
    block_exclusive(count, all);
    for (int s = s0; s < s1; ++s) {
      seg_start[s] = (int)count[0];
      count[0] += blocks_of(s);
    }
    if (tid == 0) seg_start[n_seg] = (int)min(all[0], (int64_t)0x7fffffff);
    __syncthreads();
  }
  const int n_blocks = seg_start[n_groups + B], n_prefix = seg_start[n_groups];
  if (n_blocks > p.cap_blocks) return;  // (offsets that do not ascend may ask for more than there is room for: no plan then)

  // Blocks in the order that they are laid out in: prefixes first, then the sequences' blocks from the last to the first (of
  // a causal segment's blocks the last have the most keys).
  auto block_at = [&](int x, int hint) {
    const int flat = x < n_prefix ? x : n_blocks - 1 - (x - n_prefix);
    Block k;
    k.seg = hint >= 0 && flat >= seg_start[hint] && flat < seg_start[hint + 1] ? hint : upper_segment(seg_start, n_groups + B, flat);
    k.i = flat - seg_start[k.seg];
    k.rows = (k.seg < n_groups ? groups[k.seg].tokens : seqs[k.seg - n_groups].n) * G;
    k.m = block_rows(k.rows, p.a.d);
    if (k.seg < n_groups) {
      k.first = 0;
      k.keys = groups[k.seg].shared;
    } else {
      const PlanSeq s = seqs[k.seg - n_groups];
      k.first = s.shared;
      k.keys = s.len < 0 ? 0 : own_block_keys(k.rows, k.i, k.m, G, s.n, s.len, s.shared);
    }
    k.nr = min(k.m, k.rows - k.i * k.m);
    k.steps = block_steps(k.first, k.keys);
    k.cost = step_cost(k.nr, p.a.d, p.a.cache_dtype);
    k.extra = piece_cost(k.nr, k.keys, p.a.d);
    return k;
  };
  // every thread walks over a run of blocks, several times
  const int per = (n_blocks + kPlanThreads - 1) / kPlanThreads, x0 = min(n_blocks, tid * per), x1 = min(n_blocks, x0 + per);
  auto walk = [&](auto&& visit) {
    int seg = -1;
    for (int x = x0; x < x1; ++x) {
      const Block k = block_at(x, seg);
      seg = k.seg;
      visit(x, k);
    }
  };

  // where the blocks are cut
  int64_t sum[3] = {0, 0, 0}, total[3];  // cost, keys, large blocks
  walk([&](int, const Block& k) {
    sum[0] += (int64_t)k.steps * k.cost + k.extra;
    sum[1] += k.keys;
    sum[2] += k.nr > kFewRows;
  });
  block_exclusive(sum, total);
  const bool stretched = by_stretches(n_blocks, total[2], p.a.d, p.a.H_kv);
  const int cut = make_cut(total[1], p.a.d, p.a.H_kv);
  const int n_cuts = stretched ? stretch_count(total[0], p.a.d, p.a.H_kv) : 0;
  if (stretched) {
    int64_t at = sum[0];
    walk([&](int x, const Block& k) {
      start[x] = at;
      at += (int64_t)k.steps * k.cost + k.extra;
    });
    __syncthreads();
    for (int s = tid; s <= n_cuts; s += kPlanThreads) {
      int b = s < n_cuts && n_blocks > 0 ? 0 : n_blocks, j = 0;
      if (s > 0 && s < n_cuts) {
        const int64_t x = stretch_start(total[0], n_cuts, s);
        b = last_at_most(start, n_blocks, x);
        const Block k = block_at(b, -1);
        j = step_at(x, start[b], k.steps, k.cost, k.extra);
        if (j >= k.steps && j > 0) { ++b; j = 0; }
      }
      cuts[s] = ((int64_t)b << 32) | j;
    }
    __syncthreads();
  }
  // cuts inside block x: those with (x, 0) < cut < (x + 1, 0) are `first_cut` and those behind it
  auto first_cut = [&](int x) { return last_at_most(cuts, n_cuts + 1, (int64_t)x << 32) + 1; };
  auto pieces_at = [&](int x, const Block& k) {
    return stretched ? 1 + last_at_most(cuts, n_cuts + 1, ((int64_t)(x + 1) << 32) - 1) - (first_cut(x) - 1) : pieces_of(k.keys, cut);
  };
  auto joined = [&](const Block& k) { return k.seg >= n_groups && seqs[k.seg - n_groups].shared > 0; };
  auto leaves_sums = [&](const Block& k, int pieces) { return pieces > 1 || k.seg < n_groups || joined(k); };

  enum { kUnits, kSlots, kJoins, kRows };
  int64_t at[4] = {0, 0, 0, 0}, n[4];
  walk([&](int x, const Block& k) {
    const int pieces = pieces_at(x, k);
    at[kUnits] += pieces;
    if (leaves_sums(k, pieces)) {
      at[kSlots] += (int64_t)pieces * (k.m / kSlotRows);
      at[kJoins] += k.seg >= n_groups;
      at[kRows] += k.seg >= n_groups ? k.nr : 0;
    }
  });
  block_exclusive(at, n);
  if (n[kUnits] > p.cap_units || n[kSlots] > p.cap_slots || n[kJoins] > p.cap_joins || n[kRows] > p.cap_rows) return;
  if (stretched) {
    const int run = (n_cuts + kPlanThreads - 1) / kPlanThreads, s0 = min(n_cuts, tid * run), s1 = min(n_cuts, s0 + run);
    auto units_of = [&](int s) { return (cuts[s + 1] >> 32) + ((cuts[s + 1] & 0xffffffff) != 0) - (cuts[s] >> 32); };
    int64_t count[1] = {0}, units[1];
    for (int s = s0; s < s1; ++s) count[0] += units_of(s);
    block_exclusive(count, units);
    for (int s = s0; s < s1; ++s) {
      first_unit[s] = (int)count[0];
      count[0] += units_of(s);
    }
    if (tid == 0) first_unit[n_cuts] = (int)units[0];
  }

  auto unit_of = [&](const Block& k, int k0, int k1, int64_t slot) {
    AttendUnit unit;
    int t0;
    if (k.seg < n_groups) {
      t0 = groups[k.seg].t0;
      unit.seq = clamp_int(cu_group[k.seg], 0, B - 1);
      unit.off = kNoLimit;
      unit.run = 0;
    } else {
      const PlanSeq s = seqs[k.seg - n_groups];
      t0 = s.t0;
      unit.seq = p.a.d_block_table ? k.seg - n_groups : p.a.d_cu_cache[k.seg - n_groups];
      unit.off = s.len - s.n + 1 - s.t0;
      unit.run = s.len < 0 ? kBadUnit : 0;
    }
    unit.r0 = t0 * G + k.i * k.m;
    unit.nr = k.nr;
    unit.k0 = k0;
    unit.k1 = k1;
    unit.slot = (int)slot;
    return unit;
  };
  auto put_stretch = [&](int64_t s, int first, int end, const AttendUnit& unit) {
    p.stretches[s].first = first;
    p.stretches[s].end = end;
    p.stretches[s].unit = unit;
  };
  {
    int64_t u = at[kUnits], slot = at[kSlots];
    walk([&](int x, const Block& k) {
      const int pieces = pieces_at(x, k), step = k.m / kSlotRows;
      const bool sums = leaves_sums(k, pieces);
      if (k.seg < n_groups && k.i == 0) {
        groups[k.seg].slot = (int)slot;
        groups[k.seg].pieces = pieces;
      }
      if (stretched) {
        slot_of[x] = sums ? (int)slot : -1;
      } else {
        for (int q = 0; q < pieces; ++q) {
          const AttendUnit unit = unit_of(k, piece_start(k.first, k.keys, pieces, q), piece_start(k.first, k.keys, pieces, q + 1), sums ? slot + (int64_t)q * step : -1);
          p.units[u + q] = unit;
          put_stretch(u + q, (int)(u + q), (int)(u + q + 1), unit);
        }
        u += pieces;
      }
      if (sums) slot += (int64_t)pieces * step;
    });
  }
  __syncthreads();
  if (stretched) {
    auto piece = [&](int u, int s) {
      const int64_t a = cuts[s], b = cuts[s + 1];
      const int x = (int)(a >> 32) + u - first_unit[s];
      const Block k = block_at(x, -1);
      const int j0 = x == (int)(a >> 32) ? (int)a : 0, j1 = x == (int)(b >> 32) ? (int)b : k.steps;
      const int q = j0 > 0 ? s - first_cut(x) + 1 : 0;
      return unit_of(k, step_key(k.first, k.keys, k.steps, j0), step_key(k.first, k.keys, k.steps, j1),
                     slot_of[x] < 0 ? -1 : slot_of[x] + (int64_t)q * (k.m / kSlotRows));
    };
    for (int u = tid; u < (int)n[kUnits]; u += kPlanThreads) {
      const AttendUnit x = piece(u, last_at_most(first_unit, n_cuts, u));
      alone[u] = x.run == kBadUnit || !is_short(x.nr, x.k1 - x.k0) ? 0 : x.nr <= kTileRows ? 1 : 2;
    }
    __syncthreads();
    // short pieces that are taken side by side: as many of one or of two tiles of rows as follow one another in a stretch, up to the
    // waves of a workgroup
    const int waves = attend_waves(p.a.d);
    for (int u = tid; u < (int)n[kUnits]; u += kPlanThreads) {
      const int s = last_at_most(first_unit, n_cuts, u);
      const int first = first_unit[s], end = first_unit[s + 1];
      AttendUnit unit = piece(u, s);
      int run = 0;
      while (run < waves && u + run < end && alone[u + run] && alone[u + run] == alone[u]) ++run;
      if (run > 1) unit.run = run;
      p.units[u] = unit;
      if (u == first) put_stretch(s, first, end, unit);
    }
    for (int s = tid; s < n_cuts; s += kPlanThreads)
      if (first_unit[s] == first_unit[s + 1]) p.stretches[s].first = p.stretches[s].end = 0;
  }
  int64_t slot = at[kSlots], j = at[kJoins], row = at[kRows];
  walk([&](int x, const Block& k) {
    const int pieces = pieces_at(x, k), step = k.m / kSlotRows;
    if (!leaves_sums(k, pieces)) return;
    if (k.seg >= n_groups) {
      const int b = k.seg - n_groups;
      AttendJoin e = {};
      e.r0 = seqs[b].t0 * G + k.i * k.m;
      e.nr = k.nr;
      e.own_slot = (int)slot;
      e.own_pieces = pieces;
      e.own_step = step;
      e.first = (int)row;
      row += e.nr;
      e.group = seqs[b].shared > 0 ? group_of(cu_group, n_groups, b) : -1;
      if (e.group < 0) atomicMax(&most_pieces, pieces);
      p.joins[j++] = e;
    }
    slot += (int64_t)pieces * step;
  });
  __syncthreads();
  // 16 lanes for each block that is joined, a lane for each row
  for (int64_t x = tid >> 4; x < n[kJoins]; x += kPlanThreads / 16) {
    const AttendJoin e = p.joins[x];
    for (int r = tid & 15; r < e.nr; r += 16) {
      AttendRow o = {};
      o.row = e.r0 + r;
      o.own_at = e.own_slot * kSlotRows + r;
      o.own_pieces = e.own_pieces;
      o.own_step = e.own_step * kSlotRows;
      if (e.group >= 0) {  // (the blocks of a prefix may be cut differently)
        const PlanGroup g = groups[e.group];
        const int m = block_rows(g.tokens * G, p.a.d), in = o.row - g.t0 * G, x = seg_start[e.group] + in / m;
        if (in >= 0 && in < g.tokens * G) {
          o.pre_pieces = stretched ? pieces_at(x, Block()) : g.pieces;
          o.pre_at = (stretched ? slot_of[x] : g.slot + in / m * g.pieces * (m / kSlotRows)) * kSlotRows + in % m;
          o.pre_step = m;
        }
        atomicMax(&most_pieces, o.own_pieces + o.pre_pieces);
      }
      p.rows[e.first + r] = o;
    }
  }
  __syncthreads();
  if (tid == 0) {
    p.header->n_stretches = stretched ? n_cuts : (int)n[kUnits];
    p.header->n_rows = (int)n[kRows];
    p.header->most_pieces = most_pieces;
    p.header->print = p.print;
  }
}

struct JoinDev {
  const AttendHeader* header;
  const AttendRow* rows;
  const float* sums;
  const float2* stats;
  const float* v_scale;
  uint16_t* out;
  float* lse;
  uint64_t print;
  int64_t o_ts, o_hs;
  int H, H_kv, G;
};

// Rows of several pieces: out = sum_p f_p O_p / sum_p f_p l_p with f_p = 2^(m_p - max m), added in an order that the plan alone
// fixes.  Bound by its dependent reads (record; maxima, weights' sums and values together) where rows are few and by reading the sums
// where they are many: d / 4 lanes take a row's pieces one after the other, four in flight, 16 bytes a lane; with more than 16 pieces to
// a row, or more than 4 of few rows, all of the workgroup's lanes take one row, every eighth (sixteenth, d = 64) piece each group of lanes
// (from 5 pieces on for all: one token behind 1000 keys 6 % faster, but 32 sequences that share 8K 6 to 14 % slower).
// 32 (row, KV head) pairs of 7 pieces 3.3 us, 2048 of 23 or 24 8.0, 33760 of two or three 13.8.  (Compiled with NaNs honoured: invalid rows have a NaN for l.)
template <int D>
__global__ __launch_bounds__(256) void attend_join_kernel(const JoinDev p) {
  constexpr int L = D / 4, GROUPS = 256 / L;
  __shared__ float4 part[GROUPS][L];
  __shared__ float2 stat[GROUPS];
  asm volatile("" ::"s"(p.rows), "s"(p.sums), "s"(p.stats), "s"(p.v_scale), "s"(p.out), "s"(p.lse), "s"(p.print), "s"(p.o_ts), "s"(p.o_hs),
               "s"(p.H), "s"(p.H_kv), "s"(p.G));  // (all read at once)
  const auto header = reinterpret_cast<const __attribute__((address_space(4))) AttendHeader*>(reinterpret_cast<uintptr_t>(p.header));
  const uint64_t print = header->print;
  const uint32_t n_rows = (uint32_t)header->n_rows, H_kv = (uint32_t)p.H_kv;
  const bool together = header->most_pieces > (n_rows * H_kv <= 1024 ? 4 : 16);
  const int group = threadIdx.x / L, c = threadIdx.x % L, step = together ? GROUPS : 1, first = together ? group : 0;
  // (without a plan the pieces' kernel has filled the outputs)
  const uint32_t n_items = print == p.print ? n_rows * H_kv : 0, stride = gridDim.x * (together ? 1 : GROUPS);
  for (uint32_t item0 = blockIdx.x * (together ? 1 : GROUPS); item0 < n_items; item0 += stride) {
    const uint32_t item = together ? item0 : item0 + group;
    const bool active = item < n_items;
    const int g = (int)(item % H_kv);
    AttendRow r = {};
    if (active) r = p.rows[item / H_kv];
    const float scale = p.v_scale ? p.v_scale[g] : 1.f;
    const int n = r.own_pieces + r.pre_pieces;
    // index of piece q's row among all rows of the workspace: pieces are whole slots apart
    const uint32_t own_step = r.own_step * H_kv, pre_step = r.pre_step * H_kv;
    const uint32_t own_at = ((uint32_t)r.own_at / kSlotRows * H_kv + g) * kSlotRows + r.own_at % kSlotRows;
    const uint32_t pre_at = ((uint32_t)r.pre_at / kSlotRows * H_kv + g) * kSlotRows + r.pre_at % kSlotRows - r.own_pieces * pre_step;
    float top = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int q = first; q < n; q += 4 * step) {
      float4 x[4];
      float2 s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // (beyond the last: its values again, with a weight of zero)
        const int piece = min(q + i * step, n - 1);
        const size_t place = piece < r.own_pieces ? own_at + piece * own_step : pre_at + piece * pre_step;
        s[i] = p.stats[place];
        x[i] = *reinterpret_cast<const float4*>(p.sums + place * D + c * 4);
        if (q + i * step >= n) s[i] = make_float2(-INFINITY, 0.f);
      }
      const float next = fmaxf(fmaxf(fmaxf(s[0].x, s[1].x), fmaxf(s[2].x, s[3].x)), top);
      const float base = next == -INFINITY ? 0.f : next, old = exp2f(top - base);
      top = next;
      sum *= old;
      acc.x *= old; acc.y *= old; acc.z *= old; acc.w *= old;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float w = exp2f(s[i].x - base);
        sum += w * s[i].y;
        acc.x += w * x[i].x; acc.y += w * x[i].y; acc.z += w * x[i].z; acc.w += w * x[i].w;
      }
    }
    if (together) {  // the groups' sums, in their order
      part[group][c] = acc;
      if (c == 0) stat[group] = make_float2(top, sum);
      __syncthreads();
      if (group == 0) {
        top = -INFINITY;
#pragma unroll
        for (int x = 0; x < GROUPS; ++x) top = fmaxf(top, stat[x].x);
        const float base = top == -INFINITY ? 0.f : top;
        sum = 0.f;
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int x = 0; x < GROUPS; ++x) {
          const float f = exp2f(stat[x].x - base);
          sum += f * stat[x].y;
          const float4 o = part[x][c];
          acc.x += f * o.x; acc.y += f * o.y; acc.z += f * o.z; acc.w += f * o.w;
        }
      }
      __syncthreads();
      if (group != 0) continue;
    }
    if (!active) continue;
    const int token = r.row / p.G, h = g * p.G + r.row % p.G;
    const float mul = (sum == 0.f ? 0.f : 1.f / sum) * scale;
    uint16_t* dst = p.out + token * p.o_ts + h * p.o_hs + c * 4;
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16_pair(acc.x * mul, acc.y * mul), pack_bf16_pair(acc.z * mul, acc.w * mul));
    if (c == 0 && p.lse) p.lse[(int64_t)token * p.H + h] = sum == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) + log2f(sum)) * 0.69314718055994531f;
  }
}

void launch_attend_join(const AttendDev& a, int d, hipStream_t stream) {
  const int grid = (int)(a.most_items < 2048 ? a.most_items : 2048);
  if (grid < 1) return;
  const JoinDev p = {a.header, a.rows, a.sums, a.stats, a.v_scale, a.out, a.lse, a.print, a.o_ts, a.o_hs, a.H, a.H_kv, a.G};
  if (d == 128) hipLaunchKernelGGL(attend_join_kernel<128>, dim3(grid), dim3(256), 0, stream, p);
  else hipLaunchKernelGGL(attend_join_kernel<64>, dim3(grid), dim3(256), 0, stream, p);
}

sp_status check_attend_shape(const sp_attend_args* a) {
  if (!a) return SP_ENULL;
  if (a->B < 1 || a->H < 1 || a->H > 1024 || a->H_kv < 1 || a->H % a->H_kv != 0 || a->H / a->H_kv > 16) return SP_EINVAL;
  if (a->d != 64 && a->d != 128) return SP_EINVAL;
  if (a->T_new < 0 || a->n_groups < 0 || a->n_groups > a->B) return SP_EINVAL;
  if (a->T_new >= INT64_C(0x80000000) / a->H) return SP_EINVAL;
  if (a->n_rows < 1 || a->n_rows > kMostKeys) return SP_EINVAL;
  if (a->cache_dtype != SP_K_BF16 && a->cache_dtype != SP_K_FP8_E4M3 && a->cache_dtype != SP_K_MXFP4) return SP_EINVAL;
  if (a->d_block_table) {
    if (a->page_size < 8 || (a->page_size & (a->page_size - 1)) != 0 || a->blocks_per_seq < 1) return SP_EINVAL;
    if ((int64_t)a->blocks_per_seq * a->page_size > kMostKeys || a->n_rows % a->page_size != 0) return SP_EINVAL;
  }
  return SP_OK;
}

sp_status check_attend_plan_args(const sp_attend_args* a) {
  const sp_status st = check_attend_shape(a);
  if (st != SP_OK) return st;
  if (!a->d_cu_new || !a->d_kv_len) return SP_ENULL;
  if (!a->d_block_table && !a->d_cu_cache) return SP_ENULL;
  if (a->d_block_table && a->d_cu_cache) return SP_EINVAL;
  if (a->n_groups > 0 && (!a->d_cu_group || !a->d_prefix_len)) return SP_ENULL;
  if (a->n_groups == 0 && (a->d_cu_group || a->d_prefix_len)) return SP_EINVAL;
  if (a->n_groups > 0 && !a->d_block_table) return SP_EUNSUPPORTED;
  const AttendCaps c = attend_caps(a);
  if (c.slots * kSlotRows * a->H_kv >= INT64_C(0x100000000) || c.slots * kSlotRows >= INT64_C(0x7fffffff) || c.rows >= INT64_C(0x7fffffff) || c.units * a->H_kv * 64 * attend_waves(a->d) >= INT64_C(0x100000000))
    return SP_EINVAL;  // (the last: threads of a launch)
  if (!a->d_plan) return SP_ENULL;
  if (reinterpret_cast<uintptr_t>(a->d_plan) & 255u) return SP_EALIGN;
  if (a->plan_bytes < attend_plan_layout(a).bytes) return SP_EWORKSPACE;
  return SP_OK;
}

}  // namespace sp

extern "C" size_t sp_attend_plan_bytes(const sp_attend_args* a) {
  return sp::check_attend_shape(a) == SP_OK ? sp::attend_plan_layout(a).bytes : 0;
}

extern "C" sp_status sp_attend_plan(const sp_attend_args* a, void* hip_stream) {
  using namespace sp;
  const sp_status st = check_attend_plan_args(a);
  if (st != SP_OK) return st;
  const AttendCaps c = attend_caps(a);
  const AttendPlanLayout l = attend_plan_layout(a);
  char* base = static_cast<char*>(a->d_plan);
  PlanDev p;
  p.a = *a;
  p.G = a->H / a->H_kv;
  p.cap_blocks = c.blocks; p.cap_units = c.units; p.cap_joins = c.joins; p.cap_rows = c.rows; p.cap_slots = c.slots;
  p.print = attend_print(a);
  p.header = reinterpret_cast<AttendHeader*>(base);
  p.units = reinterpret_cast<AttendUnit*>(base + l.units);
  p.stretches = reinterpret_cast<AttendStretch*>(base + l.stretches);
  p.joins = reinterpret_cast<AttendJoin*>(base + l.joins);
  p.rows = reinterpret_cast<AttendRow*>(base + l.rows);
  p.seg_start = reinterpret_cast<int32_t*>(base + l.seg_start);
  p.seqs = reinterpret_cast<PlanSeq*>(base + l.seqs);
  p.groups = reinterpret_cast<PlanGroup*>(base + l.groups);
  hipLaunchKernelGGL(attend_plan_kernel, dim3(1), dim3(kPlanThreads), 0, static_cast<hipStream_t>(hip_stream), p);
  return launch_status();
}
