// sp_attend_plan: the list of pieces of work of an attention call, made on the device from the lengths (which only the
// device knows, so that a captured graph follows them), and the kernel that joins the pieces' sums.  The cut itself is in sp_attend_plan.h.
// The plan is bound by its chain of dependent reads and barriers (one workgroup); a step makes it once for all layers.
#include "sp_attend_internal.h"

namespace sp {

namespace {

struct PlanSeq { int32_t t0, n, len, shared; };                 // len -1: invalid
struct PlanGroup { int32_t shared, active, t0, tokens, slot, pieces, pad[2]; };

struct PlanDev {
  sp_attend_args a;   // (host pointers in it are not used)
  int G;
  int64_t cap_units, cap_joins, cap_slots;
  uint64_t print;
  AttendHeader* header;
  AttendUnit* units;
  AttendJoin* joins;
  int32_t* seg_start;
  PlanSeq* seqs;
  PlanGroup* groups;
};

__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

__device__ __forceinline__ int group_of(const PlanDev& p, int b) {
  const int n = p.a.n_groups;
  if (n == 0 || b < p.a.d_cu_group[0] || b >= p.a.d_cu_group[n]) return -1;
  return upper_segment(p.a.d_cu_group, n, b);
}

// exclusive prefix of v over the workgroup's 1024 threads, and the sum over all of them
__device__ __forceinline__ int64_t block_exclusive(int64_t v, int64_t* lds, int64_t* total) {
  const int t = threadIdx.x;
  lds[t] = v;
  __syncthreads();
  for (int off = 1; off < 1024; off <<= 1) {
    const int64_t x = t >= off ? lds[t - off] : 0;
    __syncthreads();
    lds[t] += x;
    __syncthreads();
  }
  const int64_t incl = lds[t];
  *total = lds[1023];
  __syncthreads();
  return incl - v;
}

struct Block {       // a block of rows, as the walk over all blocks meets it
  int seg, i;        // segment (prefixes first, then sequences), block of it
  int64_t rows;      // of the segment
  int keys;          // of the block
};

}  // namespace

__global__ __launch_bounds__(1024) void attend_plan_kernel(const PlanDev p) {
  __shared__ int64_t scan[1024];
  const int tid = threadIdx.x, B = p.a.B, n_groups = p.a.n_groups, G = p.G, T = (int)p.a.T_new;
  if (tid == 0) p.header->print = 0;

  // the sequences' new tokens and lengths, as far as they are valid
  for (int b = tid; b < B; b += 1024) {
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
    p.seqs[b] = s;
  }
  for (int g = tid; g < n_groups; g += 1024) {
    PlanGroup x = {};
    const int b0 = clamp_int(p.a.d_cu_group[g], 0, B), b1 = clamp_int(p.a.d_cu_group[g + 1], b0, B);
    x.shared = max(p.a.d_prefix_len[g], 0);
    x.t0 = clamp_int(p.a.d_cu_new[b0], 0, T);
    x.tokens = clamp_int(p.a.d_cu_new[b1], x.t0, T) - x.t0;
    p.groups[g] = x;
  }
  __syncthreads();
  // a prefix is cut to what all queries of the group see
  if (n_groups > 0) {
    for (int b = tid; b < B; b += 1024) {
      const int g = group_of(p, b);
      if (g < 0) continue;
      const PlanSeq s = p.seqs[b];
      if (b == p.a.d_cu_group[g]) atomicMin(&p.groups[g].shared, max(s.len, 0));
      if (s.n > 0) {
        atomicMin(&p.groups[g].shared, s.len < 0 ? 0 : max(s.len - s.n, 0));
        atomicAdd(&p.groups[g].active, 1);
      }
    }
    __syncthreads();
    for (int g = tid; g < n_groups; g += 1024) {  // (atomics are done in L2: read there)
      const int active = __hip_atomic_load(&p.groups[g].active, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const int shared = __hip_atomic_load(&p.groups[g].shared, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      p.groups[g].shared = shares((int64_t)p.groups[g].tokens * G, active) ? shared : 0;
    }
    __syncthreads();
    for (int b = tid; b < B; b += 1024) {
      const int g = group_of(p, b);
      if (g >= 0) p.seqs[b].shared = p.groups[g].shared;
    }
    __syncthreads();
  }
  block_prefix_table(n_groups + B, [&](int s) -> int32_t {
    if (s < n_groups) return p.groups[s].shared > 0 ? segment_blocks((int64_t)p.groups[s].tokens * G) : 0;
    const int n = p.seqs[s - n_groups].n;
    return n > 0 ? segment_blocks((int64_t)n * G) : 0;
  }, p.seg_start);
  const int n_blocks = p.seg_start[n_groups + B], n_prefix = p.seg_start[n_groups];

  // Every thread walks over a run of blocks, several times.  Prefixes first, then the sequences' blocks from the last to the
  // first: of a causal segment's blocks the last have the most keys.
  const int per = (n_blocks + 1023) / 1024;
  const int x0 = min(n_blocks, tid * per), x1 = min(n_blocks, x0 + per);
  auto walk = [&](auto&& visit) {
    int seg = -1;
    for (int x = x0; x < x1; ++x) {
      const int flat = x < n_prefix ? x : n_blocks - 1 - (x - n_prefix);
      if (seg < 0 || flat < p.seg_start[seg] || flat >= p.seg_start[seg + 1]) seg = upper_segment(p.seg_start, n_groups + B, flat);
      Block k;
      k.seg = seg;
      k.i = flat - p.seg_start[seg];
      if (seg < n_groups) {
        k.rows = (int64_t)p.groups[seg].tokens * G;
        k.keys = p.groups[seg].shared;
      } else {
        const PlanSeq s = p.seqs[seg - n_groups];
        k.rows = (int64_t)s.n * G;
        k.keys = s.len < 0 ? 0 : own_block_keys(k.rows, k.i, G, s.n, s.len, s.shared);
      }
      visit(k);
    }
  };
  int64_t keys = 0, total_keys;
  walk([&](const Block& k) { keys += k.keys; });
  block_exclusive(keys, scan, &total_keys);
  const int cut = make_cut(total_keys, p.a.H_kv);
  auto joined = [&](const Block& k) { return k.seg >= n_groups && p.seqs[k.seg - n_groups].shared > 0; };
  auto leaves_sums = [&](const Block& k, int pieces) { return pieces > 1 || k.seg < n_groups || joined(k); };

  int64_t units = 0, slots = 0, joins = 0, n_units, n_slots, n_joins;
  walk([&](const Block& k) {
    const int pieces = pieces_of(k.keys, cut);
    units += pieces;
    if (leaves_sums(k, pieces)) {
      slots += (int64_t)pieces * (block_rows(k.rows) / kSlotRows);
      joins += k.seg >= n_groups;
    }
  });
  units = block_exclusive(units, scan, &n_units);
  slots = block_exclusive(slots, scan, &n_slots);
  joins = block_exclusive(joins, scan, &n_joins);
  if (n_units > p.cap_units || n_slots > p.cap_slots || n_joins > p.cap_joins) return;  // offsets that do not ascend: no plan

  int64_t u = units, slot = slots;
  walk([&](const Block& k) {
    const int pieces = pieces_of(k.keys, cut), m = block_rows(k.rows), step = m / kSlotRows;
    const bool sums = leaves_sums(k, pieces);
    AttendUnit unit;
    int t0, first = 0;
    if (k.seg < n_groups) {
      t0 = p.groups[k.seg].t0;
      unit.seq = clamp_int(p.a.d_cu_group[k.seg], 0, B - 1);
      unit.off = kNoLimit;
      unit.bad = 0;
      if (k.i == 0) {
        p.groups[k.seg].slot = (int)slot;
        p.groups[k.seg].pieces = pieces;
      }
    } else {
      const PlanSeq s = p.seqs[k.seg - n_groups];
      t0 = s.t0;
      first = s.shared;
      unit.seq = k.seg - n_groups;
      unit.off = s.len - s.n + 1 - s.t0;
      unit.bad = s.len < 0;
    }
    unit.r0 = t0 * G + k.i * m;
    unit.nr = (int)min((int64_t)m, k.rows - (int64_t)k.i * m);
    for (int q = 0; q < pieces; ++q) {
      unit.k0 = first + piece_start(k.keys, pieces, q);
      unit.k1 = first + piece_start(k.keys, pieces, q + 1);
      unit.slot = sums ? (int)(slot + (int64_t)q * step) : -1;
      p.units[u + q] = unit;
    }
    u += pieces;
    if (sums) slot += (int64_t)pieces * step;
  });
  __syncthreads();
  slot = slots;
  int64_t j = joins;
  walk([&](const Block& k) {
    const int pieces = pieces_of(k.keys, cut), m = block_rows(k.rows), step = m / kSlotRows;
    if (!leaves_sums(k, pieces)) return;
    if (k.seg >= n_groups) {
      const int b = k.seg - n_groups;
      AttendJoin e = {};
      e.r0 = p.seqs[b].t0 * G + k.i * m;
      e.nr = (int)min((int64_t)m, k.rows - (int64_t)k.i * m);
      e.own_slot = (int)slot;
      e.own_pieces = pieces;
      e.own_step = step;
      if (p.seqs[b].shared > 0) {
        const PlanGroup g = p.groups[group_of(p, b)];
        e.pre_slot = g.slot;
        e.pre_pieces = g.pieces;
        e.pre_r0 = g.t0 * G;
        e.pre_rows = block_rows((int64_t)g.tokens * G);
      }
      p.joins[j++] = e;
    }
    slot += (int64_t)pieces * step;
  });
  __syncthreads();
  if (tid == 0) {
    p.header->n_units = (int)n_units;
    p.header->n_joins = (int)n_joins;
    p.header->n_slots = (int)n_slots;
    p.header->print = p.print;
  }
}

// Rows of several pieces: out = sum_p f_p O_p / sum_p f_p l_p with f_p = 2^(m_p - max m), in the pieces' order, so that results
// do not depend on when the pieces were done.  A workgroup takes 16 rows of one KV head, 16 lanes a row, 8 (or 4) values a lane.
// (compiled with NaNs honoured: pieces mark invalid rows by a NaN in l)
template <int D>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendDev p) {
  constexpr int V = D / 16;
  if (p.header->print != p.print) return;  // (the pieces' kernel has filled the outputs)
  const int row = threadIdx.x >> 4, c = threadIdx.x & 15;
  const int64_t n_items = (int64_t)p.header->n_joins * p.join_slices * p.H_kv;
  for (int64_t item = blockIdx.x; item < n_items; item += gridDim.x) {
    const int g = (int)(item % p.H_kv);
    const int64_t e_i = item / p.H_kv;
    const AttendJoin e = p.joins[e_i / p.join_slices];
    const int slice = (int)(e_i % p.join_slices), r = slice * kSlotRows + row;
    if (r >= e.nr) continue;
    const int64_t flat = (int64_t)e.r0 + r;
    const int own = e.own_slot + slice;
    int pre = 0, pre_row = 0, pre_step = 0;
    if (e.pre_pieces > 0) {
      const int64_t at = flat - e.pre_r0;
      const int block = (int)(at / e.pre_rows), in = (int)(at % e.pre_rows);
      pre_step = e.pre_rows / kSlotRows;
      pre = e.pre_slot + block * e.pre_pieces * pre_step + in / kSlotRows;
      pre_row = in % kSlotRows;
    }
    const int n = e.own_pieces + e.pre_pieces;
    // index of piece q's row among all rows of the workspace
    auto place = [&](int q) -> int64_t {
      const bool mine = q < e.own_pieces;
      const int64_t slot = mine ? own + (int64_t)q * e.own_step : pre + (int64_t)(q - e.own_pieces) * pre_step;
      return (slot * p.H_kv + g) * kSlotRows + (mine ? row : pre_row);
    };
    float top = -INFINITY;
    for (int q = c; q < n; q += 16) top = fmaxf(top, p.stats[place(q)].x);
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 16));
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f, acc[V] = {};
#pragma unroll 4
    for (int q = 0; q < n; ++q) {
      const int64_t at = place(q);
      const float2 s = p.stats[at];
      const float f = exp2f(s.x - base);
      sum += f * s.y;
      const float* o = p.sums + at * D + c * V;
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const float4 x = *reinterpret_cast<const float4*>(o + i);
        acc[i] += f * x.x; acc[i + 1] += f * x.y; acc[i + 2] += f * x.z; acc[i + 3] += f * x.w;
      }
    }
    const int64_t token = flat / p.G;
    const int h = g * p.G + (int)(flat % p.G);
    const float mul = (sum == 0.f ? 0.f : 1.f / sum) * (p.v_scale ? p.v_scale[g] : 1.f);
    uint32_t w[V / 2];
#pragma unroll
    for (int i = 0; i < V; i += 2) w[i / 2] = pack_bf16_pair(acc[i] * mul, acc[i + 1] * mul);
    uint16_t* dst = p.out + token * p.o_ts + h * p.o_hs + c * V;
    if constexpr (V == 8) *reinterpret_cast<u32x4*>(dst) = u32x4{w[0], w[1], w[2], w[3]};
    else *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
    if (c == 0 && p.lse) p.lse[token * p.H + h] = sum == 0.f ? -INFINITY : (base + log2f(sum)) * 0.69314718055994531f;
  }
}

void launch_attend_join(const AttendDev& p, int d, int64_t items, hipStream_t stream) {
  const int grid = (int)(items < 2048 ? items : 2048);
  if (grid < 1) return;
  if (d == 128) hipLaunchKernelGGL(attend_join_kernel<128>, dim3(grid), dim3(256), 0, stream, p);
  else hipLaunchKernelGGL(attend_join_kernel<64>, dim3(grid), dim3(256), 0, stream, p);
}

sp_status check_attend_shape(const sp_attend_args* a) {
  if (!a) return SP_ENULL;
  if (a->B < 1 || a->H < 1 || a->H > 1024 || a->H_kv < 1 || a->H % a->H_kv != 0 || a->H / a->H_kv > 16) return SP_EINVAL;
  if (a->d != 64 && a->d != 128) return SP_EINVAL;
  if (a->T_new < 0 || a->n_groups < 0 || a->n_groups > a->B) return SP_EINVAL;
  if (a->T_new >= INT64_C(0x80000000) / a->H) return SP_EINVAL;
  if (a->n_rows < 1 || a->n_rows >= INT64_C(0x80000000)) return SP_EINVAL;
  if (a->cache_dtype != SP_K_BF16 && a->cache_dtype != SP_K_FP8_E4M3) return SP_EINVAL;
  if (a->d_block_table) {
    if (a->page_size < 8 || (a->page_size & (a->page_size - 1)) != 0 || a->blocks_per_seq < 1) return SP_EINVAL;
    if ((int64_t)a->blocks_per_seq * a->page_size >= INT64_C(0x80000000) || a->n_rows % a->page_size != 0) return SP_EINVAL;
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
  if (c.slots >= INT64_C(0x7fffffff) || c.units * a->H_kv >= INT64_C(0x7fffffff)) return SP_EINVAL;
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
  p.cap_units = c.units; p.cap_joins = c.joins; p.cap_slots = c.slots;
  p.print = attend_print(a);
  p.header = reinterpret_cast<AttendHeader*>(base);
  p.units = reinterpret_cast<AttendUnit*>(base + l.units);
  p.joins = reinterpret_cast<AttendJoin*>(base + l.joins);
  p.seg_start = reinterpret_cast<int32_t*>(base + l.seg_start);
  p.seqs = reinterpret_cast<PlanSeq*>(base + l.seqs);
  p.groups = reinterpret_cast<PlanGroup*>(base + l.groups);
  hipLaunchKernelGGL(attend_plan_kernel, dim3(1), dim3(1024), 0, static_cast<hipStream_t>(hip_stream), p);
  return launch_status();
}
