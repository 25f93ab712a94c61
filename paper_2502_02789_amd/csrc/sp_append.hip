// sp_cache_append: new tokens' keys and values into a (paged) cache, keys and queries turned to their positions on the way.
//
// One pass over the projections: bound by HBM (reads (H + 2 H_kv) d bf16 values a token, writes H d of them and 2 H_kv d
// cache elements).  A workgroup takes a few tokens: their places in the cache are looked up once, the cosines and sines of
// all frequencies formed once for all heads of queries and keys (in LDS), then every lane moves 16-byte chunks; a lane has
// both halves of the pairs that it turns, chunk c and chunk c + d/16 of a row, so nothing is exchanged.  8192 tokens, H 32, H_kv 8,
// d 128, into 8 bits: 40.3 us, 4.6 TB/s; 100K tokens, d 64, bf16: 212 us, 5.3 TB/s (a large copy: 4.8); 64 single tokens 4.4 us.
#include <cmath>

#include "sp_score_internal.h"

namespace sp {

namespace {

constexpr int kTokens = 4;  // most tokens of a workgroup (8192 tokens into 8 bits: 8 takes 2 % longer, 16 18 %; 100K of d = 64: 3 and 8 %)

constexpr int64_t kMostTokens = INT64_C(1) << 25;  // of a call: a launch has fewer than 2^32 threads

struct AppendDev {
  int B, H, H_kv, T_new, tokens, lg_page, blocks_per_seq;
  int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs;
  int64_t c_ts, c_hs, c_ps, room;  // room: tokens of a sequence in a paged cache
  uint32_t n_pages, n_rows;
  double log2_theta;
  const double* inv_freq;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* cu_new;
  const int32_t* cache_len;
  const int32_t* pos;
  const int32_t* cu_cache;
  const int32_t* table;
  const float* k_scale;
  const float* v_scale;
  uint16_t* q_out;
  char* k_cache;
  char* v_cache;
};

// two fp32 values over a scale -> two E4M3 codes in the low half (nearest even, saturating; NaN stays NaN)
__device__ __forceinline__ uint32_t e4m3_pair(float a, float b, float scale) {
  a = scale == 0.f ? 0.f : a / scale;
  b = scale == 0.f ? 0.f : b / scale;
  a = a > 448.f ? 448.f : a < -448.f ? -448.f : a;
  b = b > 448.f ? 448.f : b < -448.f ? -448.f : b;
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu;
}

// eight values as the cache holds them
template <bool FP8>
__device__ __forceinline__ void store_chunk(char* at, const float (&x)[8], float scale) {
  if constexpr (FP8) {
    const uint32_t lo = e4m3_pair(x[0], x[1], scale) | e4m3_pair(x[2], x[3], scale) << 16;
    const uint32_t hi = e4m3_pair(x[4], x[5], scale) | e4m3_pair(x[6], x[7], scale) << 16;
    *reinterpret_cast<uint2*>(at) = make_uint2(lo, hi);
  } else {
    *reinterpret_cast<u32x4*>(at) = u32x4{pack_bf16_pair(x[0], x[1]), pack_bf16_pair(x[2], x[3]), pack_bf16_pair(x[4], x[5]),
                                          pack_bf16_pair(x[6], x[7])};
  }
}

__device__ __forceinline__ void widen(const u32x4 w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
}

}  // namespace

template <int D, bool FP8, bool ROPE>
__global__ __launch_bounds__(256) void append_kernel(const AppendDev p) {
  constexpr int C = D / 16;  // pairs of chunks of a row
  __shared__ int32_t cu_lds[kStagedOffsets];
  __shared__ int64_t place[kTokens];     // byte offset of the token's row in the cache, or -1
  __shared__ int32_t position[kTokens];
  __shared__ float2 turn[kTokens][D / 2 + 1];
  const int32_t* cu = staged_offsets(p.cu_new, p.B, cu_lds);
  const int first = blockIdx.x * p.tokens;
  const int n = min(min(p.tokens, p.T_new - first), cu[p.B] - first);
  if (n <= 0) return;
  if ((int)threadIdx.x < n) {
    const int t = first + threadIdx.x;
    const int b = upper_segment(cu, p.B, t);
    const int64_t i = (int64_t)(t - cu[b]) + (p.cache_len ? p.cache_len[b] : 0);
    const bool ours = t >= cu[b];  // (not in front of the first sequence)
    int64_t at = -1;
    if (p.table) {
      if (ours && i >= 0 && i < p.room) {
        const uint32_t page = (uint32_t)p.table[(int64_t)b * p.blocks_per_seq + (i >> p.lg_page)];
        if (page < p.n_pages) at = (int64_t)page * p.c_ps + (i & (((int64_t)1 << p.lg_page) - 1)) * p.c_ts;
      }
    } else {
      const int64_t lo = p.cu_cache[b], row = lo + i;
      if (ours && i >= 0 && lo >= 0 && row < p.cu_cache[b + 1] && row < (int64_t)p.n_rows) at = row * p.c_ts;
    }
    place[threadIdx.x] = at < 0 ? -1 : at * (FP8 ? 1 : 2);
    if constexpr (ROPE) position[threadIdx.x] = p.pos ? p.pos[t] : (int)i;
  }
  __syncthreads();
  if constexpr (ROPE) {
    const int m = threadIdx.x & (D / 2 - 1);
    const double f = p.inv_freq ? p.inv_freq[m] : rope_inv_freq(m, D / 2, p.log2_theta);
    for (int t = threadIdx.x / (D / 2); t < n; t += 256 / (D / 2)) turn[t][m] = rope_cos_sin_of((double)position[t] * f);
    __syncthreads();
  }
  const int rows = p.H + 2 * p.H_kv, items = n * rows * C;
  for (int it = blockIdx.y * 256 + threadIdx.x; it < items; it += 256 * gridDim.y) {
    const int c = it % C, r = it / C % rows, tl = it / C / rows;
    const int64_t t = first + tl;
    const uint16_t* src;
    if (r < p.H) src = p.q + t * p.q_ts + r * p.q_hs;
    else if (r < p.H + p.H_kv) src = p.k + t * p.k_ts + (r - p.H) * p.k_hs;
    else src = p.v + t * p.v_ts + (r - p.H - p.H_kv) * p.v_hs;
    float lo[8], hi[8];
    widen(*reinterpret_cast<const u32x4*>(src + 8 * c), lo);
    widen(*reinterpret_cast<const u32x4*>(src + D / 2 + 8 * c), hi);
    if (ROPE && r < p.H + p.H_kv) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 x = rope_turn_exact(lo[i], hi[i], turn[tl][8 * c + i]);
        lo[i] = x.x;
        hi[i] = x.y;
      }
    }
    if (r < p.H) {
      char* dst = reinterpret_cast<char*>(p.q_out + (t * p.H + r) * D + 8 * c);
      store_chunk<false>(dst, lo, 1.f);
      store_chunk<false>(dst + D, hi, 1.f);
    } else if (place[tl] >= 0) {
      const bool key = r < p.H + p.H_kv;
      const int g = r - p.H - (key ? 0 : p.H_kv);
      const float* scales = key ? p.k_scale : p.v_scale;
      const float scale = FP8 && scales ? scales[g] : 1.f;
      constexpr int E = FP8 ? 1 : 2;
      char* dst = (key ? p.k_cache : p.v_cache) + place[tl] + (g * p.c_hs + 8 * c) * E;
      store_chunk<FP8>(dst, lo, scale);
      store_chunk<FP8>(dst + D / 2 * E, hi, scale);
    }
  }
}

namespace {

sp_status check_append(const sp_cache_append_args* a) {
  if (!a) return SP_ENULL;
  const bool queries = a->d_q != nullptr;
  if (a->B < 1 || a->H_kv < 1 || a->H_kv > 1024 || (a->d != 64 && a->d != 128) || a->T_new < 0) return SP_EINVAL;
  if (queries && (a->H < 1 || a->H > 1024 || a->H % a->H_kv != 0 || a->H / a->H_kv > 16)) return SP_EINVAL;
  if (a->T_new >= INT64_C(0x80000000) / (queries ? a->H : a->H_kv) || a->T_new > kMostTokens) return SP_EINVAL;
  if (a->n_rows < 1 || a->n_rows >= INT64_C(0x80000000)) return SP_EINVAL;
  if (a->cache_dtype != SP_K_BF16 && a->cache_dtype != SP_K_FP8_E4M3) return SP_EINVAL;
  if (a->cache_dtype == SP_K_BF16 && (a->d_k_scale || a->d_v_scale)) return SP_EINVAL;
  if (!finite_f32(a->rope_theta) || a->rope_theta < 0.f || (a->rope_theta > 0.f && a->d_inv_freq)) return SP_EINVAL;
  if (a->d_pos && a->rope_theta == 0.f && !a->d_inv_freq) return SP_EINVAL;
  if ((a->T_new > 0 && (!a->d_k || !a->d_v)) || !a->d_cu_new || !a->d_k_cache || !a->d_v_cache) return SP_ENULL;
  if (queries != (a->d_q_out != nullptr)) return SP_ENULL;
  if (!a->d_block_table && !a->d_cu_cache) return SP_ENULL;
  if (a->d_block_table && a->d_cu_cache) return SP_EINVAL;
  const int64_t in[] = {a->k_token_stride, a->k_head_stride, a->v_token_stride, a->v_head_stride, queries ? a->q_token_stride : 0,
                        queries ? a->q_head_stride : 0};
  const int64_t out[] = {a->cache_token_stride, a->cache_head_stride, a->d_block_table ? a->cache_page_stride : 0};
  for (int64_t s : in) if (s < 0) return SP_EINVAL;
  for (int64_t s : out) if (s < 0) return SP_EINVAL;
  if (a->d_block_table) {
    if (a->page_size < 8 || (a->page_size & (a->page_size - 1)) != 0 || a->blocks_per_seq < 1) return SP_EINVAL;
    if ((int64_t)a->blocks_per_seq * a->page_size >= INT64_C(0x80000000) || a->n_rows % a->page_size != 0) return SP_EINVAL;
  }
  // heads and tokens that lie in one another would be written by several lanes at once, and so would keys over values
  if (a->H_kv > 1 && a->cache_head_stride < a->d) return SP_EINVAL;
  if ((a->d_block_table || a->n_rows > 1) && a->cache_token_stride < a->d) return SP_EINVAL;
  if (a->d_block_table && a->n_rows > a->page_size && a->cache_page_stride < a->d) return SP_EINVAL;
  if (a->d_k_cache == a->d_v_cache) return SP_EINVAL;
  for (int64_t s : in) if (s & 7) return SP_EALIGN;
  for (int64_t s : out) if (s & (a->cache_dtype == SP_K_FP8_E4M3 ? 15 : 7)) return SP_EALIGN;
  if (!aligned16(a->d_q) || !aligned16(a->d_k) || !aligned16(a->d_v) || !aligned16(a->d_q_out) || !aligned16(a->d_k_cache) ||
      !aligned16(a->d_v_cache))
    return SP_EALIGN;
  return SP_OK;
}

template <int D, bool FP8>
void launch_append(const AppendDev& p, bool rope, dim3 grid, hipStream_t stream) {
  if (rope) hipLaunchKernelGGL((append_kernel<D, FP8, true>), grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((append_kernel<D, FP8, false>), grid, dim3(256), 0, stream, p);
}

}  // namespace

}  // namespace sp

extern "C" sp_status sp_cache_append(const sp_cache_append_args* a, void* hip_stream) {
  using namespace sp;
  const sp_status st = check_append(a);
  if (st != SP_OK) return st;
  if (a->T_new == 0) return SP_OK;
  AppendDev p;
  p.B = a->B; p.H = a->d_q ? a->H : 0; p.H_kv = a->H_kv; p.T_new = (int)a->T_new;
  p.q_ts = a->q_token_stride; p.q_hs = a->q_head_stride;
  p.k_ts = a->k_token_stride; p.k_hs = a->k_head_stride;
  p.v_ts = a->v_token_stride; p.v_hs = a->v_head_stride;
  p.c_ts = a->cache_token_stride; p.c_hs = a->cache_head_stride; p.c_ps = a->cache_page_stride;
  p.lg_page = 0;
  while (a->d_block_table && (1 << p.lg_page) < a->page_size) ++p.lg_page;
  p.blocks_per_seq = a->blocks_per_seq;
  p.room = (int64_t)a->blocks_per_seq * a->page_size;
  p.n_pages = a->d_block_table ? (uint32_t)(a->n_rows / a->page_size) : 0;
  p.n_rows = (uint32_t)a->n_rows;
  const bool rope = a->rope_theta > 0.f || a->d_inv_freq;
  p.log2_theta = a->rope_theta > 0.f ? std::log2((double)a->rope_theta) : 0.0;
  p.inv_freq = a->d_inv_freq;
  p.q = static_cast<const uint16_t*>(a->d_q); p.k = static_cast<const uint16_t*>(a->d_k); p.v = static_cast<const uint16_t*>(a->d_v);
  p.cu_new = a->d_cu_new; p.cache_len = a->d_cache_len; p.pos = a->d_pos; p.cu_cache = a->d_cu_cache; p.table = a->d_block_table;
  p.k_scale = a->d_k_scale; p.v_scale = a->d_v_scale;
  p.q_out = static_cast<uint16_t*>(a->d_q_out);
  p.k_cache = static_cast<char*>(a->d_k_cache); p.v_cache = static_cast<char*>(a->d_v_cache);
  // few tokens: one to a workgroup, and several workgroups to a token, until the device has some hundred
  p.tokens = (int)std::min<int64_t>(kTokens, std::max<int64_t>(1, a->T_new / 512));
  const int64_t blocks = (a->T_new + p.tokens - 1) / p.tokens;
  const int chunks = (p.tokens * (p.H + 2 * p.H_kv) * (a->d / 16) + 255) / 256;
  const int parts = blocks >= 512 ? 1 : (int)std::min<int64_t>(chunks, 512 / blocks);
  const dim3 grid((unsigned)blocks, (unsigned)std::max(parts, 1));
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const bool fp8 = a->cache_dtype == SP_K_FP8_E4M3;
  if (a->d == 128) fp8 ? launch_append<128, true>(p, rope, grid, stream) : launch_append<128, false>(p, rope, grid, stream);
  else fp8 ? launch_append<64, true>(p, rope, grid, stream) : launch_append<64, false>(p, rope, grid, stream);
  return launch_status();
}
