// sp_cache_append: new tokens' keys and values into a (paged) cache, keys and queries turned to their positions on the way.
//
// One pass over the projections: bound by HBM (reads (H + 2 H_kv) d bf16 values a token, writes H d of them and 2 H_kv d
// cache elements).  A workgroup takes a few tokens: their places in the cache are looked up once, the cosines and sines of
// all frequencies formed once for all heads of queries and keys (in LDS), then every lane moves 16-byte chunks; a lane has
// both halves of the pairs that it turns, chunk c and chunk c + d/16 of a row, so nothing is exchanged.  8192 tokens, H 32, H_kv 8,
// d 128, into 8 bits: 40.3 us, 4.6 TB/s; 100K tokens, d 64, bf16: 212 us, 5.3 TB/s (a large copy: 4.8); 64 single tokens 4.4 us.
// Into 4 bits the eight values of a lane and of its three neighbours, a quad, are one block: its largest magnitude goes round the quad, no LDS.  6592 tokens of H 64:
// 52 us, 4.8 TB/s.
#include <cmath>

#include "sp_append_grid.h"
#include "sp_score_internal.h"

namespace sp {

namespace {

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
  uint8_t* k_block_scale;
  uint8_t* v_block_scale;
};

// two fp32 values over a scale -> two E4M3 codes in the low half (nearest even, saturating; NaN stays NaN)
__device__ __forceinline__ uint32_t e4m3_pair(float a, float b, float scale) {
  a = scale == 0.f ? 0.f : a / scale;
  b = scale == 0.f ? 0.f : b / scale;
  a = a > 448.f ? 448.f : a < -448.f ? -448.f : a;
  b = b > 448.f ? 448.f : b < -448.f ? -448.f : b;
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu;
}

// The E8M0 scale of the 32 values that the lanes of a quad hold, eight each: the smallest power of two, 2^-125 at least, whose seven-fold
// is no less than any magnitude.  (The bits of a magnitude, taken as an integer, ascend with it, NaN and infinity last; 1.75 = 7/4 is
// where the exponent goes up.)
__device__ __forceinline__ uint32_t block_scale(const float (&x)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xf, 0xf, false));  // the quad's lanes 1, 0, 3, 2
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xf, 0xf, false));  // 2, 3, 0, 1
  return top >= 0x7f800000u ? 255u : (uint32_t)max((int)((top + 0x1fffffu) >> 23) - 2, 2);
}

// eight values over a scale -> E2M1 codes (the instruction rounds to nearest even and saturates at 6)
__device__ __forceinline__ uint32_t e2m1_codes(const float (&x)[8], float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
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

template <int D, int KIND, bool ROPE>
__global__ __launch_bounds__(256) void append_kernel(const AppendDev p) {
  constexpr bool FP8 = KIND == SP_K_FP8_E4M3, FP4 = KIND == SP_K_MXFP4;
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
    place[threadIdx.x] = at < 0 ? -1 : FP4 ? at / 2 : at * (FP8 ? 1 : 2);
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
      if constexpr (FP4) {  // (a quad's four chunks are one block: a row has a multiple of four)
        const int64_t at = place[tl] + (g * p.c_hs + 8 * c) / 2;
        char* codes = (key ? p.k_cache : p.v_cache) + at;
        uint8_t* scales = (key ? p.k_block_scale : p.v_block_scale) + at / 16;
        const uint32_t s_lo = block_scale(lo), s_hi = block_scale(hi);
        *reinterpret_cast<uint32_t*>(codes) = e2m1_codes(lo, __uint_as_float(s_lo << 23));
        *reinterpret_cast<uint32_t*>(codes + D / 4) = e2m1_codes(hi, __uint_as_float(s_hi << 23));
        if ((c & 3) == 0) {
          scales[0] = (uint8_t)s_lo;
          scales[D / 64] = (uint8_t)s_hi;
        }
        continue;
      }
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
  if (a->cache_dtype != SP_K_BF16 && a->cache_dtype != SP_K_FP8_E4M3 && a->cache_dtype != SP_K_MXFP4) return SP_EINVAL;
  if (a->cache_dtype != SP_K_FP8_E4M3 && (a->d_k_scale || a->d_v_scale)) return SP_EINVAL;
  if (a->cache_dtype != SP_K_MXFP4 && (a->d_k_block_scale || a->d_v_block_scale)) return SP_EINVAL;
  if (!finite_f32(a->rope_theta) || a->rope_theta < 0.f || (a->rope_theta > 0.f && a->d_inv_freq)) return SP_EINVAL;
  if (a->d_pos && a->rope_theta == 0.f && !a->d_inv_freq) return SP_EINVAL;
  if ((a->T_new > 0 && (!a->d_k || !a->d_v)) || !a->d_cu_new || !a->d_k_cache || !a->d_v_cache) return SP_ENULL;
  if (queries != (a->d_q_out != nullptr)) return SP_ENULL;
  if (a->cache_dtype == SP_K_MXFP4 && (!a->d_k_block_scale || !a->d_v_block_scale)) return SP_ENULL;
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
  if (a->d_k_cache == a->d_v_cache || (a->d_k_block_scale && a->d_k_block_scale == a->d_v_block_scale)) return SP_EINVAL;
  for (int64_t s : in) if (s & 7) return SP_EALIGN;
  for (int64_t s : out) if (s & (cache_stride_unit(a->cache_dtype, a->d) - 1)) return SP_EALIGN;
  if (!aligned_scales(a->d_k_block_scale, a->d) || !aligned_scales(a->d_v_block_scale, a->d)) return SP_EALIGN;
  if (!aligned16(a->d_q) || !aligned16(a->d_k) || !aligned16(a->d_v) || !aligned16(a->d_q_out) || !aligned16(a->d_k_cache) ||
      !aligned16(a->d_v_cache))
    return SP_EALIGN;
  return SP_OK;
}

template <int D, int KIND>
void launch_append(const AppendDev& p, bool rope, dim3 grid, hipStream_t stream) {
  if (rope) hipLaunchKernelGGL((append_kernel<D, KIND, true>), grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((append_kernel<D, KIND, false>), grid, dim3(256), 0, stream, p);
}

template <int D>
void launch_append(const AppendDev& p, int dtype, bool rope, dim3 grid, hipStream_t stream) {
  if (dtype == SP_K_MXFP4) launch_append<D, SP_K_MXFP4>(p, rope, grid, stream);
  else if (dtype == SP_K_FP8_E4M3) launch_append<D, SP_K_FP8_E4M3>(p, rope, grid, stream);
  else launch_append<D, SP_K_BF16>(p, rope, grid, stream);
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
  p.k_block_scale = a->d_k_block_scale; p.v_block_scale = a->d_v_block_scale;
  const AppendGrid cut = append_grid(a->T_new, p.H + 2 * p.H_kv, a->d, a->cache_dtype);
  p.tokens = cut.tokens;
  const dim3 grid(cut.blocks, cut.parts);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (a->d == 128) launch_append<128>(p, a->cache_dtype, rope, grid, stream);
  else launch_append<64>(p, a->cache_dtype, rope, grid, stream);
  return launch_status();
}
