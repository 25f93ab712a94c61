// sp_cache_read: tokens of a (paged) cache as bf16 keys and values.
//
// One pass: bound by HBM (reads d/2 + d/32, d or 2 d bytes of a token's key or value of a head, writes 2 d).  A workgroup takes a few rows:
// their places in the cache are looked up once, then every lane turns 8 elements into 16 bytes of the output, of four rows at a time.
// 111K tokens of d = 64 out of 4 bits: 61 us, 4.8 TB/s (a large copy: 5.2); 3200 chosen tokens, d 128, 7.8 us: a launch and four dependent reads.  (A division by the
// number of heads for every 16 bytes: 104 us.)
#include "sp_score_internal.h"

namespace sp {

namespace {

constexpr int kRows = 8;    // most rows of a workgroup
constexpr int kAhead = 4;   // rows of a lane that are on their way together
constexpr int64_t kMostRows = INT64_C(1) << 25;  // of a call: a launch has fewer than 2^32 threads

struct ReadDev {
  int B, H_kv, T, rows, arrays, lg_page, blocks_per_seq;
  int64_t c_ts, c_hs, c_ps, room;  // room: tokens of a sequence in a paged cache
  int64_t out_ts[2], out_hs[2];
  uint32_t n_pages, n_rows;
  const int32_t* cu_rows;
  const int32_t* first;
  const int32_t* index;
  const int32_t* cu_cache;
  const int32_t* table;
  const char* cache[2];            // keys, values
  const float* scale[2];
  const uint8_t* block_scale[2];
  uint16_t* out[2];
};

// eight stored elements, as they come from memory
template <int KIND> struct Stored { u32x4 x; };
template <> struct Stored<SP_K_FP8_E4M3> { uint2 x; float scale; };
template <> struct Stored<SP_K_MXFP4> { uint32_t x, scale; };

__device__ __forceinline__ u32x4 as_bf16(const Stored<SP_K_BF16>& s) { return s.x; }
__device__ __forceinline__ u32x4 as_bf16(const Stored<SP_K_FP8_E4M3>& s) {
  u32x4 out;
  const uint32_t w[2] = {s.x.x, s.x.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
    out[2 * i] = pack_bf16_pair(a[0] * s.scale, a[1] * s.scale);
    out[2 * i + 1] = pack_bf16_pair(b[0] * s.scale, b[1] * s.scale);
  }
  return out;
}
// (the instruction takes the exponent of its scale operand: 0 stands for 2^-127, 255 for NaN, as in E8M0; all results are exact)
__device__ __forceinline__ u32x4 as_bf16(const Stored<SP_K_MXFP4>& s) {
  const float scale = __uint_as_float(s.scale << 23);
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(s.x, scale, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(s.x, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(s.x, scale, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(s.x, scale, 3))};
}

// eight elements from element `at` of a cache on
template <int KIND>
__device__ __forceinline__ void load(Stored<KIND>& x, const char* cache, const uint8_t* block_scale, float scale, int64_t at) {
  if constexpr (KIND == SP_K_MXFP4) {
    x.x = *reinterpret_cast<const uint32_t*>(cache + at / 2);
    x.scale = block_scale[at / 32];
  } else if constexpr (KIND == SP_K_FP8_E4M3) {
    x.x = *reinterpret_cast<const uint2*>(cache + at);
    x.scale = scale;
  } else {
    x.x = *reinterpret_cast<const u32x4*>(cache + at * 2);
  }
}

}  // namespace

template <int D, int KIND>
__global__ __launch_bounds__(256) void read_kernel(const ReadDev p) {
  constexpr int C = D / 8;  // chunks of eight elements of a row
  __shared__ int32_t cu_lds[kStagedOffsets];
  __shared__ int64_t place[kRows];  // element offset of the row's token in the cache, or -1
  const int32_t* cu = staged_offsets(p.cu_rows, p.B, cu_lds);
  const int first = blockIdx.x * p.rows;
  const int n = min(min(p.rows, p.T - first), cu[p.B] - first);
  if (n <= 0) return;
  if ((int)threadIdx.x < n) {
    const int t = first + threadIdx.x;
    const int b = upper_segment(cu, p.B, t);
    const int64_t i = (int64_t)(p.index ? p.index[t] : t - cu[b]) + (p.first ? p.first[b] : 0);
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
    place[threadIdx.x] = at;
  }
  __syncthreads();
  // 256 threads take as many rows' chunks as they are enough for, or one row's in turn
  const int chunks = p.H_kv * C, together = max(256 / chunks, 1), step = chunks > 256 ? 256 : chunks;
  const int sub = chunks > 256 ? 0 : (int)threadIdx.x / chunks;
  if (sub >= together) return;
  for (int ch = (int)threadIdx.x - sub * chunks; ch < chunks; ch += step) {
    const int c = ch % C, g = ch / C;
    const int64_t in = g * p.c_hs + 8 * c;
    uint16_t* const k_out = p.out[0] + g * p.out_hs[0] + 8 * c;
    uint16_t* const v_out = p.out[1] + g * p.out_hs[1] + 8 * c;
    const float k_scale = KIND == SP_K_FP8_E4M3 && p.scale[0] ? p.scale[0][g] : 1.f, v_scale = KIND == SP_K_FP8_E4M3 && p.scale[1] ? p.scale[1][g] : 1.f;
    for (int t0 = sub; t0 < n; t0 += together * kAhead) {
      Stored<KIND> k[kAhead], v[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int64_t at = max(place[min(t0 + i * together, n - 1)], (int64_t)0) + in;  // (a row without a place: the pool's first, and not used)
        load<KIND>(k[i], p.cache[0], p.block_scale[0], k_scale, at);
        if (p.arrays == 2) load<KIND>(v[i], p.cache[1], p.block_scale[1], v_scale, at);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int tl = t0 + i * together;
        if (tl >= n) break;
        constexpr uint32_t nan2 = 0x7fc07fc0u;
        const u32x4 none = {nan2, nan2, nan2, nan2};
        const bool there = place[tl] >= 0;
        *reinterpret_cast<u32x4*>(k_out + (int64_t)(first + tl) * p.out_ts[0]) = there ? as_bf16(k[i]) : none;
        if (p.arrays == 2) *reinterpret_cast<u32x4*>(v_out + (int64_t)(first + tl) * p.out_ts[1]) = there ? as_bf16(v[i]) : none;
      }
    }
  }
}

namespace {

sp_status check_read(const sp_cache_read_args* a) {
  if (!a) return SP_ENULL;
  const bool values = a->d_v_cache != nullptr, fp4 = a->cache_dtype == SP_K_MXFP4;
  if (a->B < 1 || a->H_kv < 1 || a->H_kv > 1024 || (a->d != 64 && a->d != 128) || a->T_rows < 0 || a->T_rows > kMostRows) return SP_EINVAL;
  if (a->n_rows < 1 || a->n_rows >= INT64_C(0x80000000)) return SP_EINVAL;
  if (a->cache_dtype != SP_K_BF16 && a->cache_dtype != SP_K_FP8_E4M3 && !fp4) return SP_EINVAL;
  if (a->cache_dtype != SP_K_FP8_E4M3 && (a->d_k_scale || a->d_v_scale)) return SP_EINVAL;
  if (!fp4 && (a->d_k_block_scale || a->d_v_block_scale)) return SP_EINVAL;
  if (!values && (a->d_v_scale || a->d_v_block_scale)) return SP_EINVAL;
  if (!a->d_cu_rows || !a->d_k_cache || (a->T_rows > 0 && (!a->d_k_out || (values && !a->d_v_out)))) return SP_ENULL;
  if (!values && a->d_v_out) return SP_ENULL;
  if (fp4 && (!a->d_k_block_scale || (values && !a->d_v_block_scale))) return SP_ENULL;
  if (!a->d_block_table && !a->d_cu_cache) return SP_ENULL;
  if (a->d_block_table && a->d_cu_cache) return SP_EINVAL;
  const int64_t cache[] = {a->cache_token_stride, a->cache_head_stride, a->d_block_table ? a->cache_page_stride : 0};
  const int64_t out[] = {a->k_out_token_stride, a->k_out_head_stride, values ? a->v_out_token_stride : 0, values ? a->v_out_head_stride : 0};
  for (int64_t s : cache) if (s < 0) return SP_EINVAL;
  for (int64_t s : out) if (s < 0) return SP_EINVAL;
  if (a->d_block_table) {
    if (a->page_size < 8 || (a->page_size & (a->page_size - 1)) != 0 || a->blocks_per_seq < 1) return SP_EINVAL;
    if ((int64_t)a->blocks_per_seq * a->page_size >= INT64_C(0x80000000) || a->n_rows % a->page_size != 0) return SP_EINVAL;
  }
  // rows of an output that lie in one another would be written by several lanes at once, and so would keys over values
  if (a->H_kv > 1 && (out[1] < a->d || (values && out[3] < a->d))) return SP_EINVAL;
  if (a->T_rows > 1 && (out[0] < a->d || (values && out[2] < a->d))) return SP_EINVAL;
  if (values && a->d_k_out && a->d_k_out == a->d_v_out) return SP_EINVAL;
  for (int64_t s : cache) if (s & (cache_stride_unit(a->cache_dtype, a->d) - 1)) return SP_EALIGN;
  if (!aligned_scales(a->d_k_block_scale, a->d) || !aligned_scales(a->d_v_block_scale, a->d)) return SP_EALIGN;
  for (int64_t s : out) if (s & 7) return SP_EALIGN;
  if (!aligned16(a->d_k_cache) || !aligned16(a->d_v_cache) || !aligned16(a->d_k_out) || !aligned16(a->d_v_out)) return SP_EALIGN;
  return SP_OK;
}

template <int D>
void launch_read(const ReadDev& p, int dtype, dim3 grid, hipStream_t stream) {
  if (dtype == SP_K_MXFP4) hipLaunchKernelGGL((read_kernel<D, SP_K_MXFP4>), grid, dim3(256), 0, stream, p);
  else if (dtype == SP_K_FP8_E4M3) hipLaunchKernelGGL((read_kernel<D, SP_K_FP8_E4M3>), grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((read_kernel<D, SP_K_BF16>), grid, dim3(256), 0, stream, p);
}

}  // namespace

}  // namespace sp

extern "C" sp_status sp_cache_read(const sp_cache_read_args* a, void* hip_stream) {
  using namespace sp;
  const sp_status st = check_read(a);
  if (st != SP_OK) return st;
  if (a->T_rows == 0) return SP_OK;
  ReadDev p;
  p.B = a->B; p.H_kv = a->H_kv; p.T = (int)a->T_rows;
  p.arrays = a->d_v_cache ? 2 : 1;
  p.c_ts = a->cache_token_stride; p.c_hs = a->cache_head_stride; p.c_ps = a->cache_page_stride;
  p.lg_page = 0;
  while (a->d_block_table && (1 << p.lg_page) < a->page_size) ++p.lg_page;
  p.blocks_per_seq = a->blocks_per_seq;
  p.room = (int64_t)a->blocks_per_seq * a->page_size;
  p.n_pages = a->d_block_table ? (uint32_t)(a->n_rows / a->page_size) : 0;
  p.n_rows = (uint32_t)a->n_rows;
  p.cu_rows = a->d_cu_rows; p.first = a->d_first; p.index = a->d_index; p.cu_cache = a->d_cu_cache; p.table = a->d_block_table;
  p.out_ts[0] = a->k_out_token_stride; p.out_hs[0] = a->k_out_head_stride;
  p.out_ts[1] = a->v_out_token_stride; p.out_hs[1] = a->v_out_head_stride;
  p.cache[0] = static_cast<const char*>(a->d_k_cache); p.cache[1] = static_cast<const char*>(a->d_v_cache);
  p.scale[0] = a->d_k_scale; p.scale[1] = a->d_v_scale;
  p.block_scale[0] = a->d_k_block_scale; p.block_scale[1] = a->d_v_block_scale;
  p.out[0] = static_cast<uint16_t*>(a->d_k_out); p.out[1] = static_cast<uint16_t*>(a->d_v_out);
  // few rows: one to a workgroup
  p.rows = (int)std::min<int64_t>(kRows, std::max<int64_t>(1, a->T_rows / 2048));
  const dim3 grid((unsigned)((a->T_rows + p.rows - 1) / p.rows));
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (a->d == 128) launch_read<128>(p, a->cache_dtype, grid, stream);
  else launch_read<64>(p, a->cache_dtype, grid, stream);
  return launch_status();
}
