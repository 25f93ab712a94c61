// sp_verify: which drafted tokens stand against the target's probabilities, and the token that is sampled behind them.
//
// Four kernels, bound by reading the logits once (the first; the others read the rows of one place of each sequence again):
//   stats     maximum and sum of exp of every row, 8192 logits to a workgroup
//   choose    per sequence: the rows' sums, how many tokens stand, hence the row that a token is sampled from; its parts' sums in fp64
//   residual  sums of max(p - q, 0) in parts, p and q normalised by those sums
//   pick      the part in which the sum passes r times the whole, and the token in it
// Which token is picked depends on sums over the whole vocabulary: a vocabulary of 128K has so many borders between tokens that sums in fp32, off by 1e-7, would pick
// another token once in some hundred calls.  The sampled row's weights are therefore formed and added in fp64; the order of all sums is fixed.
#include "sp_score_internal.h"

namespace sp {

namespace {

constexpr int kSlice = 8192;     // logits of a row that a workgroup of the first kernel takes
constexpr int kPart = 4096;      // ... of the others
constexpr int kMine = kPart / 256;
constexpr double kLog2e64 = 1.4426950408889634074;

struct RowStats { float top, sum; int32_t arg, pad; };   // of a slice: largest logit, sum of exp((z - top) / temperature), where the largest is
struct VerifyState {                                       // of a sequence
  double inv_t;
  float top_p, top_q;
  int32_t row_p, row_q;   // rows of the target and of the draft (-1: none) that the token is sampled from
  int32_t token;          // without draft logits: the token that is taken off, or -1
  int32_t sample;         // 0: nothing is sampled
};

struct VerifyDev {
  int B, V, T, slices, parts;
  const int32_t* cu;
  const int32_t* tokens;
  const void* target;
  const void* draft;
  int64_t target_stride, draft_stride;
  const float* temperature;
  const float* u;
  const float* r;
  const int32_t* past_len;
  int32_t* n_accepted;
  int32_t* out_tokens;
  float* logprob;
  int32_t* kept_len;
  RowStats* stats;     // [T + B rows of the target, T of the draft][slices]
  VerifyState* states; // [B]
  double* sum_p;       // [B][parts]
  double* sum_q;
  double* sum_w;
};

template <bool F32> __device__ __forceinline__ float logit(const void* row, int i) {
  if constexpr (F32) return static_cast<const float*>(row)[i];
  else return bf16_lo(static_cast<const uint16_t*>(row)[i]);
}
template <bool F32> __device__ __forceinline__ const char* row_of(const void* base, int64_t stride, int64_t row) {
  return static_cast<const char*>(base) + row * stride * (F32 ? 4 : 2);
}

// 16 bytes of logits; those outside [0, V) are -infinity.  i: index of the first, at a multiple of 16 bytes of memory.
template <bool F32> constexpr int kVec = F32 ? 4 : 8;
template <bool F32>
__device__ __forceinline__ void load_logits(const char* row, int i, int V, float (&x)[kVec<F32>]) {
  constexpr int E = kVec<F32>;
  if (i >= 0 && i + E <= V) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(row + (int64_t)i * (F32 ? 4 : 2));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (F32) x[k] = __uint_as_float(w[k]);
      else { x[2 * k] = bf16_lo(w[k]); x[2 * k + 1] = bf16_hi(w[k]); }
    }
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) x[k] = i + k >= 0 && i + k < V ? logit<F32>(row, i + k) : -INFINITY;
  }
}
// logits between a row's beginning and the multiple of 16 bytes of memory in front of it
template <bool F32> __device__ __forceinline__ int misaligned(const char* row) { return (int)(reinterpret_cast<uintptr_t>(row) & 15u) / (F32 ? 4 : 2); }

__device__ __forceinline__ float row_factor(const VerifyDev& p, int b) {  // of a logit in front of exp2
  const float t = p.temperature ? p.temperature[b] : 1.f;
  return t > 0.f ? (float)(kLog2e64 / (double)t) : (float)kLog2e64;
}

// exp2 of t <= 0 in fp64: 2^n times the Taylor series of exp(f ln 2), |f| <= 1/2, whose first term left out is 2e-16
__device__ __forceinline__ double exp2_64(double t) {
  if (!(t > -1000.0)) return t != t ? t : 0.0;
  const double n = rint(t), y = (t - n) * 0.69314718055994530942;
  double s = 1.0 / 479001600.0;
  s = fma(s, y, 1.0 / 39916800.0);
  s = fma(s, y, 1.0 / 3628800.0);
  s = fma(s, y, 1.0 / 362880.0);
  s = fma(s, y, 1.0 / 40320.0);
  s = fma(s, y, 1.0 / 5040.0);
  s = fma(s, y, 1.0 / 720.0);
  s = fma(s, y, 1.0 / 120.0);
  s = fma(s, y, 1.0 / 24.0);
  s = fma(s, y, 1.0 / 6.0);
  s = fma(s, y, 0.5);
  s = fma(s, y, 1.0);
  s = fma(s, y, 1.0);
  return __longlong_as_double(__double_as_longlong(s) + ((long long)n << 52));
}
__device__ __forceinline__ double weight64(float z, float top, double inv_t) { return exp2_64(((double)z - (double)top) * inv_t * kLog2e64); }

// the workgroup's 256 numbers added, in an order that does not change; all threads get the sum
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, kWave);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

}  // namespace

template <bool F32>
__global__ __launch_bounds__(256) void verify_stats_kernel(const VerifyDev p) {
  constexpr int E = kVec<F32>, N = kSlice / (256 * E);
  __shared__ float tops[4], sums[4];
  __shared__ int args[4];
  const int slice = (int)(blockIdx.x % (uint32_t)p.slices), row = (int)(blockIdx.x / (uint32_t)p.slices);
  const bool target = row < p.T + p.B;
  const int r = target ? row : row - (p.T + p.B);
  const int used = p.cu[p.B];
  if (r >= (target ? used + p.B : used)) return;  // (a row of nobody)
  float c = (float)kLog2e64;
  bool greedy = false;
  if (p.temperature) {
    int lo = 0, hi = p.B;  // the sequence: the last b with cu[b] (+ b) <= r
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.cu[mid] + (target ? mid : 0) <= r) lo = mid; else hi = mid;
    }
    c = row_factor(p, lo);
    greedy = p.temperature[lo] == 0.f;
  }
  const char* at = target ? row_of<F32>(p.target, p.target_stride, r) : row_of<F32>(p.draft, p.draft_stride, r);
  const int first = slice * kSlice - misaligned<F32>(at);
  float x[N][E];
#pragma unroll
  for (int k = 0; k < N; ++k) load_logits<F32>(at, first + (k * 256 + (int)threadIdx.x) * E, p.V, x[k]);
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) top = fmaxf(top, x[k][e]);
  top = wave_max(top);
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) tops[w] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) sum += exp2f((x[k][e] - base) * c);
  sum = wave_sum(sum);
  int arg = 0x7fffffff;
  if (greedy) {
#pragma unroll
    for (int k = N - 1; k >= 0; --k)
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (x[k][e] == top) arg = first + (k * 256 + (int)threadIdx.x) * E + e;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) arg = min(arg, __shfl_xor(arg, off, kWave));
  }
  if ((threadIdx.x & 63) == 0) { sums[w] = sum; args[w] = arg; }
  __syncthreads();
  if (threadIdx.x == 0) {
    RowStats s;
    s.top = top;
    s.sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    s.arg = min(min(args[0], args[1]), min(args[2], args[3]));
    s.pad = 0;
    p.stats[(int64_t)row * p.slices + slice] = s;
  }
}

template <bool F32>
__global__ __launch_bounds__(256) void verify_choose_kernel(const VerifyDev p) {
  constexpr int kRows = 2 * SP_VERIFY_MAX_DRAFTED + 1;
  __shared__ float tops[kRows];
  __shared__ double sums[kRows], lds[4];
  __shared__ int args[kRows];
  __shared__ int shared_a, shared_bad;
  const int part = (int)(blockIdx.x % (uint32_t)p.parts), b = (int)(blockIdx.x / (uint32_t)p.parts), tid = threadIdx.x;
  const int t0 = p.cu[b], n = p.cu[b + 1] - t0;
  const float t = p.temperature ? p.temperature[b] : 1.f;
  const bool valid = t0 >= 0 && n >= 0 && n <= SP_VERIFY_MAX_DRAFTED && (int64_t)t0 + n <= p.T && t >= 0.f && t < INFINITY;
  const float c = row_factor(p, b);
  if (valid) {
    const int rows = n + 1 + (p.draft ? n : 0);
    for (int i = tid; i < rows; i += 256) {
      const RowStats* s = p.stats + (i <= n ? (int64_t)t0 + b + i : (int64_t)p.T + p.B + t0 + (i - n - 1)) * p.slices;
      float top = -INFINITY;
      for (int k = 0; k < p.slices; ++k) top = fmaxf(top, s[k].top);
      const float base = top == -INFINITY ? 0.f : top;
      double sum = 0.0;
      int arg = 0x7fffffff;
      for (int k = 0; k < p.slices; ++k) {
        sum += (double)(s[k].sum * exp2f((s[k].top - base) * c));
        if (s[k].top == top) arg = min(arg, s[k].arg);
      }
      tops[i] = top;
      sums[i] = sum;
      args[i] = arg;
    }
  }
  __syncthreads();
  const auto sound = [&](int i) { return sums[i] > 0.0 && sums[i] < (double)INFINITY; };
  if (tid < 64) {
    bool stands = false, bad = false;
    double lp = 0.0;
    if (valid && tid < n) {
      const int x = p.tokens[t0 + tid];
      bad = x < 0 || x >= p.V || !sound(tid) || (p.draft && !sound(n + 1 + tid));
      if (!bad) {
        double px, qx = 1.0;
        if (t > 0.f) {
          const double z = ((double)logit<F32>(row_of<F32>(p.target, p.target_stride, (int64_t)t0 + b + tid), x) - (double)tops[tid]) / (double)t;
          px = exp2_64(z * kLog2e64) / sums[tid];
          lp = z - log(sums[tid]);
          if (p.draft)
            qx = weight64(logit<F32>(row_of<F32>(p.draft, p.draft_stride, t0 + tid), x), tops[n + 1 + tid], 1.0 / (double)t) / sums[n + 1 + tid];
        } else {
          px = args[tid] == x ? 1.0 : 0.0;
          if (p.draft) qx = args[n + 1 + tid] == x ? 1.0 : 0.0;
        }
        stands = (double)p.u[t0 + tid] * qx < px;
      }
    }
    const uint64_t falls = __builtin_amdgcn_ballot_w64(tid < n && !stands), bads = __builtin_amdgcn_ballot_w64(bad);
    const int a = falls ? __builtin_ctzll(falls) : n;
    const bool wrong = !valid || (a < n && (bads >> a & 1)) || (a == n && !sound(n));
    if (tid == 0) { shared_a = a; shared_bad = wrong; }
    if (part == 0) {
      const int64_t first = (int64_t)t0 + b;
      const int rows = t0 >= 0 && n >= 0 && (int64_t)t0 + n <= p.T ? n + 1 : 0;
      for (int j = tid; j < rows; j += 64) {
        if (wrong) {
          p.out_tokens[first + j] = -1;
          if (p.logprob) p.logprob[first + j] = __uint_as_float(0x7fc00000u);
        } else if (j < a) {
          p.out_tokens[first + j] = p.tokens[t0 + j];
          if (p.logprob) p.logprob[first + j] = (float)lp;
        } else if (j > a) {
          p.out_tokens[first + j] = -1;
          if (p.logprob) p.logprob[first + j] = -INFINITY;
        } else if (t == 0.f) {
          p.out_tokens[first + j] = args[a];  // (where x_a does not stand, all of p is at another token, and q cannot have more there)
          if (p.logprob) p.logprob[first + j] = 0.f;
        }
      }
      if (tid == 0) {
        p.n_accepted[b] = wrong ? -1 : a;
        if (p.kept_len) p.kept_len[b] = p.past_len[b] + (wrong ? 0 : 1 + a);
        VerifyState s;
        s.inv_t = t > 0.f ? 1.0 / (double)t : 0.0;
        s.sample = !wrong && t > 0.f;
        s.row_p = s.sample ? t0 + b + a : 0;
        s.row_q = s.sample && a < n && p.draft ? t0 + a : -1;
        s.token = s.sample && a < n && !p.draft ? p.tokens[t0 + a] : -1;
        s.top_p = s.sample ? tops[a] : 0.f;
        s.top_q = s.row_q >= 0 ? tops[n + 1 + a] : 0.f;
        p.states[b] = s;
      }
    }
  }
  __syncthreads();
  const int a = shared_a;
  if (shared_bad || t == 0.f) return;
  const bool with_q = a < n && p.draft;
  const char* row_p = row_of<F32>(p.target, p.target_stride, (int64_t)t0 + b + a);
  const char* row_q = with_q ? row_of<F32>(p.draft, p.draft_stride, (int64_t)t0 + a) : nullptr;
  const double inv_t = 1.0 / (double)t;
  const float top_p = tops[a], top_q = with_q ? tops[n + 1 + a] : 0.f;
  double zp = 0.0, zq = 0.0;
  for (int k = 0; k < kMine; ++k) {
    const int i = part * kPart + k * 256 + tid;
    if (i >= p.V) break;
    zp += weight64(logit<F32>(row_p, i), top_p, inv_t);
    if (with_q) zq += weight64(logit<F32>(row_q, i), top_q, inv_t);
  }
  zp = block_sum(zp, lds);
  zq = block_sum(zq, lds);
  if (tid == 0) {
    p.sum_p[(int64_t)b * p.parts + part] = zp;
    p.sum_q[(int64_t)b * p.parts + part] = zq;
  }
}

// sums over a sequence's parts, by 256 threads
__device__ __forceinline__ double parts_sum(const double* parts, int n, double* lds) {
  double v = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) v += parts[i];
  return block_sum(v, lds);
}

// what is left of p_i over the draft: max(p_i - q_i, 0), p and q normalised
template <bool F32>
__device__ __forceinline__ double residual_weight(const VerifyDev& p, const VerifyState& s, const char* row_p, const char* row_q, int i, double inv_p, double inv_q) {
  const double w = weight64(logit<F32>(row_p, i), s.top_p, s.inv_t) * inv_p;
  if (i == s.token) return 0.0;
  if (!row_q) return w;
  const double left = w - weight64(logit<F32>(row_q, i), s.top_q, s.inv_t) * inv_q;
  return left > 0.0 ? left : 0.0;
}

template <bool F32>
__global__ __launch_bounds__(256) void verify_residual_kernel(const VerifyDev p) {
  __shared__ double lds[4];
  const int part = (int)(blockIdx.x % (uint32_t)p.parts), b = (int)(blockIdx.x / (uint32_t)p.parts);
  const VerifyState s = p.states[b];
  if (!s.sample) return;
  const char* row_p = row_of<F32>(p.target, p.target_stride, s.row_p);
  const char* row_q = s.row_q >= 0 ? row_of<F32>(p.draft, p.draft_stride, s.row_q) : nullptr;
  const double inv_p = 1.0 / parts_sum(p.sum_p + (int64_t)b * p.parts, p.parts, lds);
  const double inv_q = row_q ? 1.0 / parts_sum(p.sum_q + (int64_t)b * p.parts, p.parts, lds) : 0.0;
  double sum = 0.0;
  for (int k = 0; k < kMine; ++k) {
    const int i = part * kPart + k * 256 + (int)threadIdx.x;
    if (i >= p.V) break;
    sum += residual_weight<F32>(p, s, row_p, row_q, i, inv_p, inv_q);
  }
  sum = block_sum(sum, lds);
  if (threadIdx.x == 0) p.sum_w[(int64_t)b * p.parts + part] = sum;
}

template <bool F32>
__global__ __launch_bounds__(256) void verify_pick_kernel(const VerifyDev p) {
  __shared__ double lds[4], run[256];
  __shared__ int found, last, picked;
  __shared__ double before;
  const int b = blockIdx.x, tid = threadIdx.x;
  VerifyState s = p.states[b];
  if (!s.sample) return;
  const char* row_p = row_of<F32>(p.target, p.target_stride, s.row_p);
  const char* row_q = s.row_q >= 0 ? row_of<F32>(p.draft, p.draft_stride, s.row_q) : nullptr;
  const double sum_p = parts_sum(p.sum_p + (int64_t)b * p.parts, p.parts, lds);
  const double inv_p = 1.0 / sum_p;
  double inv_q = row_q ? 1.0 / parts_sum(p.sum_q + (int64_t)b * p.parts, p.parts, lds) : 0.0;
  const double* parts = p.sum_w + (int64_t)b * p.parts;
  double total = parts_sum(parts, p.parts, lds), unit = 1.0;
  if (!(total > 0.0)) {  // nothing is left: p itself
    parts = p.sum_p + (int64_t)b * p.parts;
    unit = inv_p;
    total = sum_p * inv_p;
    row_q = nullptr;
    s.token = -1;
  }
  const double bound = (double)p.r[b] * total;
  // the first part whose end lies beyond the bound, else the last that has anything
  if (tid == 0) {
    double at = 0.0, start = 0.0;
    int pick = 0;
    for (int i = 0; i < p.parts; ++i) {
      const double w = parts[i] * unit;
      if (w > 0.0) {
        pick = i;
        start = at;
        if (at + w > bound) break;
      }
      at += w;
    }
    found = 0x7fffffff;
    last = -1;
    picked = pick;
    before = start;
  }
  __syncthreads();
  const int part = picked;
  const double start = before;
  // every thread has neighbours of its own
  const int first = part * kPart + tid * kMine;
  double w[kMine], mine = 0.0;
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    w[k] = first + k < p.V ? residual_weight<F32>(p, s, row_p, row_q, first + k, inv_p, inv_q) : 0.0;
    mine += w[k];
  }
  run[tid] = mine;
  __syncthreads();
  for (int off = 1; off < 256; off <<= 1) {
    const double v = tid >= off ? run[tid - off] : 0.0;
    __syncthreads();
    run[tid] += v;
    __syncthreads();
  }
  double at = start + (tid > 0 ? run[tid - 1] : 0.0);
  int hit = 0x7fffffff, end = -1;
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    at += w[k];
    if (w[k] > 0.0) {
      end = first + k;
      if (at > bound && hit == 0x7fffffff) hit = first + k;
    }
  }
  if (hit != 0x7fffffff) atomicMin(&found, hit);
  if (end >= 0) atomicMax(&last, end);
  __syncthreads();
  if (tid == 0) {
    const int y = found != 0x7fffffff ? found : max(last, 0);
    p.out_tokens[s.row_p] = y;
    if (p.logprob) p.logprob[s.row_p] = (float)(((double)logit<F32>(row_p, y) - (double)s.top_p) * s.inv_t - log(sum_p));
  }
}

namespace {

struct VerifyLayout { size_t states, sum_p, sum_q, sum_w, bytes; };

int verify_slices(const sp_verify_args* a) { return (int)(((int64_t)a->V + 7 + kSlice - 1) / kSlice); }  // (a row may begin up to 7 logits behind a multiple of 16 bytes)
int verify_parts(const sp_verify_args* a) { return (a->V + kPart - 1) / kPart; }

VerifyLayout verify_layout(const sp_verify_args* a) {
  VerifyLayout l;
  size_t at = align_up(sizeof(RowStats) * (size_t)(2 * a->T + a->B) * (size_t)verify_slices(a), 256);
  const size_t sums = align_up(8 * (size_t)a->B * (size_t)verify_parts(a), 256);
  l.states = at; at += align_up(sizeof(VerifyState) * (size_t)a->B, 256);
  l.sum_p = at; at += sums;
  l.sum_q = at; at += sums;
  l.sum_w = at; at += sums;
  l.bytes = at;
  return l;
}

sp_status check_verify_shape(const sp_verify_args* a) {
  if (!a) return SP_ENULL;
  if (a->B < 1 || a->V < 1 || a->V >= 1 << 24 || a->T < 0 || a->T + a->B >= 1 << 24) return SP_EINVAL;
  if (a->logits_dtype != SP_LOGITS_BF16 && a->logits_dtype != SP_LOGITS_F32) return SP_EINVAL;
  // threads of a launch
  if ((2 * a->T + a->B) * verify_slices(a) >= 1 << 24 || (int64_t)a->B * verify_parts(a) >= 1 << 24) return SP_EINVAL;
  return SP_OK;
}

sp_status check_verify(const sp_verify_args* a) {
  const sp_status st = check_verify_shape(a);
  if (st != SP_OK) return st;
  if (!a->d_cu_draft || !a->d_target || !a->d_r || !a->d_n_accepted || !a->d_out_tokens) return SP_ENULL;
  if (a->T > 0 && (!a->d_tokens || !a->d_u)) return SP_ENULL;
  if ((a->d_past_len != nullptr) != (a->d_kept_len != nullptr)) return SP_ENULL;
  if (a->T + a->B > 1 && a->target_stride < a->V) return SP_EINVAL;
  if (a->d_draft && a->T > 1 && a->draft_stride < a->V) return SP_EINVAL;
  const uintptr_t unit = a->logits_dtype == SP_LOGITS_F32 ? 3 : 1;
  if ((reinterpret_cast<uintptr_t>(a->d_target) & unit) || (reinterpret_cast<uintptr_t>(a->d_draft) & unit)) return SP_EALIGN;
  if (!a->d_workspace || a->workspace_bytes < verify_layout(a).bytes) return SP_EWORKSPACE;
  if (reinterpret_cast<uintptr_t>(a->d_workspace) & 255u) return SP_EALIGN;
  return SP_OK;
}

template <bool F32>
void launch_verify(const VerifyDev& p, hipStream_t stream) {
  const uint32_t rows = (uint32_t)(p.T + p.B + (p.draft ? p.T : 0));
  hipLaunchKernelGGL(verify_stats_kernel<F32>, dim3(rows * (uint32_t)p.slices), dim3(256), 0, stream, p);
  hipLaunchKernelGGL(verify_choose_kernel<F32>, dim3((uint32_t)(p.B * p.parts)), dim3(256), 0, stream, p);
  hipLaunchKernelGGL(verify_residual_kernel<F32>, dim3((uint32_t)(p.B * p.parts)), dim3(256), 0, stream, p);
  hipLaunchKernelGGL(verify_pick_kernel<F32>, dim3((uint32_t)p.B), dim3(256), 0, stream, p);
}

}  // namespace

}  // namespace sp

extern "C" size_t sp_verify_workspace_bytes(const sp_verify_args* a) {
  return sp::check_verify_shape(a) == SP_OK ? sp::verify_layout(a).bytes : 0;
}

extern "C" sp_status sp_verify(const sp_verify_args* a, void* hip_stream) {
  using namespace sp;
  const sp_status st = check_verify(a);
  if (st != SP_OK) return st;
  const VerifyLayout l = verify_layout(a);
  char* base = static_cast<char*>(a->d_workspace);
  VerifyDev p;
  p.B = a->B; p.V = a->V; p.T = (int)a->T; p.slices = verify_slices(a); p.parts = verify_parts(a);
  p.cu = a->d_cu_draft; p.tokens = a->d_tokens;
  p.target = a->d_target; p.draft = a->T > 0 ? a->d_draft : nullptr;
  p.target_stride = a->target_stride; p.draft_stride = a->draft_stride;
  p.temperature = a->d_temperature; p.u = a->d_u; p.r = a->d_r; p.past_len = a->d_past_len;
  p.n_accepted = a->d_n_accepted; p.out_tokens = a->d_out_tokens; p.logprob = a->d_logprob; p.kept_len = a->d_kept_len;
  p.stats = reinterpret_cast<RowStats*>(base);
  p.states = reinterpret_cast<VerifyState*>(base + l.states);
  p.sum_p = reinterpret_cast<double*>(base + l.sum_p);
  p.sum_q = reinterpret_cast<double*>(base + l.sum_q);
  p.sum_w = reinterpret_cast<double*>(base + l.sum_w);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (a->logits_dtype == SP_LOGITS_F32) launch_verify<true>(p, stream);
  else launch_verify<false>(p, stream);
  return launch_status();
}
