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
  double c;               // of a logit in front of exp2
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

template <bool F32> __device__ __forceinline__ const char* row_of(const void* base, int64_t stride, int64_t row) {
  return static_cast<const char*>(base) + row * stride * (F32 ? 4 : 2);
}
template <bool F32> __device__ __forceinline__ float logit(const char* row, int i) {
  if constexpr (F32) return reinterpret_cast<const float*>(row)[i];
  else return bf16_lo(reinterpret_cast<const uint16_t*>(row)[i]);
}

// 16 bytes of logits from element i on, wherever the row begins; those from V on are -infinity
template <bool F32> constexpr int kVec = F32 ? 4 : 8;
template <bool F32>
__device__ __forceinline__ void load_logits(const char* row, int i, int V, float (&x)[kVec<F32>]) {
  constexpr int E = kVec<F32>;
  struct __attribute__((packed, aligned(F32 ? 4 : 2))) Words { u32x4 w; };
  if (i + E <= V) {
    const u32x4 w = reinterpret_cast<const Words*>(row + (int64_t)i * (F32 ? 4 : 2))->w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (F32) x[k] = __uint_as_float(w[k]);
      else { x[2 * k] = bf16_lo(w[k]); x[2 * k + 1] = bf16_hi(w[k]); }
    }
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) x[k] = i + k < V ? logit<F32>(row, i + k) : -INFINITY;
  }
}

// of a logit in front of exp2
__device__ __forceinline__ double exp2_factor(float t) { return t > 0.f ? kLog2e64 / (double)t : kLog2e64; }

// exp2 of t <= 0 in fp64: 2^n times the Taylor series of exp(f ln 2), |f| <= 1/2, whose first term left out is 7e-15
__device__ __forceinline__ double exp2_64(double t) {
  const double n = rint(fmax(t, -1000.0)), y = (fmax(t, -1000.0) - n) * 0.69314718055994530942;
  double s = 1.0 / 39916800.0;
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
  return t > -1000.0 ? ldexp(s, (int)n) : 0.0;
}
__device__ __forceinline__ double weight64(float z, float top, double c) { return exp2_64(((double)z - (double)top) * c); }

// N numbers added over the workgroup's 256 threads, in an order that does not change; all threads get the sums
template <int N>
__device__ __forceinline__ void block_sums(double (&v)[N], double (*lds)[N]) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], off, kWave);
  __syncthreads();
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) lds[threadIdx.x >> 6][i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (lds[0][i] + lds[1][i]) + (lds[2][i] + lds[3][i]);
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
  if (r >= p.cu[p.B] + (target ? p.B : 0)) return;  // (a row of nobody)
  const char* at = target ? row_of<F32>(p.target, p.target_stride, r) : row_of<F32>(p.draft, p.draft_stride, r);
  float x[N][E];
#pragma unroll
  for (int k = 0; k < N; ++k) load_logits<F32>(at, slice * kSlice + (k * 256 + (int)threadIdx.x) * E, p.V, x[k]);
  float c = (float)kLog2e64;
  bool greedy = false;
  if (p.temperature) {
    int lo = 0, hi = p.B;  // the sequence: the last b with cu[b] (+ b) <= r
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.cu[mid] + (target ? mid : 0) <= r) lo = mid; else hi = mid;
    }
    const float t = p.temperature[lo];
    c = (float)exp2_factor(t);
    greedy = t == 0.f;
  }
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
    for (int e = 0; e < E; ++e) sum += __builtin_amdgcn_exp2f((x[k][e] - base) * c);
  sum = wave_sum(sum);
  int arg = 0x7fffffff;
  if (greedy) {
#pragma unroll
    for (int k = N - 1; k >= 0; --k)
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (x[k][e] == top) arg = slice * kSlice + (k * 256 + (int)threadIdx.x) * E + e;
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
  constexpr int kRows = 2 * SP_VERIFY_MAX_DRAFTED + 1, E = kVec<F32>;
  __shared__ float tops[kRows];
  __shared__ double sums[kRows], lds[4][2];
  __shared__ int args[kRows];
  __shared__ int shared_a, shared_bad;
  const int part = (int)(blockIdx.x % (uint32_t)p.parts), b = (int)(blockIdx.x / (uint32_t)p.parts), tid = threadIdx.x;
  const int t0 = p.cu[b], n = p.cu[b + 1] - t0;
  const float t = p.temperature ? p.temperature[b] : 1.f;
  const bool valid = t0 >= 0 && n >= 0 && n <= SP_VERIFY_MAX_DRAFTED && (int64_t)t0 + n <= p.T && t >= 0.f && t < INFINITY;
  const double c = exp2_factor(t);
  // lane j of the first wave has drafted token j
  const bool mine = valid && tid < n;
  const int x = mine ? p.tokens[t0 + tid] : 0;
  const float u = mine ? p.u[t0 + tid] : 0.f;
  const bool there = x >= 0 && x < p.V;
  const float zp = mine && there ? logit<F32>(row_of<F32>(p.target, p.target_stride, (int64_t)t0 + b + tid), x) : 0.f;
  const float zq = mine && there && p.draft ? logit<F32>(row_of<F32>(p.draft, p.draft_stride, t0 + tid), x) : 0.f;
  if (valid) {  // the rows' sums, 16 lanes to a row
    const int rows = n + 1 + (p.draft ? n : 0), lane = tid & 15;
    for (int i = tid >> 4; i < rows; i += 16) {
      const RowStats* s = p.stats + (i <= n ? (int64_t)t0 + b + i : (int64_t)p.T + p.B + t0 + (i - n - 1)) * p.slices;
      float top = -INFINITY;
      double sum = 0.0;
      int arg = 0x7fffffff;
      for (int k = lane; k < p.slices; k += 16) {
        const RowStats y = s[k];
        if (y.top == top) arg = min(arg, y.arg);
        else if (y.top > top) arg = y.arg;
        const float next = fmaxf(top, y.top), base = next == -INFINITY ? 0.f : next;
        sum = sum * (double)__builtin_amdgcn_exp2f((top - base) * (float)c) + (double)(y.sum * __builtin_amdgcn_exp2f((y.top - base) * (float)c));
        top = next;
      }
#pragma unroll
      for (int off = 8; off >= 1; off >>= 1) {
        const float top2 = __shfl_xor(top, off, kWave);
        const double sum2 = __shfl_xor(sum, off, kWave);
        const int arg2 = __shfl_xor(arg, off, kWave);
        const float next = fmaxf(top, top2), base = next == -INFINITY ? 0.f : next;
        sum = sum * (double)__builtin_amdgcn_exp2f((top - base) * (float)c) + sum2 * (double)__builtin_amdgcn_exp2f((top2 - base) * (float)c);
        arg = top == top2 ? min(arg, arg2) : top > top2 ? arg : arg2;
        top = next;
      }
      if (lane == 0) { tops[i] = top; sums[i] = sum; args[i] = arg; }
    }
  }
  __syncthreads();
  const auto sound = [&](int i) { return sums[i] > 0.0 && sums[i] < (double)INFINITY; };
  if (tid < 64) {
    bool stands = false, bad = false;
    double lp = 0.0;
    if (mine) {
      bad = !there || !sound(tid) || (p.draft && !sound(n + 1 + tid));
      double px, qx = 1.0;
      if (t > 0.f) {
        px = weight64(zp, tops[tid], c) / sums[tid];
        if (p.draft) qx = weight64(zq, tops[n + 1 + tid], c) / sums[n + 1 + tid];
        if (p.logprob && part == 0) lp = ((double)zp - (double)tops[tid]) / (double)t - log(sums[tid]);
      } else {
        px = args[tid] == x ? 1.0 : 0.0;
        if (p.draft) qx = args[n + 1 + tid] == x ? 1.0 : 0.0;
      }
      stands = !bad && (double)u * qx < px;
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
          p.out_tokens[first + j] = x;
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
        s.c = c;
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
  // the row's part of the sums in fp64, and the draft's
  const bool with_q = a < n && p.draft;
  const char* row_p = row_of<F32>(p.target, p.target_stride, (int64_t)t0 + b + a);
  const char* row_q = with_q ? row_of<F32>(p.draft, p.draft_stride, (int64_t)t0 + a) : row_p;
  const float top_p = tops[a], top_q = with_q ? tops[n + 1 + a] : 0.f;
  float vp[kMine / E][E], vq[kMine / E][E];
  const int first = part * kPart;
#pragma unroll
  for (int k = 0; k < kMine / E; ++k) load_logits<F32>(row_p, first + (k * 256 + tid) * E, p.V, vp[k]);
  if (with_q) {
#pragma unroll
    for (int k = 0; k < kMine / E; ++k) load_logits<F32>(row_q, first + (k * 256 + tid) * E, p.V, vq[k]);
  }
  double z[2] = {0.0, 0.0};
#pragma unroll
  for (int k = 0; k < kMine / E; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) z[0] += weight64(vp[k][e], top_p, c);
  if (with_q) {
#pragma unroll
    for (int k = 0; k < kMine / E; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) z[1] += weight64(vq[k][e], top_q, c);
  }
  block_sums(z, lds);
  if (tid == 0) {
    p.sum_p[(int64_t)b * p.parts + part] = z[0];
    p.sum_q[(int64_t)b * p.parts + part] = z[1];
  }
}

// what is left of p_i over the draft: max(p_i - q_i, 0), p and q normalised
__device__ __forceinline__ double residual_weight(const VerifyState& s, float zp, float zq, bool with_q, int i, double inv_p, double inv_q) {
  double w = weight64(zp, s.top_p, s.c) * inv_p;
  if (with_q) w = fmax(w - weight64(zq, s.top_q, s.c) * inv_q, 0.0);
  return i == s.token ? 0.0 : w;
}

template <bool F32>
__global__ __launch_bounds__(256) void verify_residual_kernel(const VerifyDev p) {
  constexpr int E = kVec<F32>;
  __shared__ double lds[4][2], lds1[4][1];
  const int part = (int)(blockIdx.x % (uint32_t)p.parts), b = (int)(blockIdx.x / (uint32_t)p.parts), tid = threadIdx.x;
  const VerifyState s = p.states[b];
  if (!s.sample) return;
  const bool with_q = s.row_q >= 0;
  const char* row_p = row_of<F32>(p.target, p.target_stride, s.row_p);
  const char* row_q = row_of<F32>(p.draft, p.draft_stride, s.row_q);
  float vp[kMine / E][E], vq[kMine / E][E];
  const int first = part * kPart;
#pragma unroll
  for (int k = 0; k < kMine / E; ++k) load_logits<F32>(row_p, first + (k * 256 + tid) * E, p.V, vp[k]);
  if (with_q) {
#pragma unroll
    for (int k = 0; k < kMine / E; ++k) load_logits<F32>(row_q, first + (k * 256 + tid) * E, p.V, vq[k]);
  }
  double z[2] = {0.0, 0.0};
  for (int i = tid; i < p.parts; i += 256) {
    z[0] += p.sum_p[(int64_t)b * p.parts + i];
    if (with_q) z[1] += p.sum_q[(int64_t)b * p.parts + i];
  }
  block_sums(z, lds);
  const double inv_p = 1.0 / z[0], inv_q = with_q ? 1.0 / z[1] : 0.0;
  double sum[1] = {0.0};
#pragma unroll
  for (int k = 0; k < kMine / E; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) sum[0] += residual_weight(s, vp[k][e], with_q ? vq[k][e] : 0.f, with_q, first + (k * 256 + tid) * E + e, inv_p, inv_q);
  block_sums(sum, lds1);
  if (tid == 0) p.sum_w[(int64_t)b * p.parts + part] = sum[0];
}

// exclusive sums over the workgroup's 256 threads
__device__ __forceinline__ double block_before(double v, double* lds) {
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  double x = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double y = __shfl_up(x, off, kWave);
    if (l >= off) x += y;
  }
  __syncthreads();
  if (l == 63) lds[w] = x;
  __syncthreads();
  double before = 0.0;
  for (int i = 0; i < w; ++i) before += lds[i];
  return before + (x - v);
}

template <bool F32>
__global__ __launch_bounds__(256) void verify_pick_kernel(const VerifyDev p) {
  constexpr int E = kVec<F32>;
  __shared__ double lds[4][3], run[4], start;
  __shared__ int found, last, hit_part, last_part;
  const int b = blockIdx.x, tid = threadIdx.x;
  VerifyState s = p.states[b];
  if (!s.sample) return;
  if (tid == 0) { found = hit_part = 0x7fffffff; last = last_part = -1; }
  bool with_q = s.row_q >= 0;
  const char* row_p = row_of<F32>(p.target, p.target_stride, s.row_p);
  const char* row_q = row_of<F32>(p.draft, p.draft_stride, s.row_q);
  const double* sum_p = p.sum_p + (int64_t)b * p.parts;
  const double* sum_q = p.sum_q + (int64_t)b * p.parts;
  const double* parts = p.sum_w + (int64_t)b * p.parts;
  double z[3] = {0.0, 0.0, 0.0};
  for (int i = tid; i < p.parts; i += 256) {
    z[0] += sum_p[i];
    if (with_q) z[1] += sum_q[i];
    z[2] += parts[i];
  }
  block_sums(z, lds);
  const double inv_p = 1.0 / z[0], inv_q = with_q ? 1.0 / z[1] : 0.0;
  double total = z[2], unit = 1.0;
  if (!(total > 0.0)) {  // nothing is left: p itself
    parts = sum_p;
    unit = inv_p;
    total = z[0] * inv_p;
    with_q = false;
    s.token = -1;
  }
  const double bound = (double)p.r[b] * total;
  // the first part whose end lies beyond the bound, else the last that has anything; every thread has neighbours of its own
  const int per = (p.parts + 255) / 256, i0 = min(p.parts, tid * per), i1 = min(p.parts, i0 + per);
  double sum = 0.0;
  for (int i = i0; i < i1; ++i) sum += parts[i] * unit;
  const double before = block_before(sum, run);
  double at = before;
  for (int i = i0; i < i1; ++i) {
    const double w = parts[i] * unit;
    if (w > 0.0) {
      atomicMax(&last_part, i);
      if (at + w > bound) atomicMin(&hit_part, i);
    }
    at += w;
  }
  __syncthreads();
  const int part = hit_part != 0x7fffffff ? hit_part : max(last_part, 0);
  // what lies before it (the thread that has it says so)
  if (part >= i0 && part < i1) {
    at = before;
    for (int i = i0; i < part; ++i) at += parts[i] * unit;
    start = at;
  }
  __syncthreads();
  const int first = part * kPart + tid * kMine;
  double w[kMine], mine = 0.0;
#pragma unroll
  for (int k = 0; k < kMine / E; ++k) {
    float vp[E], vq[E];
    load_logits<F32>(row_p, first + k * E, p.V, vp);
    if (with_q) load_logits<F32>(row_q, first + k * E, p.V, vq);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      w[k * E + e] = residual_weight(s, vp[e], with_q ? vq[e] : 0.f, with_q, first + k * E + e, inv_p, inv_q);
      mine += w[k * E + e];
    }
  }
  at = start + block_before(mine, run);
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
    if (p.logprob) p.logprob[s.row_p] = (float)(((double)logit<F32>(row_p, y) - (double)s.top_p) * s.c * 0.69314718055994530942 - log(z[0]));
  }
}

namespace {

struct VerifyLayout { size_t states, sum_p, sum_q, sum_w, bytes; };

int verify_slices(const sp_verify_args* a) { return (a->V + kSlice - 1) / kSlice; }
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
