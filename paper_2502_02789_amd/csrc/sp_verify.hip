// sp_verify: which drafted tokens stand against the target's probabilities, and the token that is sampled behind them.
//
// Three kernels, bound by reading the logits once (the first; the others read the rows of one place of each sequence again):
//   stats     maximum and sum of exp of every row, 8192 logits to a workgroup
//   choose    per sequence: the rows' sums, how many tokens stand, hence the row that a token is sampled from; in strips of it, the sums of the weights of p and
//             q, and of both over the tokens with something left: with Zp, Zq the sums over all, what is left in a strip is (sum of wp - Zp/Zq sum of wq) / Zp
//   pick      the strip in which the sum passes r times the whole, and the token in it
// 64 sequences of 1 to 8 tokens, V = 128256, bf16, with the draft's logits (149 MB): 49.5 to 50.9 us a pass; traced one by one, which counts each one's start and end, the
// kernels take 27 + 21 + 5.5.  The first kernel reads 5.5 TB/s, its vector ALUs busy for about
// 60 % of the time; the second forms 16 M weights in fp64, ALUs busy for 40 %, its workgroups all at once first waiting (row sums, logits), then computing.
// One sequence of four tokens: 13.3 us, three launches, each a chain of dependent reads.
// Which token is picked depends on sums over the whole vocabulary: a vocabulary of 128K has so many borders between tokens that sums in fp32, off by 1e-7, would pick
// another token once in some hundred calls.  The sampled row's weights are therefore formed and added in fp64; the order of all sums is fixed.  Only which
// tokens have something left is decided with the ratio Zp/Zq of the first kernel's sums in fp32, so that one pass does: a token whose p and q are within the two sums' errors
// of one another (1.4e-5 at most, V = 128256) may count as one of which nothing is left, or, with less than nothing, as one of which something is.  What such tokens come to
// is that share of the whole at most: of 0.3 left and differences of the draft's logits of 0.7, as in the cases measured, some 1e-10.
#include "sp_score_internal.h"

namespace sp {

namespace {

constexpr int kSlice = 8192;     // logits of a row that a workgroup of the first kernel takes
// ... of the others.  Their sums are kept by strips, a wave's.  (Smaller ones where there is little to do: one sequence of four tokens 13.6 us instead of 14.7, 64 of four,
// V = 1000, 15.3 instead of 16.8; but 32 of four, V = 128256, 33.9 instead of 31.7, as every workgroup looks its sequence's rows up.)
constexpr int kSmallPart = 2048, kLargePart = 4096;
constexpr int strip_of(int part) { return part / 4; }
constexpr double kLog2e64 = 1.4426950408889634074;

struct RowStats { float top, sum; int32_t arg, pad; };   // of a slice: largest logit, sum of exp((z - top) / temperature), where the largest is
struct VerifyState {                                       // of a sequence
  double c;               // of a logit in front of exp2
  double ratio;           // of the sums of the two rows' weights, in fp32's accuracy: what is left of p_i over q_i is something if its weight exceeds q_i's so many times
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
  double* sums;        // [B][4 parts strips][4]: weights of p, of q, and both over the tokens of which something is left
};

template <bool F32> __device__ __forceinline__ const char* row_of(const void* base, int64_t stride, int64_t row) {
  return static_cast<const char*>(base) + row * stride * (F32 ? 4 : 2);
}
template <bool F32> __device__ __forceinline__ float logit(const char* row, int i) {
  if constexpr (F32) return reinterpret_cast<const float*>(row)[i];
  else return bf16_lo(reinterpret_cast<const uint16_t*>(row)[i]);
}

// N times 16 bytes of logits, those of k from element first + k step on, wherever the row begins; those from V on are -infinity.  inside: none of the workgroup's are.  (All loads are on their way
// together: what would lie outside the row is read at its beginning instead, and the one vector that a row ends in comes element by element.)
template <bool F32> constexpr int kVec = F32 ? 4 : 8;
template <bool F32, int N>
__device__ __forceinline__ void load_logits(const char* row, int first, int step, int V, bool inside, float (&x)[N][kVec<F32>]) {
  constexpr int E = kVec<F32>;
  typedef u32x4 words_t __attribute__((aligned(2)));

  u32x4 w[N];
  if (inside) {  // (the same for all lanes)
#pragma unroll
    for (int k = 0; k < N; ++k) w[k] = __builtin_nontemporal_load(reinterpret_cast<const words_t*>(row + (uint32_t)(first + k * step) * (F32 ? 4 : 2)));
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (F32) {
          x[k][e] = __uint_as_float(w[k][e]);
        } else {
          x[k][2 * e] = bf16_lo(w[k][e]);
          x[k][2 * e + 1] = bf16_hi(w[k][e]);
        }
      }
    return;
  }
  if (V >= E) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int i = first + k * step;
      w[k] = __builtin_nontemporal_load(reinterpret_cast<const words_t*>(row + (uint32_t)(i + E <= V ? i : 0) * (F32 ? 4 : 2)));
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const bool whole = first + k * step + E <= V;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (F32) {
        x[k][e] = whole ? __uint_as_float(w[k][e]) : -INFINITY;
      } else {
        const uint32_t y = whole ? w[k][e] : 0xff80ff80u;
        x[k][2 * e] = bf16_lo(y);
        x[k][2 * e + 1] = bf16_hi(y);
      }
    }
  }
  if (V % E != 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int i = first + k * step;
      if (i < V && i + E > V) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (i + e < V) x[k][e] = logit<F32>(row, i + e);
      }
    }
  }
}

// of a logit in front of exp2 (finite in fp32 too)
__device__ __forceinline__ double exp2_factor(float t) { return t > 0.f ? fmin(kLog2e64 / (double)t, 3e38) : kLog2e64; }

// exp((z - top) / temperature) in fp64, c = log2(e) / temperature: 2^n times a polynomial for 2^f, |f| <= 1/2, the one that equals it at the ten Chebyshev nodes of
// that interval (2e-14 off at most; of the same degree, Taylor's would be 7e-12).  (n comes out of the low bits of the sum with 1.5 2^52.)  Below 2^-1021, where the exponent's
// field ends, it is 0: a strip in which all is masked must weigh exactly nothing, or r = 0 would pick it.
struct Exp64 {
  static constexpr int N = 10;
  double k[N] = {1.0205905413765595e-07, 1.325964524488711e-06, 1.5252672924850737e-05, 0.0001540343375125101, 0.0013333558200794592, 0.009618129193934313,
                 0.05550410866465167, 0.2402265069564034, 0.6931471805599462, 1.0000000000000135};
  __device__ __forceinline__ Exp64() {  // (kept in scalar registers: as literals, each would be moved into a vector register in front of its use)
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+s"(k[i]));
  }
  __device__ __forceinline__ double operator()(float z, double top, double c) const {
    const double t = ((double)z - top) * c, shifted = t + 6755399441055744.0, f = t - (shifted - 6755399441055744.0);
    double s = k[0];
#pragma unroll
    for (int i = 1; i < N; ++i) s = fma(s, f, k[i]);
    const uint64_t bits = (uint64_t)__double_as_longlong(s);
    const double y = __longlong_as_double((long long)((bits & 0xffffffffull) | (uint64_t)((uint32_t)(bits >> 32) + ((uint32_t)__double_as_longlong(shifted) << 20)) << 32));
    return t >= -1021.0 ? y : 0.0;
  }
};

// the wave's numbers added, in an order that does not change; lane 63 gets the sum
template <int CTRL, int ROWS> __device__ __forceinline__ double moved(double v) {  // (0 where a lane gets none)
  const uint64_t x = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xf, false);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
// ... every lane the sum of those up to its own
__device__ __forceinline__ double wave_prefix(double v) {
  v += moved<0x111, 0xf>(v);   // from the lane 1, 2, 4, 8 below, in rows of 16
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);   // a row's last lane into the next row, into the upper half
  v += moved<0x143, 0xc>(v);
  return v;
}

// N numbers added over the workgroup's 256 threads, in an order that does not change; all threads get the sums
template <int N>
__device__ __forceinline__ void block_sums(double (&v)[N], double (*lds)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_prefix(v[i]);
  if ((threadIdx.x & 63) == 63)
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
  load_logits<F32, N>(at, slice * kSlice + (int)threadIdx.x * E, 256 * E, p.V, (slice + 1) * kSlice <= p.V, x);
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
  // every thread's own maximum and sum, then the wave's, then the workgroup's
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) top = fmaxf(top, x[k][e]);
  const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) sum += __builtin_amdgcn_exp2f((x[k][e] - base) * c);
  const float wave_top = wave_max(top), wave_base = wave_top == -INFINITY ? 0.f : wave_top;
  sum = wave_sum(sum * __builtin_amdgcn_exp2f((top - wave_base) * c));
  int arg = 0x7fffffff;
  if (greedy) {
#pragma unroll
    for (int k = N - 1; k >= 0; --k)
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (x[k][e] == wave_top) arg = slice * kSlice + (k * 256 + (int)threadIdx.x) * E + e;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) arg = min(arg, __shfl_xor(arg, off, kWave));
  }
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) { tops[w] = wave_top; sums[w] = sum; args[w] = arg; }
  __syncthreads();
  if (threadIdx.x == 0) {
    RowStats s;
    s.top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float all = s.top == -INFINITY ? 0.f : s.top;
    s.sum = 0.f;
    s.arg = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s.sum += sums[i] * __builtin_amdgcn_exp2f((tops[i] - all) * c);
      if (tops[i] == s.top) s.arg = min(s.arg, args[i]);
    }
    s.pad = 0;
    p.stats[(int64_t)row * p.slices + slice] = s;
  }
}

template <bool F32, int PART>
__global__ __launch_bounds__(256) void verify_choose_kernel(const VerifyDev p) {
  constexpr int kRows = 2 * SP_VERIFY_MAX_DRAFTED + 1, E = kVec<F32>, kMine = PART / 256, kStrip = strip_of(PART);
  __shared__ float tops[kRows];
  __shared__ double sums[kRows];
  __shared__ int args[kRows];
  __shared__ int shared_a, shared_bad;
  const int part = (int)(blockIdx.x % (uint32_t)p.parts), b = (int)(blockIdx.x / (uint32_t)p.parts), tid = threadIdx.x;
  const int t0 = p.cu[b], n = p.cu[b + 1] - t0;
  const float t = p.temperature ? p.temperature[b] : 1.f;
  const bool valid = t0 >= 0 && n >= 0 && n <= SP_VERIFY_MAX_DRAFTED && (int64_t)t0 + n <= p.T && t >= 0.f && t < INFINITY;
  const double c = exp2_factor(t);
  const Exp64 exp64;
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
        px = exp64(zp, tops[tid], c) / sums[tid];
        if (p.draft) qx = exp64(zq, tops[n + 1 + tid], c) / sums[n + 1 + tid];
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
        } else {  // (until one is picked)
          p.out_tokens[first + j] = -1;
          if (p.logprob) p.logprob[first + j] = __uint_as_float(0x7fc00000u);
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
        s.ratio = s.row_q >= 0 ? sums[a] / sums[n + 1 + a] : 0.0;
        p.states[b] = s;
      }
    }
  }
  __syncthreads();
  const int a = shared_a;
  if (shared_bad || t == 0.f) return;
  // the row's part of the sums in fp64, and the draft's, a strip to a wave
  const bool with_q = a < n && p.draft;
  const char* row_p = row_of<F32>(p.target, p.target_stride, (int64_t)t0 + b + a);
  const char* row_q = with_q ? row_of<F32>(p.draft, p.draft_stride, (int64_t)t0 + a) : row_p;
  const double top_p = tops[a], top_q = with_q ? tops[n + 1 + a] : 0.0;
  float vp[kMine / E][E], vq[kMine / E][E];
  const int strip = part * 4 + (tid >> 6), first = strip * kStrip + (tid & 63) * E;
  load_logits<F32, kMine / E>(row_p, first, 64 * E, p.V, (part + 1) * PART <= p.V, vp);
  if (with_q) load_logits<F32, kMine / E>(row_q, first, 64 * E, p.V, (part + 1) * PART <= p.V, vq);
  double z[4] = {0.0, 0.0, 0.0, 0.0};
  if (with_q) {
    const double ratio = sums[a] / sums[n + 1 + a];
#pragma unroll
    for (int k = 0; k < kMine / E; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const double wp = exp64(vp[k][e], top_p, c), wq = exp64(vq[k][e], top_q, c);
        const bool left = wp > wq * ratio;
        z[0] += wp;
        z[1] += wq;
        z[2] += left ? wp : 0.0;
        z[3] += left ? wq : 0.0;
      }
  } else {
    const int token = a < n ? p.tokens[t0 + a] : -1;
#pragma unroll
    for (int k = 0; k < kMine / E; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const double wp = exp64(vp[k][e], top_p, c);
        z[0] += wp;
        z[2] += first + k * 64 * E + e != token ? wp : 0.0;
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) z[i] = wave_prefix(z[i]);
  if ((tid & 63) == 63) {
    double* dst = p.sums + ((int64_t)b * 4 * p.parts + strip) * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[i] = z[i];
  }
}

// what is left of p_i over the draft, in units of p's weights
struct Residual { double c, top_p, top_q, first_ratio, ratio; int token; bool with_q; };
__device__ __forceinline__ double residual_weight(const Exp64& exp64, const Residual& s, float zp, float zq, int i) {
  double w = exp64(zp, s.top_p, s.c);
  if (s.with_q) {
    const double wq = exp64(zq, s.top_q, s.c);
    w = w > wq * s.first_ratio ? fmax(w - wq * s.ratio, 0.0) : 0.0;
  }
  return i == s.token ? 0.0 : w;
}

// exclusive sums over the workgroup's 256 threads
__device__ __forceinline__ double block_before(double v, double* lds) {
  const int w = threadIdx.x >> 6;
  const double x = wave_prefix(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) lds[w] = x;
  __syncthreads();
  double before = 0.0;
  for (int i = 0; i < w; ++i) before += lds[i];
  return before + (x - v);
}

// The first of the workgroup's threads' hits (ascending with the threads; kNone: none), or, where no thread has one, the last of their ends (-1: none).  (LDS
// atomics by all lanes on one word are done lane after lane: 4 us each here.)
constexpr int kNone = 0x7fffffff;
__device__ __forceinline__ int first_hit(int hit, int end, int (*lds)[2]) {
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint64_t hits = __builtin_amdgcn_ballot_w64(hit != kNone), ends = __builtin_amdgcn_ballot_w64(end >= 0);
  if (hits ? l == __builtin_ctzll(hits) : l == 0) lds[w][0] = hit;
  if (ends ? l == 63 - __builtin_clzll(ends) : l == 0) lds[w][1] = end;
  __syncthreads();
  int found = kNone, last = -1;
#pragma unroll
  for (int i = 3; i >= 0; --i)
    if (lds[i][0] != kNone) found = lds[i][0];
#pragma unroll
  for (int i = 0; i < 4; ++i) last = max(last, lds[i][1]);
  return found != kNone ? found : last;
}

template <bool F32, int PART>
__global__ __launch_bounds__(256) void verify_pick_kernel(const VerifyDev p) {
  constexpr int kStrip = strip_of(PART), M = kStrip / 256;
  __shared__ double lds[4][4], run[4], start, log_sum;
  __shared__ int strip_hits[4][2], hits[4][2];
  const int b = blockIdx.x, tid = threadIdx.x;
  // every thread has neighbours of its own among the strips, one in a vocabulary of up to 2^18: their sums stay in registers
  const int strips = 4 * p.parts, per = (strips + 255) / 256, i0 = min(strips, tid * per), i1 = min(strips, i0 + per);
  const double* sums = p.sums + (int64_t)b * strips * 4;
  double own[4] = {0.0, 0.0, 0.0, 0.0}, z[4];
  if (i0 < i1)
#pragma unroll
    for (int k = 0; k < 4; ++k) own[k] = sums[4 * i0 + k];
#pragma unroll
  for (int k = 0; k < 4; ++k) z[k] = own[k];
  const float r = p.r[b];
  const VerifyState s = p.states[b];
  if (!s.sample) return;
  for (int i = i0 + 1; i < i1; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) z[k] += sums[4 * i + k];
  const Exp64 exp64;
  const bool with_q = s.row_q >= 0;
  const char* row_p = row_of<F32>(p.target, p.target_stride, s.row_p);
  const char* row_q = row_of<F32>(p.draft, p.draft_stride, s.row_q);
  block_sums(z, lds);
  Residual res = {s.c, s.top_p, s.top_q, s.ratio, with_q ? z[0] / z[1] : 0.0, s.token, with_q};
  double total = z[2] - z[3] * res.ratio;
  const bool nothing = !(total > 1e-12 * z[0]);
  if (nothing) {  // p itself
    total = z[0];
    res.with_q = false;
    res.token = -1;
  }
  const double bound = (double)r * total;
  // the first strip whose end lies beyond the bound, else the last that has anything
  const auto weight_of = [&](int i) {
    double x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = i == i0 ? own[k] : sums[4 * i + k];
    return nothing ? x[0] : fmax(x[2] - x[3] * res.ratio, 0.0);
  };
  double sum = 0.0;
  for (int i = i0; i < i1; ++i) sum += weight_of(i);
  const double before = block_before(sum, run);
  double at = before;
  int hit = kNone, end = -1;
  for (int i = i0; i < i1; ++i) {
    const double w = weight_of(i);
    if (w > 0.0) {
      end = i;
      if (at + w > bound && hit == kNone) hit = i;
    }
    at += w;
  }
  const int strip = max(first_hit(hit, end, strip_hits), 0);
  if (strip >= i0 && strip < i1) {  // (the thread that has it says what lies before it)
    at = before;
    for (int i = i0; i < strip; ++i) at += weight_of(i);
    start = at;
  }
  const int first = strip * kStrip + tid * M;
  float zp[M], zq[M];
#pragma unroll
  for (int k = 0; k < M; ++k) {
    const int i = first + k < p.V ? first + k : 0;
    zp[k] = logit<F32>(row_p, i);
    zq[k] = res.with_q ? logit<F32>(row_q, i) : 0.f;
  }
  if (tid == 255 && p.logprob) log_sum = log(z[0]);
  double w[M], mine = 0.0;
#pragma unroll
  for (int k = 0; k < M; ++k) {
    w[k] = first + k < p.V ? residual_weight(exp64, res, zp[k], zq[k], first + k) : 0.0;
    mine += w[k];
  }
  at = block_before(mine, run);
  at += start;
  hit = kNone;
  end = -1;
#pragma unroll
  for (int k = 0; k < M; ++k) {
    at += w[k];
    if (w[k] > 0.0) {
      end = first + k;
      if (at > bound && hit == kNone) hit = first + k;
    }
  }
  int y = first_hit(hit, end, hits);
  if (y < 0) {  // (what was left in the strip is no more than a rounding: its first token with a probability, and there is one, as the strip has a weight)
    hit = kNone;
#pragma unroll
    for (int k = M - 1; k >= 0; --k)
      if (first + k < p.V && first + k != res.token && exp64(zp[k], s.top_p, s.c) > 0.0) hit = first + k;
    y = first_hit(hit, -1, strip_hits);
  }
#pragma unroll
  for (int k = 0; k < M; ++k)
    if (first + k == y) {  // (one thread's)
      p.out_tokens[s.row_p] = y;
      if (p.logprob) p.logprob[s.row_p] = (float)(((double)zp[k] - (double)s.top_p) * s.c * 0.69314718055994530942 - log_sum);
    }
}

namespace {

struct VerifyLayout { size_t states, sums, bytes; };

int verify_slices(const sp_verify_args* a) { return (a->V + kSlice - 1) / kSlice; }
int verify_part(const sp_verify_args* a) {
  const int64_t large = (int64_t)a->B * ((a->V + kLargePart - 1) / kLargePart);
  return large <= 512 ? kSmallPart : kLargePart;
}
int verify_parts(const sp_verify_args* a) { return (a->V + verify_part(a) - 1) / verify_part(a); }

VerifyLayout verify_layout(const sp_verify_args* a) {
  VerifyLayout l;
  size_t at = align_up(sizeof(RowStats) * (size_t)(2 * a->T + a->B) * (size_t)verify_slices(a), 256);
  l.states = at; at += align_up(sizeof(VerifyState) * (size_t)a->B, 256);
  l.sums = at; at += align_up(4 * 32 * (size_t)a->B * (size_t)verify_parts(a), 256);
  l.bytes = at;
  return l;
}

sp_status check_verify_shape(const sp_verify_args* a) {
  if (!a) return SP_ENULL;
  if (a->B < 1 || a->V < 1 || a->V >= 1 << 24 || a->T < 0 || a->T + a->B >= 1 << 24) return SP_EINVAL;
  if (a->logits_dtype != SP_LOGITS_BF16 && a->logits_dtype != SP_LOGITS_F32) return SP_EINVAL;
  // workgroups of a launch (as many parts of the smaller size are far below)
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

template <bool F32, int PART>
void launch_verify(const VerifyDev& p, hipStream_t stream) {
  const uint32_t rows = (uint32_t)(p.T + p.B + (p.draft ? p.T : 0));
  hipLaunchKernelGGL((verify_stats_kernel<F32>), dim3(rows * (uint32_t)p.slices), dim3(256), 0, stream, p);
  hipLaunchKernelGGL((verify_choose_kernel<F32, PART>), dim3((uint32_t)(p.B * p.parts)), dim3(256), 0, stream, p);
  hipLaunchKernelGGL((verify_pick_kernel<F32, PART>), dim3((uint32_t)p.B), dim3(256), 0, stream, p);
}
template <bool F32>
void launch_verify(const VerifyDev& p, int part, hipStream_t stream) {
  if (part == kSmallPart) launch_verify<F32, kSmallPart>(p, stream);
  else launch_verify<F32, kLargePart>(p, stream);
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
  p.sums = reinterpret_cast<double*>(base + l.sums);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (a->logits_dtype == SP_LOGITS_F32) launch_verify<true>(p, verify_part(a), stream);
  else launch_verify<false>(p, verify_part(a), stream);
  return launch_status();
}
