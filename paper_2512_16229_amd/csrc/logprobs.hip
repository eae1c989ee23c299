// Log probabilities of given tokens, entropy and the most probable tokens of rows
// of logits.
//
// Mathematics. With a reference m (the largest logit), S = sum 2^((x - m) log2 e) and
// T = sum (x - m) 2^(...): ln p_t = (x_t - m) - ln S, entropy = ln S - T / S; two
// pieces join as (S 2^d + S', (T + (m - m') S) 2^d + T') with d = (m - m') log2 e.
//
// What bounds it: memory, every logit read once (16-bit rows near the vector units
// too: six operations a logit, one of them an exponential at a quarter of the rate).
// A workgroup takes a segment of a row, THREADS x NV 16-byte vectors, into registers
// and makes everything of it there; a second kernel joins the segments of a row.
//
// Top tokens. The n-th largest maximum of groups of lanes is a bound that at least n
// logits of the segment reach (each wavefront's, then the largest of the four); with
// twice as many groups as n about 1.4 n logits pass it. Those go to LDS as 64-bit keys
// that order by (value, lowest token), and a key's rank is the number of larger ones.
// Rows of many equal values can pass more than CAND; they are taken one by one.
#include "common.h"
#include "kernels.h"

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int CAND = 1024;
constexpr int LISTS = 64;  // segments that a join takes at a time, the result so far among them
constexpr float LOG2E = 1.44269504f;
typedef unsigned long long u64;

// order of (value, token): larger value first, then lower token; 0: nothing
__device__ __forceinline__ u64 key_of(float x, uint32_t token) {
  uint32_t b = __float_as_uint(x + 0.f);  // -0 as 0
  b = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return ((u64)b << 32) | (0xffffffffu - token);
}
__device__ __forceinline__ int token_of(u64 k) { return (int)(0xffffffffu - (uint32_t)k); }
__device__ __forceinline__ float value_of(u64 k) {
  const uint32_t b = (uint32_t)(k >> 32);
  return __uint_as_float((b & 0x80000000u) ? b & 0x7fffffffu : ~b);
}

struct Sums {
  float m, S, T;
};
// a NaN in S stays (a row with a NaN or +inf has no distribution)
__device__ __forceinline__ Sums join(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  Sums r{m, 0.f, 0.f};
  for (const Sums& x : {a, b}) {
    if (x.m == -INFINITY) {
      r.S += x.S;
      continue;
    }
    const float d = x.m - m, f = __builtin_amdgcn_exp2f(d * LOG2E);
    r.S += x.S * f;
    r.T += (x.T + fmaxf(d, -200.f) * x.S) * f;
  }
  return r;
}
__device__ __forceinline__ Sums wave_join(Sums a) {
  for (int o = 32; o > 0; o >>= 1) {
    const Sums b{__shfl_xor(a.m, o), __shfl_xor(a.S, o), __shfl_xor(a.T, o)};
    a = join(a, b);
  }
  return a;
}

// the row's results from its sums and its sorted top keys (thread 0 and the first n threads)
template <typename T>
__device__ __forceinline__ void finish(const LogprobArgs& a, int row, Sums s, const u64* top) {
  const bool bad = s.S != s.S, none = s.m == -INFINITY;
  const float lnS = logf(s.S);
  const int t = threadIdx.x;
  if (t == 0) {
    if (a.entropy) a.entropy[row] = bad ? NAN : none ? 0.f : lnS - s.T / s.S;
    if (a.logprob) {
      const int tok = a.tokens[row];
      float r = 0.f;
      if (tok >= a.vocab || (tok >= 0 && bad))
        r = NAN;
      else if (tok >= 0)
        r = none || tok == a.exclude ? -INFINITY : (float)((const T*)a.logits)[row * a.ld + tok] - s.m - lnS;
      a.logprob[row] = r;
    }
  }
  if (t < a.n_top) {
    const u64 k = top[t];
    const int64_t at = (int64_t)row * a.n_top + t;
    a.top_ids[at] = bad || k == 0 ? -1 : token_of(k);
    a.top_logprobs[at] = bad ? NAN : k == 0 ? -INFINITY : value_of(k) - s.m - lnS;
  }
}

// Workspace: [rows][segs] Sums, then [rows][segs][n_top] keys.
template <typename T, int NV>
__global__ void __launch_bounds__(THREADS) logprobs_kernel(LogprobArgs a, int segs, int groups) {
  constexpr int VE = 16 / sizeof(T), EPT = NV * VE, SEG = THREADS * EPT;
  typedef T vec __attribute__((ext_vector_type(VE)));
  __shared__ Sums part[WAVES];
  __shared__ float bound[WAVES];
  __shared__ u64 cand[CAND];
  __shared__ u64 top[32];
  __shared__ int count;
  const int row = blockIdx.x / segs, seg = blockIdx.x % segs, t = threadIdx.x;
  const T* const x0 = (const T*)a.logits + row * a.ld;
  // vectors are aligned in memory: the row starts `off` elements into its first one
  const int off = (int)(((uintptr_t)x0 / sizeof(T)) % VE);
  const int first = seg * SEG + t * VE - off;  // token of this thread's first element

  float x[EPT];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = first + k * THREADS * VE;
    if (i >= 0 && i + VE <= a.vocab) {
      const vec v = *(const vec*)(x0 + i);
#pragma unroll
      for (int e = 0; e < VE; ++e) x[k * VE + e] = (float)v[e];
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e)
        x[k * VE + e] = i + e >= 0 && i + e < a.vocab ? (float)x0[i + e] : -INFINITY;
    }
  }
  const int ex = a.exclude + off - seg * SEG;  // the excluded token's place in the segment
  if (a.exclude >= 0 && ex >= 0 && ex < SEG) {
#pragma unroll
    for (int j = 0; j < EPT; ++j)
      if (ex == (j / VE) * THREADS * VE + t * VE + j % VE) x[j] = -INFINITY;
  }
  float mine = -INFINITY;  // the largest of this thread
#pragma unroll
  for (int j = 0; j < EPT; ++j) mine = fmaxf(mine, x[j]);
  Sums s{wave_max(mine), 0.f, 0.f};
  {
    const float m = s.m == -INFINITY ? 0.f : s.m;
#pragma unroll
    for (int j = 0; j < EPT; ++j) {
      const float d = x[j] - m, e = __builtin_amdgcn_exp2f(d * LOG2E);
      s.S += e;
      s.T += fmaxf(d, -200.f) * e;  // -inf: no part (-200 x 0)
    }
    s.S = wave_sum(s.S), s.T = wave_sum(s.T);
  }
  const int lane = t & 63, wave = t >> 6;
  if (a.n_top) {
    // the n-th largest maximum of `groups` groups of lanes
    float g = mine;
    for (int o = 32; o >= groups; o >>= 1) g = fmaxf(g, __shfl_xor(g, o));
    int above = 0;
    for (int i = 0; i < groups; ++i)
      above += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g), i)) > g;
    float b = above < a.n_top ? g : INFINITY;
    for (int o = 32; o > 0; o >>= 1) b = fminf(b, __shfl_xor(b, o));
    if (lane == 0) bound[wave] = b;
  }
  if (lane == 0) part[wave] = s;
  if (t == 0) count = 0;
  if (t < 32) top[t] = 0;
  __syncthreads();
  s = part[0];
  for (int w = 1; w < WAVES; ++w) s = join(s, part[w]);
  if (a.n_top) {
    float b = bound[0];
    for (int w = 1; w < WAVES; ++w) b = fmaxf(b, bound[w]);
    if (mine >= b && mine > -INFINITY) {
#pragma unroll
      for (int j = 0; j < EPT; ++j)
        if (x[j] >= b && x[j] > -INFINITY) {
          const int at = atomicAdd(&count, 1);
          if (at < CAND) cand[at] = key_of(x[j], first + (j / VE) * THREADS * VE + j % VE);
        }
    }
    __syncthreads();
    const int n = count;
    if (n <= CAND) {
      for (int i = t; i < n; i += THREADS) {
        const u64 k = cand[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += cand[j] > k;
        if (rank < a.n_top) top[rank] = k;
      }
    } else {
      u64 last = ~0ull;
      for (int r = 0; r < a.n_top && last; ++r) {
        u64 best = 0;
#pragma unroll
        for (int j = 0; j < EPT; ++j) {
          const u64 k = x[j] > -INFINITY ? key_of(x[j], first + (j / VE) * THREADS * VE + j % VE) : 0;
          if (k < last && k > best) best = k;
        }
        for (int o = 32; o > 0; o >>= 1) {
          const u64 k = __shfl_xor(best, o);
          best = k > best ? k : best;
        }
        __syncthreads();
        if (lane == 0) cand[wave] = best;
        __syncthreads();
        last = cand[0];
        for (int w = 1; w < WAVES; ++w) last = cand[w] > last ? cand[w] : last;
        if (t == 0) top[r] = last;
      }
    }
    __syncthreads();
  }
  if (segs == 1) {
    finish<T>(a, row, s, top);
    return;
  }
  const int64_t at = (int64_t)row * segs + seg;
  if (t == 0) ((Sums*)a.ws)[at] = s;
  u64* keys = (u64*)((char*)a.ws + (((int64_t)a.rows * segs * sizeof(Sums) + 15) & ~(int64_t)15));
  if (t < a.n_top) keys[at * a.n_top + t] = top[t];
}

// Joins a row's segments: one workgroup per row.
template <typename T>
__global__ void __launch_bounds__(THREADS) logprobs_join_kernel(LogprobArgs a, int segs) {
  __shared__ Sums part[WAVES];
  __shared__ u64 list[LISTS * 32];
  __shared__ u64 top[32];
  const int row = blockIdx.x, t = threadIdx.x, n = a.n_top;
  const Sums* const sums = (const Sums*)a.ws + (int64_t)row * segs;
  const u64* const keys = (const u64*)((const char*)a.ws +
                                       (((int64_t)a.rows * segs * sizeof(Sums) + 15) & ~(int64_t)15)) +
                          (int64_t)row * segs * n;
  Sums s{-INFINITY, 0.f, 0.f};
  for (int i = t; i < segs; i += THREADS) s = join(s, sums[i]);
  s = wave_join(s);
  if ((t & 63) == 0) part[t >> 6] = s;
  if (t < 32) top[t] = 0;
  __syncthreads();
  s = part[0];
  for (int w = 1; w < WAVES; ++w) s = join(s, part[w]);
  // sorted lists of n keys, the result so far as list 0: a key's rank is the number of
  // larger ones, by bisection in every list
  for (int base = 0; n && base < segs; base += LISTS - 1) {
    const int lists = 1 + (segs - base < LISTS - 1 ? segs - base : LISTS - 1);
    for (int i = t; i < lists * n; i += THREADS) list[i] = i < n ? top[i] : keys[(int64_t)base * n + i - n];
    __syncthreads();
    if (t < 32) top[t] = 0;
    __syncthreads();
    for (int i = t; i < lists * n; i += THREADS) {
      const u64 k = list[i];
      if (k == 0) continue;
      int rank = 0;
      for (int j = 0; j < lists && rank < n; ++j) {
        int lo = 0, hi = n;  // keys of list j above k
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (list[j * n + mid] > k) lo = mid + 1;
          else hi = mid;
        }
        rank += lo;
      }
      if (rank < n) top[rank] = k;
    }
    __syncthreads();
  }
  finish<T>(a, row, s, top);
}

int64_t segments(int64_t vocab, int nv, int elem) {
  // a row may start up to VE - 1 elements into its first vector
  const int64_t ve = 16 / elem, seg = THREADS * nv * ve;
  return (vocab + ve - 1 + seg - 1) / seg;
}

// Few segments in all: short ones (2 vectors a thread), so that more compute units share
// the rows.
int vectors(int64_t rows, int64_t vocab, int elem) { return rows * segments(vocab, 8, elem) >= 512 ? 8 : 2; }

template <typename T, int NV>
hipError_t launch(const LogprobArgs& a, int segs, hipStream_t s) {
  const int64_t n = (int64_t)a.rows * segs;
  int groups = 1;  // at least twice n where the lanes allow it
  while (groups < 64 && groups < 2 * a.n_top) groups *= 2;
  logprobs_kernel<T, NV><<<dim3((unsigned)n), dim3(THREADS), 0, s>>>(a, segs, groups);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || segs == 1) return e;
  logprobs_join_kernel<T><<<dim3(a.rows), dim3(THREADS), 0, s>>>(a, segs);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const LogprobArgs& a, hipStream_t s) {
  const int nv = vectors(a.rows, a.vocab, sizeof(T));
  const int segs = (int)segments(a.vocab, nv, sizeof(T));
  return nv == 8 ? launch<T, 8>(a, segs, s) : launch<T, 2>(a, segs, s);
}

}  // namespace

// The type is not among the sizes: the larger of the two.
LogprobPlan logprobs_plan(int rows, int vocab, int n_top) {
  LogprobPlan p{};
  for (int elem : {2, 4}) {
    const int64_t segs = segments(vocab, vectors(rows, vocab, elem), elem);
    const int64_t bytes =
        segs == 1 ? 0 : ((rows * segs * (int64_t)sizeof(Sums) + 15) & ~(int64_t)15) + rows * segs * n_top * 8;
    p.bytes = bytes > p.bytes ? bytes : p.bytes;
    p.workgroups = rows * segs > p.workgroups ? rows * segs : p.workgroups;
  }
  return p;
}

hipError_t launch_token_logprobs(const LogprobArgs& a, const LogprobPlan&, hipStream_t s) {
  if (a.dtype == LOPA_BF16) return launch_type<__bf16>(a, s);
  if (a.dtype == LOPA_F16) return launch_type<_Float16>(a, s);
  return launch_type<float>(a, s);
}
