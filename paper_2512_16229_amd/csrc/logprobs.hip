// Log probabilities of given tokens, entropy and the most probable tokens of rows
// of logits.
//
// Mathematics. In units of log2: with y = x log2 e and a reference r (of the largest
// logit), S = sum 2^(y - r) and T = sum (y - r) 2^(y - r): ln p_t = (y_t - r - log2 S) ln 2,
// entropy = (log2 S - T / S) ln 2; a piece moves to another reference by 2^(r - r') and
// T + (r - r') S.
//
// What bounds it: memory, every logit read once (16-bit rows near the vector units too:
// nine operations a logit counting the exponential as four).
// A workgroup streams a part of a row, segments of THREADS x NV 16-byte vectors, the
// next one's loads in flight while one is summed; every thread keeps its own r, S and T,
// so nothing is exchanged before the end. A second kernel joins the parts of a row.
// (2047 rows of 126464 bf16 logits 94 us, 5.5 TB/s; 256 rows of 152064 fp32 logits with 20
// top tokens 35 + 11 us; one row of 152064 with 5 3.7 + 7.2 us.)
//
// Top tokens. The pass only keeps the maximum of every group of 16 vectors (256 bytes,
// consecutive tokens). The n best groups by (maximum, lowest group) hold the n best
// tokens by (value, lowest token): a token of another group is behind the best token of
// each of the n. They are found among the maxima, and their logits are read again and
// ranked. (Keeping the n best of each wavefront's stream in the pass itself took 48
// instead of 30 us at 256 rows of 152064 fp32 logits, n = 20: nearly every segment
// brings some logit that passes.)
// Selection works on 64-bit keys that order by (value, lowest index). A bound that n
// values reach comes first (of the maxima: the n-th largest maximum of groups of lanes,
// the largest of the wavefronts'; of the groups' logits: the n-th group's maximum); what
// passes it goes to a buffer in LDS, a key's rank being the number of larger ones there.
// Only rows of very many equal values pass more than the buffer holds: they are taken one
// by one.
#include "common.h"
#include "kernels.h"

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int CAND = 512;    // keys of the buffer (ranking more takes longer than taking n one by one)
constexpr int STEP = 8;      // keys read at a time, the last ones padded with 0
constexpr int GROUP = 16;    // vectors of a group
constexpr int LDS_GROUPS = 4096;  // groups of a row whose maxima stay in LDS where one workgroup has the row
constexpr int PARTS = 256;   // parts of a row at most
constexpr float LOG2E = 1.44269504f, LN2 = 0.69314718f;
constexpr float HUGE_X = 1e30f;  // references past it: y overflows, and equal logits are 0 apart, others infinitely
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

// y - r for a logit x and the logit m of the reference; the reference is m log2 e as rounded
__device__ __forceinline__ float above(float x, float m) {
  return fabsf(m) < HUGE_X ? fmaf(x, LOG2E, -(m * LOG2E)) : (x - m) * LOG2E;
}
// the same between two references (the products rounded first, as references are: a fused
// one leaves its rounding error, which is large for large logits)
__device__ __forceinline__ float between(float m, float to) {
#pragma clang fp contract(off)
  return fabsf(m) < HUGE_X && fabsf(to) < HUGE_X ? m * LOG2E - to * LOG2E : (m - to) * LOG2E;
}

struct Sums {
  float m, S, T;
};
// s at the reference of the logit m >= s.m (a NaN stays: a row with a NaN or +inf has no
// distribution)
__device__ __forceinline__ Sums moved(Sums s, float m) {
  if (s.m == -INFINITY) return {m, s.S, 0.f};
  const float d = between(s.m, m), f = __builtin_amdgcn_exp2f(d);
  return {m, s.S * f, (s.T + fmaxf(d, -300.f) * s.S) * f};
}
// the workgroup's sums: every thread gets them
__device__ __forceinline__ Sums block_sums(Sums s, float* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float mw = wave_max(s.m);
  s = moved(s, mw);
  s.S = wave_sum(s.S), s.T = wave_sum(s.T);
  if (lane == 0) lds[3 * wave] = mw, lds[3 * wave + 1] = s.S, lds[3 * wave + 2] = s.T;
  __syncthreads();
  float m = lds[0];
  for (int w = 1; w < WAVES; ++w) m = fmaxf(m, lds[3 * w]);
  Sums r{m, 0.f, 0.f};
  for (int w = 0; w < WAVES; ++w) {
    const Sums x = moved({lds[3 * w], lds[3 * w + 1], lds[3 * w + 2]}, m);
    r.S += x.S, r.T += x.T;
  }
  return r;
}

// v[k] becomes the largest of its 16 lanes of a DPP row, in all of them
template <int CTRL, int K>
__device__ __forceinline__ void row_max_step(float (&v)[K]) {
#pragma unroll
  for (int k = 0; k < K; ++k)
    v[k] = fmaxf(v[k], __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v[k]), CTRL, 0xf, 0xf, true)));
}
template <int K>
__device__ __forceinline__ void row_max(float (&v)[K]) {
  row_max_step<0x128>(v);  // rotations by 8, 4, 2, 1
  row_max_step<0x124>(v);
  row_max_step<0x122>(v);
  row_max_step<0x121>(v);
}

struct Select {
  u64 buf[CAND + STEP];
  u64 top[32];      // the result, sorted; 0: none left
  int group[32];    // the n best groups
  u64 best[WAVES];
  float bound[64];
  int count;
};

// A bound that at least n of get(i), i < cnt, reach (or -inf): the n-th largest maximum of `lanes`
// groups of lanes over the workgroup, lanes / WAVES of each wavefront; every wavefront ranks them all.
template <typename G>
__device__ __forceinline__ float nth_bound(Select& sel, int n, int lanes, int cnt, G get) {
  const int t = threadIdx.x, lane = t & 63, own = lanes / WAVES;
  float g = -INFINITY;
  for (int i = t; i < cnt; i += 4 * THREADS) {
    float x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = i + k * THREADS < cnt ? get(i + k * THREADS) : -INFINITY;
#pragma unroll
    for (int k = 0; k < 4; ++k) g = fmaxf(g, x[k]);
  }
  for (int o = 32; o >= own; o >>= 1) g = fmaxf(g, __shfl_xor(g, o));
  if (lane < own) sel.bound[(t >> 6) * own + lane] = g;
  __syncthreads();
  g = lane < lanes ? sel.bound[lane] : -INFINITY;
  int higher = 0;
  for (int i = 0; i < lanes; i += 4)  // a multiple of 4
#pragma unroll
    for (int k = 0; k < 4; ++k)
      higher += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g), i + k)) > g;
  return -wave_max(lane < lanes && higher < n ? -g : -INFINITY);
}

// The n best of get(i), i < cnt (-inf: none), at keys of index(i), to sel.top, by the whole
// workgroup. At least n of them, or all, reach `bound`.
template <typename G, typename I>
__device__ __forceinline__ void select_best(Select& sel, int n, int cnt, float bound, G get, I index) {
  const int t = threadIdx.x;
  if (t == 0) sel.count = 0;
  __syncthreads();  // top may have been read until here
  if (t < 32) sel.top[t] = 0;
  constexpr int K = 8;  // reads in flight
  for (int base = t; base < cnt; base += K * THREADS) {
    float x[K];
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = base + k * THREADS < cnt ? get(base + k * THREADS) : -INFINITY;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (x[k] >= bound && x[k] > -INFINITY) {
        const int at = atomicAdd(&sel.count, 1);
        if (at < CAND) sel.buf[at] = key_of(x[k], index(base + k * THREADS));
      }
  }
  __syncthreads();
  const int c = sel.count;
  if (c <= CAND) {
    if (t < STEP) sel.buf[c + t] = 0;
    __syncthreads();
    for (int i = t; i < c; i += THREADS) {
      const u64 k = sel.buf[i];
      int rank = 0;
      for (int j = 0; j < c; j += STEP) {
        u64 o[STEP];
#pragma unroll
        for (int u = 0; u < STEP; ++u) o[u] = sel.buf[j + u];
#pragma unroll
        for (int u = 0; u < STEP; ++u) rank += o[u] > k;
      }
      if (rank < n) sel.top[rank] = k;
    }
  } else {
    u64 last = ~0ull;
    for (int r = 0; r < n && last; ++r) {
      u64 best = 0;
      for (int i = t; i < cnt; i += THREADS) {
        const float x = get(i);
        const u64 k = x > -INFINITY ? key_of(x, index(i)) : 0;
        if (k < last && k > best) best = k;
      }
      for (int o = 32; o > 0; o >>= 1) {
        const u64 k = __shfl_xor(best, o);
        best = k > best ? k : best;
      }
      if ((t & 63) == 0) sel.best[t >> 6] = best;
      __syncthreads();
      last = sel.best[0];
      for (int w = 1; w < WAVES; ++w) last = sel.best[w] > last ? sel.best[w] : last;
      if (t == 0) sel.top[r] = last;
      __syncthreads();
    }
  }
  __syncthreads();
}

// The row's results from its sums and its groups' maxima (LDS or workspace), by the whole
// workgroup. `lanes`: groups of lanes for the bound of the maxima.
template <typename T>
__device__ __forceinline__ void finish(const LogprobArgs& a, int row, Sums s, const float* maxima, int lanes,
                                       Select& sel) {
  constexpr int VE = 16 / sizeof(T), GT = GROUP * VE;  // tokens of a group
  const int t = threadIdx.x, n = a.n_top;
  const T* const x0 = (const T*)a.logits + row * a.ld;
  const bool bad = s.S != s.S, none = s.m == -INFINITY;
  const float l2 = log2f(s.S);
  const auto logprob = [&](float x) {
    return fabsf(x) < HUGE_X && fabsf(s.m) < HUGE_X ? (above(x, s.m) - l2) * LN2 : x - s.m - l2 * LN2;
  };
  if (t == 0) {
    if (a.entropy) a.entropy[row] = bad ? NAN : none ? 0.f : (l2 - s.T / s.S) * LN2;
    if (a.logprob) {
      const int tok = a.tokens[row];
      float r = 0.f;
      if (tok >= a.vocab || (tok >= 0 && bad))
        r = NAN;
      else if (tok >= 0)
        r = none || tok == a.exclude ? -INFINITY : logprob((float)x0[tok]);
      a.logprob[row] = r;
    }
  }
  if (n == 0) return;
  const int off = (int)(((uintptr_t)x0 / sizeof(T)) % VE);
  const int groups = (off + a.vocab + GT - 1) / GT;
  const int lane = t & 63;
  const auto maximum = [&](int i) { return maxima[i]; };
  float bound = nth_bound(sel, n, lanes, groups, maximum);
  select_best(sel, n, groups, bound, maximum, [](int i) { return i; });
  // the groups' logits
  const int have = __popcll(__ballot(lane < n && sel.top[lane]));
  const float last = have == n ? value_of(sel.top[n - 1]) : 0.f;
  if (t < n) sel.group[t] = token_of(sel.top[t]);
  __syncthreads();
  const auto token = [&](int i) { return sel.group[i / GT] * GT + i % GT - off; };
  const auto logit = [&](int i) {
    const int k = token(i);
    return (unsigned)k < (unsigned)a.vocab && k != a.exclude ? (float)x0[k] : -INFINITY;
  };
  // fewer groups than n (a small vocabulary): a bound of their logits
  bound = have == n ? last : nth_bound(sel, n, lanes, have * GT, logit);
  select_best(sel, n, have * GT, bound, logit, token);
  if (t < n) {
    const u64 k = sel.top[t];
    const int64_t at = (int64_t)row * n + t;
    a.top_ids[at] = bad || k == 0 ? -1 : token_of(k);
    a.top_logprobs[at] = bad ? NAN : k == 0 ? -INFINITY : logprob(value_of(k));
  }
}

// Workspace: [rows][parts] Sums if parts > 1, then [rows][groups] maxima.
__device__ __forceinline__ float* ws_maxima(const LogprobArgs& a, int parts, int row, int groups) {
  return (float*)a.ws + (parts > 1 ? (int64_t)a.rows * parts * 3 : 0) + (int64_t)row * groups;
}

template <typename T, int NV>
__global__ void __launch_bounds__(THREADS, 4)
logprobs_kernel(LogprobArgs a, int segs, int parts, int groups, int lanes) {
  constexpr int VE = 16 / sizeof(T), EPT = NV * VE, SEG = THREADS * EPT;
  typedef T vec __attribute__((ext_vector_type(VE)));
  __shared__ float sums[3 * WAVES];
  __shared__ Select sel;
  extern __shared__ float lds_maxima[];
  const int row = blockIdx.x / parts, part = blockIdx.x % parts, t = threadIdx.x;
  const int seg0 = (int)((int64_t)segs * part / parts), seg1 = (int)((int64_t)segs * (part + 1) / parts);
  const T* const x0 = (const T*)a.logits + row * a.ld;
  // vectors are aligned in memory: the row starts `off` elements into its first one
  const int off = (int)(((uintptr_t)x0 / sizeof(T)) % VE);
  float* const maxima = parts == 1 && groups <= LDS_GROUPS ? lds_maxima : ws_maxima(a, parts, row, groups);

  // Vectors outside the row are read as its last one and its edge vectors whole (16 aligned
  // bytes that hold a logit of the row): no branch lies between the loads and their use a
  // segment later. What is not the row's is set to -inf there.
  const vec* const v0 = (const vec*)(x0 - off);
  const int v_last = (off + a.vocab - 1) / VE;
  vec next[NV];
  const auto load = [&](int seg) {
    const int v = seg * THREADS * NV + t;
#pragma unroll
    for (int k = 0; k < NV; ++k) next[k] = v0[v + k * THREADS < v_last ? v + k * THREADS : v_last];
  };
  Sums s{-INFINITY, 0.f, 0.f};
  load(seg0);
  for (int seg = seg0; seg < seg1; ++seg) {
    const int first = seg * SEG + t * VE - off;  // token of this thread's first element
    float x[EPT];
#pragma unroll
    for (int j = 0; j < EPT; ++j) x[j] = (float)next[j / VE][j % VE];
    if (seg + 1 < seg1) load(seg + 1);
    if (seg * SEG < off || (seg + 1) * SEG > off + a.vocab) {
#pragma unroll
      for (int j = 0; j < EPT; ++j)
        if ((unsigned)(first + (j / VE) * THREADS * VE + j % VE) >= (unsigned)a.vocab) x[j] = -INFINITY;
    }
    const int ex = a.exclude + off - seg * SEG;  // the excluded token's place in the segment
    if (a.exclude >= 0 && ex >= 0 && ex < SEG) {
#pragma unroll
      for (int j = 0; j < EPT; ++j)
        if (ex == (j / VE) * THREADS * VE + t * VE + j % VE) x[j] = -INFINITY;
    }
    float vhi[NV], hi = -INFINITY, lo = INFINITY;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      vhi[k] = x[k * VE];
#pragma unroll
      for (int e = 1; e < VE; ++e) vhi[k] = fmaxf(vhi[k], x[k * VE + e]);
      hi = fmaxf(hi, vhi[k]);
    }
#pragma unroll
    for (int j = 0; j < EPT; ++j) lo = fminf(lo, x[j]);
    if (hi > s.m) s = moved(s, hi);
    {
      const float m = s.m == -INFINITY ? 0.f : s.m;
      float S = 0.f, M = 0.f;  // of the segment: short sums
      if (!__any(lo < -HUGE_X || fabsf(m) >= HUGE_X)) {
        const float r = m * LOG2E;
#pragma unroll
        for (int j = 0; j < EPT; ++j) {
          const float d = fmaf(x[j], LOG2E, -r), e = __builtin_amdgcn_exp2f(d);
          S += e;
          M = fmaf(d, e, M);
        }
      } else {
#pragma unroll
        for (int j = 0; j < EPT; ++j) {
          const float d = above(x[j], m), e = __builtin_amdgcn_exp2f(d);
          S += e;
          M = fmaf(fmaxf(d, -300.f), e, M);  // -inf: no part (-300 x 0)
        }
      }
      s.S += S, s.T += M;
    }
    if (a.n_top) {
      row_max(vhi);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int i = (seg * NV + k) * (THREADS / GROUP) + t / GROUP;
        if (t % GROUP == 0 && i < groups) maxima[i] = vhi[k];
      }
    }
  }
  s = block_sums(s, sums);
  if (parts == 1) {
    finish<T>(a, row, s, maxima, lanes, sel);
    return;
  }
  if (t == 0) ((Sums*)a.ws)[(int64_t)row * parts + part] = s;
}

// Joins a row's parts: one workgroup per row.
template <typename T>
__global__ void __launch_bounds__(THREADS) logprobs_join_kernel(LogprobArgs a, int parts, int groups, int lanes) {
  __shared__ float sums[3 * WAVES];
  __shared__ Select sel;
  const int row = blockIdx.x, t = threadIdx.x;
  Sums s{-INFINITY, 0.f, 0.f};
  if (t < parts) s = ((const Sums*)a.ws)[(int64_t)row * parts + t];
  s = block_sums(s, sums);
  finish<T>(a, row, s, ws_maxima(a, parts, row, groups), lanes, sel);
}

int64_t groups_of(int64_t vocab, int elem) {
  const int64_t ve = 16 / elem;
  return (vocab + ve - 1 + GROUP * ve - 1) / (GROUP * ve);
}

int64_t segments(int64_t vocab, int nv, int elem) {
  // a row may start up to VE - 1 elements into its first vector
  const int64_t ve = 16 / elem, seg = THREADS * nv * ve;
  return (vocab + ve - 1 + seg - 1) / seg;
}

struct Cut {
  int nv, segs, parts;
};
// How rows are cut: long segments (4 vectors a thread) unless those leave compute units
// without one, and the parts that end soonest with WGS workgroups at a time (a row's
// joining counts as one segment).
Cut cut_rows(int64_t rows, int64_t vocab, int elem) {
  constexpr int64_t WGS = 256 * 4;
  Cut c{};
  c.nv = rows * segments(vocab, 4, elem) >= 256 ? 4 : 1;
  c.segs = (int)segments(vocab, c.nv, elem);
  int64_t least = INT64_MAX;
  for (int p = 1; p <= c.segs && p <= PARTS && rows * p <= MAX_GROUPS; ++p) {
    const int64_t rounds = (rows * p + WGS - 1) / WGS, cost = rounds * ((c.segs + p - 1) / p) + (p > 1);
    if (cost < least) least = cost, c.parts = p;
    if (rounds > 1 && p >= 8) break;
  }
  return c;
}

template <typename T, int NV>
hipError_t launch(const LogprobArgs& a, const Cut& c, hipStream_t s) {
  int lanes = WAVES;  // at least twice n where there are as many
  while (lanes < 64 && lanes < 2 * a.n_top) lanes *= 2;
  const int groups = (int)groups_of(a.vocab, sizeof(T));
  const int lds = a.n_top && c.parts == 1 && groups <= LDS_GROUPS ? groups * 4 : 0;
  logprobs_kernel<T, NV><<<dim3((unsigned)a.rows * c.parts), dim3(THREADS), lds, s>>>(a, c.segs, c.parts, groups, lanes);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.parts == 1) return e;
  logprobs_join_kernel<T><<<dim3(a.rows), dim3(THREADS), 0, s>>>(a, c.parts, groups, lanes);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const LogprobArgs& a, hipStream_t s) {
  const Cut c = cut_rows(a.rows, a.vocab, sizeof(T));
  return c.nv == 4 ? launch<T, 4>(a, c, s) : launch<T, 1>(a, c, s);
}

}  // namespace

// The type is not among the sizes: the larger of the two.
int64_t logprobs_workspace(int rows, int vocab, int n_top) {
  int64_t most = 0;
  for (int elem : {2, 4}) {
    const int64_t parts = rows ? cut_rows(rows, vocab, elem).parts : 1, groups = groups_of(vocab, elem);
    const bool maxima = n_top && (parts > 1 || groups > LDS_GROUPS);
    const int64_t bytes = 4 * rows * ((parts > 1 ? 3 * parts : 0) + (maxima ? groups : 0));
    most = bytes > most ? bytes : most;
  }
  return most;
}

hipError_t launch_token_logprobs(const LogprobArgs& a, hipStream_t s) {
  if (a.dtype == LOPA_BF16) return launch_type<__bf16>(a, s);
  if (a.dtype == LOPA_F16) return launch_type<_Float16>(a, s);
  return launch_type<float>(a, s);
}
