// Log probabilities of given tokens, entropy and the most probable tokens of rows
// of logits.
//
// Mathematics: with the row's maximum m, S = sum e^(x - m) and
// T = sum (x - m) e^(x - m): lse = m + ln S, entropy = ln S - T / S.
//
// One workgroup per row: a pass for the maximum, one for the sums, and one per top
// token for the largest (value, lowest token) below the one before.
#include "common.h"
#include "kernels.h"

namespace {

constexpr int THREADS = 256;

// order of (value, token): larger value first, then lower token
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token) {
  uint32_t b = __float_as_uint(x + 0.f);
  b = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return ((uint64_t)b << 32) | (0xffffffffu - token);
}

template <typename F, typename V>
__device__ __forceinline__ V block_reduce(V v, V* lds, F f) {
  for (int o = 32; o > 0; o >>= 1) v = f(v, (V)__shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  V r = lds[0];
  for (int i = 1; i < THREADS / 64; ++i) r = f(r, lds[i]);
  return r;
}

template <typename T>
__global__ void __launch_bounds__(THREADS) logprobs_kernel(LogprobArgs a) {
  __shared__ float lf[4];
  __shared__ unsigned long long lk[4];
  const int row = blockIdx.x, t = threadIdx.x;
  const T* x = (const T*)a.logits + row * a.ld;
  const auto add = [](float p, float q) { return p + q; };
  const auto big = [](float p, float q) { return fmaxf(p, q); };
  float m = -INFINITY, bad = 0.f;
  for (int i = t; i < a.vocab; i += THREADS) {
    if (i == a.exclude) continue;
    const float v = (float)x[i];
    if (v != v || v == INFINITY) bad = 1.f;
    m = fmaxf(m, v);
  }
  m = block_reduce(m, lf, big);
  bad = block_reduce(bad, lf, big);
  float S = 0.f, M = 0.f;
  for (int i = t; i < a.vocab; i += THREADS) {
    const float v = (float)x[i];
    if (i == a.exclude || v == -INFINITY) continue;
    const float d = fmaxf(v - m, -200.f), e = expf(d);
    S += e;
    M += d * e;
  }
  S = block_reduce(S, lf, add);
  M = block_reduce(M, lf, add);
  const bool none = m == -INFINITY;
  const float lnS = logf(S);
  if (t == 0) {
    if (a.entropy) a.entropy[row] = bad ? NAN : none ? 0.f : lnS - M / S;
    if (a.logprob) {
      const int tok = a.tokens[row];
      float r = 0.f;
      if (tok >= a.vocab || (tok >= 0 && bad))
        r = NAN;
      else if (tok >= 0)
        r = none || tok == a.exclude ? -INFINITY : (float)x[tok] - m - lnS;
      a.logprob[row] = r;
    }
  }
  unsigned long long last = ~0ull;
  for (int n = 0; n < a.n_top; ++n) {
    unsigned long long best = 0;
    for (int i = t; i < a.vocab; i += THREADS) {
      const float v = (float)x[i];
      if (i == a.exclude || !(v > -INFINITY)) continue;
      const unsigned long long k = key_of(v, i);
      if (k < last && k > best) best = k;
    }
    last = block_reduce(best, lk, [](unsigned long long p, unsigned long long q) { return p > q ? p : q; });
    if (t == 0) {
      const int id = bad || last == 0 ? -1 : (int)(0xffffffffu - (uint32_t)last);
      a.top_ids[(int64_t)row * a.n_top + n] = id;
      a.top_logprobs[(int64_t)row * a.n_top + n] = bad ? NAN : id < 0 ? -INFINITY : (float)x[id] - m - lnS;
    }
  }
}

}  // namespace

LogprobPlan logprobs_plan(int, int, int) { return {0}; }

hipError_t launch_token_logprobs(const LogprobArgs& a, const LogprobPlan&, hipStream_t s) {
  const dim3 g(a.rows), b(THREADS);
  if (a.dtype == LOPA_BF16) logprobs_kernel<__bf16><<<g, b, 0, s>>>(a);
  else if (a.dtype == LOPA_F16) logprobs_kernel<_Float16><<<g, b, 0, s>>>(a);
  else logprobs_kernel<float><<<g, b, 0, s>>>(a);
  return hipGetLastError();
}
