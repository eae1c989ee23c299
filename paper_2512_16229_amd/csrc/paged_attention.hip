// Attention of a ragged batch's rows over paged K / V.
//
// One wavefront per (row, query head) walks the row's keys with a running maximum
// and sum: m' = max(m, s), l' = l 2^(m - m') + 2^(s - m'), o likewise. A lane holds
// d / 64 dimensions; keys that the row does not see are not read.
#include "paged.h"

namespace {

template <typename T, int D>
__global__ void __launch_bounds__(64) paged_attention_kernel(PagedAttnArgs a) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x, head = blockIdx.x % a.heads, row = blockIdx.x / a.heads;
  const int s = seq_of_row(a.batch.q_start, a.batch.n_seq, row);
  if (s < 0) return;
  const int start = a.batch.q_start[s], end = a.batch.q_start[s + 1], len = a.batch.kv_len[s];
  if (start < 0 || row >= end || end > a.batch.rows || end - start > a.max_rows || len > a.max_len) return;
  const int pos = len - (end - row), ps = a.pages.page_size, Hkv = a.pages.kv_heads;
  int seen = len;
  if (a.block > 0) {
    const int64_t lim = pos < 0 ? 0 : ((int64_t)(pos / a.block) + 1) * a.block;
    if (lim < seen) seen = (int)lim;
  }
  const T* q = (const T*)a.q + row * a.ld_q + head * D;
  float qv[E], o[E] = {};
  for (int e = 0; e < E; ++e) qv[e] = (float)q[lane * E + e];
  float m = -INFINITY, l = 0.f;
  const int kvh = head / (a.heads / Hkv);
  for (int p = 0; p < seen; ++p) {
    const int page = a.batch.table[(int64_t)s * a.batch.table_ld + p / ps];
    if (page < 0 || page >= a.pages.n_pages) continue;
    const int64_t at = (((int64_t)page * Hkv + kvh) * ps + p % ps) * D + lane * E;
    float x = 0.f;
    for (int e = 0; e < E; ++e) x += qv[e] * (float)((const T*)a.pages.k)[at + e];
    x = wave_sum(x) * a.scale;
    if (a.softcap > 0.f) x = a.softcap * tanhf(x / a.softcap);
    if (x == -INFINITY) continue;
    const float m2 = fmaxf(m, x), f = expf(m - m2), w = expf(x - m2);
    l = l * f + w;
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + w * (float)((const T*)a.pages.v)[at + e];
    m = m2;
  }
  T* out = (T*)a.out + row * a.ld_out + head * D;
  for (int e = 0; e < E; ++e) out[lane * E + e] = (T)(l == 0.f ? 0.f : o[e] / l);
  if (a.lse && lane == 0) a.lse[(int64_t)row * a.heads + head] = l == 0.f ? -INFINITY : m + logf(l);
}

template <typename T, int D>
hipError_t launch(const PagedAttnArgs& a, hipStream_t s) {
  // at most 2^24 rows and 1024 heads
  const int64_t n = (int64_t)a.batch.rows * a.heads;
  if (n >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
  paged_attention_kernel<T, D><<<dim3((unsigned)n), dim3(64), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

PagedPlan paged_attention_plan(int, int, int, int, int, int, int) { return {0}; }

hipError_t launch_paged_attention(const PagedAttnArgs& a, const PagedPlan&, hipStream_t s) {
  const bool h = a.pages.dtype == LOPA_F16;
  if (a.pages.head_dim == 64) return h ? launch<_Float16, 64>(a, s) : launch<__bf16, 64>(a, s);
  return h ? launch<_Float16, 128>(a, s) : launch<__bf16, 128>(a, s);
}
