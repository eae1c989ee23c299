// C ABI of the serving operators (paged K / V cache, token log probabilities):
// argument checks on the host, then one enqueue on the caller's stream. No
// handle, no device allocation.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/lopa.h"
#include "kernels.h"
#include "verify.h"

namespace {

constexpr int32_t MAX_SEQ = 65535;
constexpr int32_t MAX_BATCH_ROWS = 1 << 24;
constexpr int32_t MAX_HEADS = 1024;
constexpr int32_t MAX_VOCAB = 1 << 24;
// Factors of a score: in units of log2, and in those of the cap, a score of 0 stays 0 and no factor
// is infinite.
constexpr float MAX_FACTOR = 0x1p100f;

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

int check_heads(int32_t heads, int32_t kv_heads, int32_t head_dim) {
  if (head_dim != 64 && head_dim != 128)
    return lopa_fail(LOPA_ESHAPE, "head_dim %d not supported (64, 128)", head_dim);
  if (heads < 1 || kv_heads < 1 || heads > MAX_HEADS || heads % kv_heads)
    return lopa_fail(LOPA_ESHAPE, "heads %d, kv_heads %d: need 1 <= heads <= %d, a multiple of kv_heads",
                     heads, kv_heads, MAX_HEADS);
  return LOPA_OK;
}

int check_paged(const lopa_pages* p, const lopa_paged_batch* b, int32_t heads) {
  if (!p || !b) return lopa_fail(LOPA_EINVAL, "null pages or batch");
  if (p->dtype != LOPA_BF16 && p->dtype != LOPA_F16)
    return lopa_fail(LOPA_EINVAL, "pages of type %d (LOPA_BF16 or LOPA_F16)", p->dtype);
  if (int e = check_heads(heads, p->kv_heads, p->head_dim)) return e;
  const int32_t ps = p->page_size;
  if (ps < 16 || ps > 256 || (ps & (ps - 1)))
    return lopa_fail(LOPA_ESHAPE, "page_size %d not in 16, 32, 64, 128, 256", ps);
  if (p->n_pages < 1) return lopa_fail(LOPA_EINVAL, "n_pages %d < 1", p->n_pages);
  if (!p->k || !p->v) return lopa_fail(LOPA_EINVAL, "null K or V pages");
  if (!aligned16(p->k) || !aligned16(p->v))
    return lopa_fail(LOPA_EINVAL, "K or V pages not 16-byte aligned");
  if (b->n_seq < 0 || b->n_seq > MAX_SEQ || b->rows < 0 || b->rows > MAX_BATCH_ROWS)
    return lopa_fail(LOPA_ESHAPE, "n_seq %d outside [0, %d] or rows %d outside [0, %d]", b->n_seq,
                     MAX_SEQ, b->rows, MAX_BATCH_ROWS);
  if ((int64_t)b->rows * heads >= ((int64_t)1 << 31))
    return lopa_fail(LOPA_ESHAPE, "%d rows of %d heads: need fewer than 2^31", b->rows, heads);
  if (b->n_seq && b->rows) {
    if (!b->table || !b->q_start || !b->kv_len)
      return lopa_fail(LOPA_EINVAL, "null table, q_start or kv_len");
    if (b->table_ld < 1 || (int64_t)b->table_ld * ps >= (1 << 30))
      return lopa_fail(LOPA_ESHAPE, "table_ld %d of pages of %d: need 1 to 2^30 - 1 positions",
                       b->table_ld, ps);
  }
  return LOPA_OK;
}

// a [rows][heads][d] array whose rows lie ld elements apart
int check_rows(const char* name, const void* p, int64_t ld, int32_t heads, int32_t d) {
  if (!p) return lopa_fail(LOPA_EINVAL, "null %s", name);
  if (!aligned16(p)) return lopa_fail(LOPA_EINVAL, "%s not 16-byte aligned", name);
  if (ld < (int64_t)heads * d || ld % 8)
    return lopa_fail(LOPA_EINVAL, "%s: rows %lld elements apart (at least %d, a multiple of 8)", name,
                     (long long)ld, heads * d);
  return LOPA_OK;
}

// Whether two arrays of `rows` rows of 2-byte elements share one: w_a elements each ld_a apart, and
// w_b each ld_b apart. Views of one buffer may interleave without sharing.
bool share(const void* a, int64_t ld_a, int64_t w_a, const void* b, int64_t ld_b, int64_t w_b, int64_t rows) {
  const int64_t d = ((intptr_t)b - (intptr_t)a) / 2;  // both 16-byte aligned
  if (d >= (rows - 1) * ld_a + w_a || -d >= (rows - 1) * ld_b + w_b) return false;
  if (rows == 1) return true;
  if (ld_a == ld_b) {  // row i of a and row i + k of b, |k| < rows: -w_b < d + k ld < w_a
    const auto floor_div = [&](int64_t n) { return n / ld_a - (n % ld_a < 0); };
    const int64_t lo = floor_div(-w_b - d) + 1, hi = floor_div(w_a - 1 - d);
    return (lo > 1 - rows ? lo : 1 - rows) <= (hi < rows - 1 ? hi : rows - 1);
  }
  for (int64_t i = 0, j = 0; i < rows && j < rows;) {
    const int64_t x = i * ld_a, y = d + j * ld_b;
    if (x + w_a <= y)
      ++i;
    else if (y + w_b <= x)
      ++j;
    else
      return true;
  }
  return false;
}

int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? LOPA_OK : lopa_fail(LOPA_EHIP, "%s: %s", what, hipGetErrorString(e));
}

int check_bounds(int32_t heads, int32_t n_seq, int32_t rows, int32_t max_rows, int32_t max_len) {
  if (n_seq < 0 || n_seq > MAX_SEQ || rows < 0 || rows > MAX_BATCH_ROWS)
    return lopa_fail(LOPA_ESHAPE, "n_seq %d outside [0, %d] or rows %d outside [0, %d]", n_seq,
                     MAX_SEQ, rows, MAX_BATCH_ROWS);
  if ((int64_t)rows * heads >= ((int64_t)1 << 31))
    return lopa_fail(LOPA_ESHAPE, "%d rows of %d heads: need fewer than 2^31", rows, heads);
  if (max_rows < 0 || max_len < 0)
    return lopa_fail(LOPA_EINVAL, "max_rows %d or max_len %d negative", max_rows, max_len);
  if (max_len >= (1 << 30)) return lopa_fail(LOPA_ESHAPE, "max_len %d: need less than 2^30", max_len);
  return LOPA_OK;
}

int check_fits(const PagedPlan& plan, int32_t heads, int32_t kv_heads, int32_t n_seq, int32_t rows) {
  if (plan.fits) return LOPA_OK;
  return lopa_fail(LOPA_ESHAPE, "%d rows of %d heads in %d sequences of %d K / V heads: more workgroups than a launch has",
                   rows, heads, n_seq, kv_heads);
}

}  // namespace

extern "C" {

int lopa_paged_append(const lopa_pages* pages, const lopa_paged_batch* batch, int32_t heads,
                      const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v,
                      int64_t ld_v, const void* q_norm, const void* k_norm, float eps,
                      float rope_theta, void* q_out, int64_t ld_out, void* stream) {
  if (int e = check_paged(pages, batch, heads)) return e;
  if ((q_norm || k_norm) && !(eps >= 0.f && std::isfinite(eps)))
    return lopa_fail(LOPA_EINVAL, "eps must be finite and not negative");
  if (!(rope_theta >= 0.f && std::isfinite(rope_theta)))
    return lopa_fail(LOPA_EINVAL, "rope_theta must be finite and not negative (0: no rotation)");
  if (!aligned16(q_norm) || !aligned16(k_norm))
    return lopa_fail(LOPA_EINVAL, "q_norm or k_norm not 16-byte aligned");
  if (batch->rows == 0 || batch->n_seq == 0) return LOPA_OK;
  const int d = pages->head_dim;
  if (int e = check_rows("q", q, ld_q, heads, d)) return e;
  if (int e = check_rows("k", k, ld_k, pages->kv_heads, d)) return e;
  if (int e = check_rows("v", v, ld_v, pages->kv_heads, d)) return e;
  if (int e = check_rows("q_out", q_out, ld_out, heads, d)) return e;
  const int64_t rows = batch->rows, wq = (int64_t)heads * d, wk = (int64_t)pages->kv_heads * d;
  if (share(q_out, ld_out, wq, k, ld_k, wk, rows) || share(q_out, ld_out, wq, v, ld_v, wk, rows) ||
      (!(q_out == q && (ld_out == ld_q || rows == 1)) && share(q_out, ld_out, wq, q, ld_q, wq, rows)))
    return lopa_fail(LOPA_EINVAL, "q_out shares memory with k, v or other rows of q");
  AppendArgs a{};
  a.pages = *pages;
  a.batch = *batch;
  a.heads = heads;
  a.q = q, a.k = k, a.v = v, a.q_out = q_out;
  a.ld_q = ld_q, a.ld_k = ld_k, a.ld_v = ld_v, a.ld_out = ld_out;
  a.q_norm = q_norm, a.k_norm = k_norm;
  a.eps = eps;
  a.rotate = rope_theta > 0.f;
  a.page_shift = __builtin_ctz(pages->page_size);
  // turns per position of each pair, in fp64 (one product a pair: off by j 2^-53)
  const double ratio = a.rotate ? std::pow((double)rope_theta, -2.0 / d) : 0.0;
  double turns = a.rotate ? 1.0 / (2.0 * M_PI) : 0.0;
  for (int j = 0; j < d / 2; ++j, turns *= ratio) a.turns[j] = turns;
  return launched(launch_paged_append(a, (hipStream_t)stream), "paged append");
}

int64_t lopa_paged_attention_workspace(int32_t heads, int32_t kv_heads, int32_t head_dim,
                                       int32_t n_seq, int32_t rows, int32_t max_rows,
                                       int32_t max_len) {
  if (int e = check_heads(heads, kv_heads, head_dim)) return e;
  if (int e = check_bounds(heads, n_seq, rows, max_rows, max_len)) return e;
  const PagedPlan plan = paged_attention_plan(heads, kv_heads, head_dim, n_seq, rows, max_rows, max_len);
  if (int e = check_fits(plan, heads, kv_heads, n_seq, rows)) return e;
  return plan.bytes;
}

int lopa_paged_attention(const lopa_pages* pages, const lopa_paged_batch* batch, int32_t heads,
                         int32_t max_rows, int32_t max_len, const void* q, int64_t ld_q,
                         int32_t block, float scale, float softcap, void* out, int64_t ld_out,
                         float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  if (int e = check_paged(pages, batch, heads)) return e;
  if (int e = check_bounds(heads, batch->n_seq, batch->rows, max_rows, max_len)) return e;
  if (block < 0) return lopa_fail(LOPA_EINVAL, "block %d negative (0 full, 1 causal, c block-causal)", block);
  if (!(std::fabs(scale) <= MAX_FACTOR)) return lopa_fail(LOPA_EINVAL, "scale outside [-2^100, 2^100]");
  if (softcap != 0.f && !(softcap >= 1 / MAX_FACTOR && softcap <= MAX_FACTOR &&
                          std::fabs(scale) / softcap <= MAX_FACTOR))
    return lopa_fail(LOPA_EINVAL, "softcap, 1 / softcap or |scale| / softcap outside [0, 2^100] (softcap 0: none)");
  if (batch->rows == 0 || batch->n_seq == 0 || max_rows == 0) return LOPA_OK;
  if (max_len > (int64_t)batch->table_ld * pages->page_size)
    return lopa_fail(LOPA_ECAPACITY, "max_len %d exceeds the table's %lld positions", max_len,
                     (long long)batch->table_ld * pages->page_size);
  const int d = pages->head_dim;
  if (int e = check_rows("q", q, ld_q, heads, d)) return e;
  if (int e = check_rows("out", out, ld_out, heads, d)) return e;
  const PagedPlan plan = paged_attention_plan(heads, pages->kv_heads, d, batch->n_seq, batch->rows,
                                              max_rows, max_len);
  if (int e = check_fits(plan, heads, pages->kv_heads, batch->n_seq, batch->rows)) return e;
  if (plan.bytes > 0) {
    if (workspace_bytes < plan.bytes)
      return lopa_fail(LOPA_ESHAPE, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes,
                       (long long)plan.bytes);
    if (!workspace || !aligned16(workspace))
      return lopa_fail(LOPA_EINVAL, "workspace null or not 16-byte aligned");
  }
  // workgroups of other key splits read q while one writes out
  if (share(q, ld_q, (int64_t)heads * d, out, ld_out, (int64_t)heads * d, batch->rows))
    return lopa_fail(LOPA_EINVAL, "q and out share memory");
  PagedAttnArgs a{};
  a.pages = *pages;
  a.batch = *batch;
  a.heads = heads;
  a.max_rows = max_rows, a.max_len = max_len;
  a.page_shift = __builtin_ctz(pages->page_size);
  a.q = q, a.out = out, a.ld_q = ld_q, a.ld_out = ld_out;
  a.block = block;
  a.scale = scale, a.softcap = softcap;
  a.lse = lse;
  a.ws = (float*)workspace;
  return launched(launch_paged_attention(a, plan, (hipStream_t)stream), "paged attention");
}

int64_t lopa_token_logprobs_workspace(int32_t rows, int32_t vocab, int32_t n_top) {
  if (rows < 0 || rows > MAX_GROUPS || vocab < 1 || vocab > MAX_VOCAB || n_top < 0 ||
      n_top > LOPA_MAX_TOP)
    return lopa_fail(LOPA_ESHAPE, "rows %d, vocab %d or n_top %d outside [0, 2^24 - 1], [1, 2^24], [0, %d]",
                     rows, vocab, n_top, LOPA_MAX_TOP);
  return logprobs_workspace(rows, vocab, n_top);
}

int lopa_token_logprobs(const void* logits, int32_t dtype, int64_t ld, int32_t rows,
                        int32_t vocab, int32_t exclude, const int32_t* tokens, int32_t n_top,
                        float* logprob, float* entropy, int32_t* top_ids, float* top_logprobs,
                        void* workspace, int64_t workspace_bytes, void* stream) {
  const int64_t need = lopa_token_logprobs_workspace(rows, vocab, n_top);
  if (need < 0) return (int)need;
  if (dtype != LOPA_BF16 && dtype != LOPA_F16 && dtype != LOPA_F32)
    return lopa_fail(LOPA_EINVAL, "logits of type %d (LOPA_BF16, LOPA_F16, LOPA_F32)", dtype);
  if (ld < vocab) return lopa_fail(LOPA_EINVAL, "rows %lld elements apart, vocab %d", (long long)ld, vocab);
  if (exclude < -1 || exclude >= vocab)
    return lopa_fail(LOPA_EINVAL, "exclude %d outside [-1, %d)", exclude, vocab);
  if (rows == 0) return LOPA_OK;  // arrays of no rows may be null
  if (!logprob != !tokens)
    return lopa_fail(LOPA_EINVAL, "tokens and logprob go together: both or neither");
  if (n_top ? !top_ids || !top_logprobs : top_ids || top_logprobs)
    return lopa_fail(LOPA_EINVAL, "n_top %d: %s top_ids and top_logprobs", n_top,
                     n_top ? "needs" : "takes no");
  if (!logits) return lopa_fail(LOPA_EINVAL, "null logits");
  if ((uintptr_t)logits % (dtype == LOPA_F32 ? 4 : 2))
    return lopa_fail(LOPA_EINVAL, "logits not aligned to their type");
  if (!logprob && !entropy && !n_top) return LOPA_OK;
  if (need > 0) {
    if (workspace_bytes < need)
      return lopa_fail(LOPA_ESHAPE, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes,
                       (long long)need);
    if (!workspace || !aligned16(workspace))
      return lopa_fail(LOPA_EINVAL, "workspace null or not 16-byte aligned");
  }
  LogprobArgs a{};
  a.logits = logits, a.dtype = dtype, a.ld = ld, a.rows = rows, a.vocab = vocab;
  a.exclude = exclude, a.tokens = tokens, a.n_top = n_top;
  a.logprob = logprob, a.entropy = entropy, a.top_ids = top_ids, a.top_logprobs = top_logprobs;
  a.ws = workspace;
  return launched(launch_token_logprobs(a, (hipStream_t)stream), "token logprobs");
}

}  // extern "C"
