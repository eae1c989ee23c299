// How attention over pages is launched: row tiles and key splits by the sizes of a call
// (host only).
#pragma once
#include <algorithm>
#include <cstdint>

// workgroups of 256 threads that a launch can have: its grid is counted in 32-bit work-items
constexpr int64_t MAX_GROUPS = ((int64_t)1 << 24) - 1;

struct PagedPlan {
  struct Part {           // one launch: the sequences with m_lo < rows x group <= m_hi
    int wm;               // 32 wm rows a workgroup
    int64_t m_lo, m_hi;
    bool single;          // no sequence has more than one row tile
    int64_t slots;        // row tiles' places
    int splits, chunk;    // key splits of `chunk` keys
    int64_t ws_bytes;
    double us;            // an estimate that orders the forms (see below)
  } part[2];
  int n;
  int64_t bytes;  // workspace of all parts
  bool fits;      // no launch has more than MAX_GROUPS workgroups
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// One launch's place in the plan, and an estimate of what it takes in us, by which row tiles and
// splits are chosen. It is an order of the forms near the sizes it was fitted at and no time: every
// sequence counts as max_len keys, masks, a cap and the host's part do not count (one token over
// 1501 keys 7.5 against 13.1 measured, a capped mixed batch 14.8 / 21.5, 48 sequences of unequal
// lengths 686 / 292, a causal prompt 1893 / 1120). `tiles` row tiles of `seqs` sequences. The keys
// are split where that ends sooner:
//   an iteration of a workgroup is 128 keys by 32 rows (wm = 1), 128 by 64 (2) or 64 by 128 (4);
//   at head_dim 128 it takes 1.55 where a wavefront has 64 keys (2.13 for each of two workgroups
//   on a CU), 1.2 where it has 32, and the running sequences' share of 8 TB/s on top of that
//   where all keys come from memory (one token over 131072 keys and 8 K / V heads: 158 us in 13
//   parts, 114 in 22, 102 in 32);
//   workgroups run in rounds of 256 occ;
//   joining takes 4.5 and the parts' way to memory and back at 4 TB/s (8 branches of 32 rows over
//   544 keys, wm = 4: 21 unsplit, 15 and 7.5 for joining in 5 parts).
// No more than `groups` workgroups with split keys.
inline PagedPlan::Part paged_part(int wm, int64_t m_lo, int64_t m_hi, bool single, int64_t slots, int64_t tiles,
                                  int64_t seqs, int kv_heads, int d, int max_len, int64_t groups) {
  const int bm = 32 * wm, step = wm == 4 ? 64 : 128;
  const int occ = (wm == 4 ? 2 : 1) * (d == 64 ? 2 : 1);
  const double work = d == 64 ? 0.65 : 1.0;
  const int64_t items = std::max<int64_t>(1, tiles * kv_heads);
  const int64_t most = std::max<int64_t>(1, ceil_div(max_len, step));
  double least = 1e30;
  int64_t splits = 1;
  for (int64_t s = 1; s <= most && s <= 1024; s = s < 4 ? s + 1 : s * 4 / 3) {
    if (s > 1 && slots * kv_heads * s > groups) break;
    const double iters = ceil_div(ceil_div(max_len, s), step), n = (double)items * s;
    const double load = n / (256 * occ), rounds = load <= 1.0 ? 1.0 : load + 0.5;
    const double streams = std::min(n, 256.0 * occ) * std::min(1.0, (double)seqs / tiles);
    double t_it = wm == 1 ? 1.2 * work + streams * step * d * 4 / 8e6 : wm == 4 && n > 256 ? 2.13 * work : 1.55 * work;
    double t = (wm == 1 ? 0.0 : 2.0) + rounds * iters * t_it;
    if (s > 1) t += 4.5 + n * bm * d * 8 / 4e6;
    if (t < least) least = t, splits = s;
  }
  const int64_t chunk = std::max<int64_t>(1, ceil_div(ceil_div(max_len, splits), step)) * step;
  splits = std::max<int64_t>(1, ceil_div(max_len, chunk));
  PagedPlan::Part p{};
  p.wm = wm, p.m_lo = m_lo, p.m_hi = m_hi, p.single = single;
  p.slots = slots, p.splits = (int)splits, p.chunk = (int)chunk;
  p.ws_bytes = splits > 1 ? slots * kv_heads * splits * (int64_t)bm * (d + 2) * 4 : 0;
  p.us = least;
  return p;
}

// Rows of a sequence and K / V head up to 32 (a decode step): the wavefronts split the keys.
// More: 32, 64 or 128 rows a workgroup, whichever is expected to end first - many small ones
// where they all run at once, large ones where they do not (8 branches of 32 rows, 28 / 4 heads,
// over 544 keys: 14 us in tiles of 32 rows, 21 in tiles of 128; an 8191-row prompt takes 1.5
// times as long in tiles of 32). In a batch of unequal sequences tiles of 64 and 128 rows leave
// those of up to 32 to a launch of their own.
inline PagedPlan paged_attention_plan(int heads, int kv_heads, int d, int n_seq, int rows, int max_rows,
                                      int max_len) {
  PagedPlan best{};
  best.fits = true;
  if (n_seq < 1 || rows < 1 || max_rows < 1) return best;
  if (max_rows > rows) max_rows = rows;
  const int64_t G = heads / kv_heads, most = max_rows * G, all = INT64_MAX;
  const bool even = rows == (int64_t)n_seq * max_rows;
  const int64_t groups = rows <= MAX_GROUPS ? MAX_GROUPS : 0;  // joining takes one per row
  double least = 1e300;
  for (int wm : {1, 2, 4}) {
    const int bm = 32 * wm;
    if (wm > 1 && most <= bm / 2) break;
    const bool single = most <= bm;
    const int64_t slots = single ? n_seq : rows * G / bm + n_seq;
    const int64_t tiles = single ? n_seq : even ? n_seq * ceil_div(most, bm) : ceil_div(rows * G, bm) + n_seq / 2;
    PagedPlan plan{};
    double us;
    if (wm == 1 || even) {
      plan.part[plan.n++] = paged_part(wm, 0, all, single, slots, tiles, n_seq, kv_heads, d, max_len, groups);
      us = plan.part[0].us;
    } else {
      const int64_t large = std::max<int64_t>(1, std::min<int64_t>(n_seq, rows * G / most));
      plan.part[plan.n++] =
          paged_part(wm, 32, all, single, slots, ceil_div(rows * G, bm), large, kv_heads, d, max_len, groups);
      plan.part[plan.n++] = paged_part(1, 0, 32, true, n_seq, n_seq, n_seq, kv_heads, d, max_len, groups);
      us = plan.part[0].us + plan.part[1].us + 6.0;
    }
    plan.fits = true;
    for (int i = 0; i < plan.n; ++i)
      plan.fits &= plan.part[i].slots * plan.part[i].splits * kv_heads <= MAX_GROUPS;
    if (!plan.fits) us += 1e200;  // only where no other does
    if (us < least) least = us, best = plan;
  }
  for (int i = 0; i < best.n; ++i) best.bytes += best.part[i].ws_bytes;
  return best;
}
