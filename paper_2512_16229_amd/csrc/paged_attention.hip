// Attention of a ragged batch's rows over paged K / V.
//
// Mathematics. One pass over the keys with a running reference r and sum l: for a
// tile of keys, x_j = log2(e) s_j, p_j = 2^(x_j - r), l += sum p_j, o += sum p_j V_j;
// out = o / l, lse = (r + log2 l) ln 2. r follows the maximum lazily: o and l are
// rescaled by 2^(r - r') only when some row's maximum has passed r by 2^LIM, so
// most tiles multiply nothing. p is rounded to the pages' type for the product
// with V; fp16 has no exponents below 2^-24, so its numerators are kept 2^8 larger.
//
// Layout. The rows of a tile are (row, query head) pairs of one sequence and K / V
// head, m = row G + head: one read of a K / V tile serves all G query heads. Scores
// are computed transposed, S^T = K Q^T (v_mfma_f32_32x32x16), so a lane holds 16
// keys of one row: the softmax needs one exchange between the two lane halves, and
// its numerators, as they lie, are the right operand of O^T = V^T P^T (the sum over
// keys may be taken in any order, so the keys of a step are those a lane has). V^T's
// operand comes from the row-major V by the transposing LDS read.
//
// K / V tiles go global -> LDS without registers, double-buffered, their page ids read two
// tiles ahead. 16-byte chunks of a row are stored permuted by the row (`swz`), so that the
// reads of 32 rows and the transposing reads of 4 rows touch different banks (no conflicts by
// the counters); the permutation is in the copy's global address.
//
// Split of the work. A workgroup has 4 wavefronts, WM along the rows (32 each) and
// WK = 4 / WM along the keys: few rows take WM = 1, where the wavefronts walk
// different key tiles without a barrier and join at the end. Where the tiles alone
// would leave compute units idle, the keys are also split over workgroups and a
// second kernel joins the parts, in order (paged_plan.h).
//
// What bounds it (MI355X, bf16, head_dim 128): one token a sequence, memory: 48 sequences of up
// to 4000 keys and 32 heads 1.66 GB in 294 us, 5.7 TB/s. A prompt (8191 rows over 14191 keys,
// 28 / 4 heads, causal) 1.13-1.2 ms, 1.0 PFLOP/s: of a key tile's 3100 to 3800 cycles (two
// wavefronts a SIMD) 1830-2250 go to products and exponentials, 640-780 to issuing the eight
// copies, 225-300 to the maximum, 130-230 to the barrier. Few rows and keys: the chain of
// lengths, page ids and first tiles, 7 to 9 us for one key tile.
// Tiles of 128 rows have 256 registers a lane. At head_dim 128 they spill 7 of them, and 63 with a
// cap, whose reloads wait for the copies issued before them: 2047 rows over 4047 keys take 107 us
// uncapped and 309 capped.
#include "paged.h"

#include <type_traits>

namespace {

constexpr float LOG2E = 1.44269504f;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

#define LDS_PTR(T, addr) ((__attribute__((address_space(3))) T*)(uint32_t)(addr))

template <typename T>
struct Num;
template <>
struct Num<__bf16> {
  typedef bf16x8 vec8;
  // numerators reach 2^(x - r) <= 2^LIM; a new reference is the maximum - SHIFT
  static constexpr float SHIFT = 0.f, LIM = 8.f, SCALE = 1.f;  // SCALE = 2^-SHIFT
  static constexpr uint16_t MAX = 0x7f7f;  // bits of the largest finite value
  static __device__ __forceinline__ f32x16 mfma(vec8 a, vec8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Num<_Float16> {
  typedef f16x8 vec8;
  static constexpr float SHIFT = 8.f, LIM = 14.f, SCALE = 0.00390625f;
  static constexpr uint16_t MAX = 0x7bff;
  static __device__ __forceinline__ f32x16 mfma(vec8 a, vec8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

// n / d for 32-bit n by two products, with m = ceil(2^64 / d) from the host (0 for d = 1): the
// error n (m d - 2^64) / (2^64 d) stays below 1 / d. A kernel of few keys is bound by the
// instructions on its way to them, and a division is about forty.
struct Div {
  uint32_t d;
  uint32_t hi, lo;
};
Div divider(uint32_t d) {
  const uint64_t m = d > 1 ? UINT64_MAX / d + 1 : 0;
  return {d, (uint32_t)(m >> 32), (uint32_t)m};
}
__device__ __forceinline__ uint32_t quotient(uint32_t n, const Div& v) {
  return v.d == 1 ? n : (uint32_t)(((uint64_t)n * v.hi + (((uint64_t)n * v.lo) >> 32)) >> 32);
}

// A launch covers the sequences with m_lo < rows x G <= m_hi.
struct AttnLaunch {
  int64_t m_lo, m_hi;
  Div group, kv_heads, per_split, block;  // heads / kv_heads; kv_heads; splits; the mask's block
  int slots;   // row tiles' places: tile t of sequence s at floor(q_start[s] G / BM) + s + t,
  int single;  // or at s where no sequence has more than one
  int splits;  // key splits of `chunk` keys
  int chunk;
  float* ws;   // splits > 1: [slots][Hkv][splits] x ([BM][D] sums, [BM][2] reference and l)
};

template <int V>
using Parity = std::integral_constant<int, V>;  // which of the two buffers

template <int WM>
struct Shape {
  static constexpr int WK = 4 / WM, BM = 32 * WM;
  static constexpr int KT = WM == 1 ? 32 : 64;  // keys of a tile
};

template <int D>
constexpr int part_floats(int bm) { return bm * (D + 2); }

// position limit: keys at or past it are hidden from a row at position p
__device__ __forceinline__ int key_limit(int p, const Div& block, int len) {
  if (block.d == 0) return len;
  if (p < 0) return 0;
  const int64_t lim = ((int64_t)quotient(p, block) + 1) * block.d;
  return lim < len ? (int)lim : len;
}

// ln of a row's sum of 2^x: the reference's shift is taken from both parts exactly
template <typename N>
__device__ __forceinline__ float log_sum(float ref, float l) {
  return l == 0.f ? -INFINITY : ((ref + N::SHIFT) + log2f(l * N::SCALE)) * 0.69314718f;
}

__device__ __forceinline__ float max_halves(float v) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

struct Seq {
  int start, n, len;
};
// false: no such sequence, or one outside the call's bounds
__device__ __forceinline__ bool read_seq(const PagedAttnArgs& a, int s, Seq& q) {
  if (s < 0 || s >= a.batch.n_seq) return false;
  const int start = a.batch.q_start[s], end = a.batch.q_start[s + 1];
  q = {start, end - start, a.batch.kv_len[s]};
  return start >= 0 && end > start && end <= a.batch.rows && q.n <= a.max_rows && q.len >= 0 &&
         q.len <= a.max_len;
}

// nonzero for each of the two 16-bit values that is infinite or NaN
template <typename T>
__device__ __forceinline__ u16x2 over_finite(uint32_t v) {
  return __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, v & 0x7fff7fffu),
                                       u16x2{Num<T>::MAX, Num<T>::MAX});
}

// chunk permutation of a K / V row in LDS (D / 8 chunks of 16 bytes)
template <int D>
__device__ __forceinline__ int swz(int row) {
  if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
  return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

template <typename T, int D, int WM, bool CAP>
__global__ void __launch_bounds__(256, WM == 4 ? 2 : 1) attn_kernel(PagedAttnArgs a, AttnLaunch L) {
  typedef Num<T> N;
  typedef typename N::vec8 vec8;
  constexpr int WK = Shape<WM>::WK, BM = Shape<WM>::BM, KT = Shape<WM>::KT, NB = KT / 32;
  constexpr int TILE = KT * D * 2, STAGE = 2 * TILE;     // bytes of K or V, of both
  constexpr int GROUPS = KT / 16, MYG = WM == 4 ? 1 : 2; // 16-row groups of a tile, a wavefront's
  constexpr uint32_t ALL = (1u << GROUPS) - 1;
  constexpr int RPI = 512 / D, IPG = 16 / RPI;           // rows of a copy, copies of a group
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int put_back[1];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wk = wave / WM;
  const int Hkv = a.pages.kv_heads, G = L.group.d, ps = a.pages.page_size;
  const int rest = quotient(blockIdx.x, L.kv_heads), kvh = blockIdx.x - rest * Hkv;
  const int back = quotient(rest, L.per_split), split = rest - back * L.splits, slot = L.slots - 1 - back;

  // which sequence and row tile
  int s = slot, tile = 0;
  if (!L.single)
    s = last_that(a.batch.n_seq, [&](int i) { return (int64_t)a.batch.q_start[i] * G / BM + i <= slot; });
  Seq q;
  if (!read_seq(a, s, q)) return;
  if (!L.single) tile = slot - (int)((int64_t)q.start * G / BM + s);
  const int64_t M = (int64_t)q.n * G;
  if (M <= L.m_lo || M > L.m_hi || tile < 0 || (int64_t)tile * BM >= M) return;  // tile < 0: q_start out of order
  const int m0 = tile * BM, m1 = (int)(M < m0 + BM ? M : m0 + BM);  // this tile's rows
  const int pos0 = q.len - q.n;
  const int lim_tile = key_limit(pos0 + (int)quotient(m1 - 1, L.group), L.block, q.len);
  const int k0 = split * L.chunk;
  if (split > 0 && k0 >= lim_tile) return;
  const int k1 = lim_tile < k0 + L.chunk ? lim_tile : k0 + L.chunk;

  // this lane's row (a row tile's last rows repeat its last one and are not stored)
  const int c = lane & 31, h = lane >> 5;
  const int w0 = m0 + 32 * wm;  // the wavefront's first row
  const int m = w0 + c < m1 ? w0 + c : m1 - 1;
  const int mr = quotient(m, L.group), row = q.start + mr, head = kvh * G + m - mr * G;
  const int lim = key_limit(pos0 + mr, L.block, q.len);
  // rows are in order, and so are their limits
  const int lim_min = w0 < m1 ? __builtin_amdgcn_readlane(lim, 0) : 0;
  const int lim_max = w0 < m1 ? __builtin_amdgcn_readlane(lim, 31) : 0;

  // scores in units of log2: x = sc (q . K), the sign of the scale in q; a scale of 0 is q = 0
  const float sc = a.scale == 0.f ? 1.f : fabsf(a.scale) * LOG2E;
  vec8 qf[D / 16];
  {
    const T* qp = (const T*)a.q + row * a.ld_q + head * D + 8 * h;
#pragma unroll
    for (int st = 0; st < D / 16; ++st) {
      qf[st] = *(const vec8*)(qp + 16 * st);
      if (a.scale <= 0.f) qf[st] = a.scale == 0.f ? vec8{} : -qf[st];
    }
  }

  // copies: this lane's offset inside a 16-row group
  uint32_t voff[IPG];
#pragma unroll
  for (int i = 0; i < IPG; ++i) {
    const int r = RPI * i + lane / (D / 8);
    voff[i] = r * D * 2 + (((lane % (D / 8)) ^ swz<D>(r)) << 4);
  }
  const uint32_t k_ring = lds0 + wk * 2 * STAGE, v_ring = k_ring + 2 * TILE;
  const int64_t page_elems = (int64_t)Hkv * ps * D;
  const T* const kbase = (const T*)a.pages.k + (int64_t)kvh * ps * D;
  const T* const vbase = (const T*)a.pages.v + (int64_t)kvh * ps * D;
  const int32_t* const table = a.batch.table + (int64_t)s * a.batch.table_ld;

  // the pages of a tile: lane j < GROUPS reads that of 16-key group j (-1: none there)
  const int first = k0 / KT + wk, last = (k1 + KT - 1) / KT;  // key tiles first, first + WK, ... < last
  const int iters = (last - k0 / KT + WK - 1) / WK;
  const auto page_of = [&](int it) {
    const int p = (first + it * WK) * KT + 16 * (lane % GROUPS);
    return it < iters && p < k1 ? table[p >> a.page_shift] : -1;
  };
  const auto there = [&](int ids) {  // bit j: group j has a page
    return (uint32_t)(__ballot(ids >= 0 && ids < a.pages.n_pages) & ALL);
  };
  const auto copy = [&](const T* from, uint32_t ring, int it, int ids) {
#pragma unroll
    for (int g = 0; g < MYG; ++g) {
      const int j = WM == 1 ? g : WM == 2 ? 2 * wm + g : wm;
      const int id = __builtin_amdgcn_readlane(ids, j);
      const bool ok = id >= 0 && id < a.pages.n_pages;
      const int64_t off = ok ? id * page_elems + (int64_t)(((first + it * WK) * KT + 16 * j) & (ps - 1)) * D : 0;
      const uint32_t to = ring + (it & 1) * TILE + j * 16 * D * 2;
#pragma unroll
      for (int i = 0; i < IPG; ++i) copy_to_lds(from + off, voff[i], to + i * 1024);
    }
  };
  // A value of V that is not finite would reach rows that do not see its key as 0 x infinity.
  // Where a tile hides keys from some row of the workgroup such values are taken as zeros, by
  // the wavefront that copied them, and put back after the loop for the rows that see them. (Also
  // where no row sees them, with nothing to put back: one token over 1501 keys takes 13.6 us, and
  // 52.5 where the unwritten slots of its last page hold NaN.)
  const int lim_first = key_limit(pos0 + (int)quotient(m0, L.group), L.block, q.len);  // of the tile's first row
  const auto hides = [&](int it, uint32_t have) {
    return have != ALL || (first + it * WK + 1) * KT > lim_first;
  };
  if (threadIdx.x == 0) *put_back = 0;
  __syncthreads();
  const auto make_finite = [&](int it) {
    for (int g = 0; g < MYG; ++g) {
      const int j = WM == 1 ? g : WM == 2 ? 2 * wm + g : wm;
      const uint32_t at = v_ring + (it & 1) * TILE + j * 16 * D * 2 + lane * 16;
#pragma unroll
      for (int i = 0; i < IPG; ++i) {
        u32x4 v = *LDS_PTR(u32x4, at + i * 1024);
        u16x2 any = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) any |= over_finite<T>(v[k]);
        if (__builtin_bit_cast(uint32_t, any) != 0) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const u16x2 d = over_finite<T>(v[k]);
            if (d[0]) v[k] &= 0xffff0000u;
            if (d[1]) v[k] &= 0xffffu;
          }
          *LDS_PTR(u32x4, at + i * 1024) = v;
          *put_back = 1;
        }
      }
    }
  };

  f32x16 o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float ref = -INFINITY, l = 0.f;

  // LDS addresses of a ring, K rows by chunk step and V by (dimension block, key half); the tile's
  // buffer and its rows are constant offsets
  const uint32_t k_swz = (h ^ swz<D>(c)) << 4;
  const int v_r = 4 * h + ((lane & 15) >> 2);
  const uint32_t v_swz = ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swz<D>(v_r)) << 4;
  uint32_t k_at[D / 16], v_at[D / 32][2];
#pragma unroll
  for (int st = 0; st < D / 16; ++st) k_at[st] = k_ring + c * D * 2 + (k_swz ^ (st << 5));
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int u = 0; u < 2; ++u)
      v_at[db][u] = k_ring + v_r * D * 2 + 8 * (lane & 1) + (v_swz ^ (db << 6) ^ (u << 5));
  const auto read_v = [&](auto buf, int t, int db) {
    constexpr int AT = 2 * TILE + decltype(buf)::value * TILE;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, v_at[db][0]) + (AT + t * 16 * D * 2) / 8);
    const s16x4 hi =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, v_at[db][1]) + (AT + (t * 16 + 8) * D * 2) / 8);
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(vec8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  const auto scores = [&](auto buf, f32x16 (&x)[NB]) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[nb][i] = 0.f;
#pragma unroll
    for (int st = 0; st < D / 16; ++st)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const u32x4 kf = LDS_PTR(u32x4, k_at[st])[(decltype(buf)::value * TILE + nb * 32 * D * 2) / 16];
        x[nb] = N::mfma(__builtin_bit_cast(vec8, kf), qf[st], x[nb]);
      }
  };

  // Pipeline: iteration i multiplies K of tile i + 1 while it takes the exponentials of tile i,
  // then V of tile i; the copies of K of tile i + 2 and V of tile i + 1 are in flight meanwhile.
  f32x16 xa[NB], xb[NB];
  uint32_t have = 0;
  int ids1 = -1, ids2 = -1;  // pages of tiles it + 1 and it + 2
  if (iters > 0) {
    const int ids0 = page_of(0);
    ids1 = page_of(1);
    have = there(ids0);
    copy(kbase, k_ring, 0, ids0);
    copy(vbase, v_ring, 0, ids0);
    if (iters > 1) copy(kbase, k_ring, 1, ids1);
    ids2 = page_of(2);
    wait_loads();
    if constexpr (WM > 1) lds_barrier();
    scores(Parity<0>{}, xa);
  }
  // x: the tile's scores; xn: the next one's
  const auto step = [&](auto even, auto odd, int it, f32x16 (&x)[NB], f32x16 (&xn)[NB]) {
    wait_loads();
    if (hides(it, have)) make_finite(it);
    if constexpr (WM > 1)
      lds_barrier();  // every wavefront's copies have landed, and it is done with the tiles before
    else
      wait_lds();
    const uint32_t have_next = there(ids1);
    if (it + 2 < iters) copy(kbase, k_ring, it + 2, ids2);
    if (it + 1 < iters) copy(vbase, v_ring, it + 1, ids1);
    ids1 = ids2;
    ids2 = page_of(it + 3);
    const int kt = (first + it * WK) * KT;
    if constexpr (CAP) {
      // log2(e) cap tanh(y), y = s / cap: for |y| <= TINY by its series (the next term is below
      // 2^-26), else as 1 - 2 / (e^(2y) + 1), which is off by 2^-24 of the cap itself
      constexpr float TINY = 0.35f;
      const float in = (a.scale == 0.f ? 1.f : fabsf(a.scale)) / a.softcap, out = LOG2E * a.softcap;
      float big = 0.f;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[nb][i] *= in, big = fmaxf(big, fabsf(x[nb][i]));
      const auto series = [](float y) {
        const float z = y * y;
        float t = fmaf(z, -1382.f / 155925.f, 62.f / 2835.f);
        t = fmaf(z, t, -17.f / 315.f);
        t = fmaf(z, t, 2.f / 15.f);
        t = fmaf(z, t, -1.f / 3.f);
        return fmaf(y * z, t, y);
      };
      if (!__any(big > TINY)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 16; ++i) x[nb][i] = series(x[nb][i]) * out;
      } else {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float y = x[nb][i], s = series(y);
            const float w = 1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * (2.f * LOG2E)) + 1.f);
            x[nb][i] = (fabsf(y) > TINY ? w : s) * out;
          }
      }
    }
    const float mul = CAP ? 1.f : sc;
    if (have != ALL || kt + KT > lim_min) {
      // hidden keys: those at or past the row's limit and those of missing pages
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int grp = nb * 2 + i / 8;
          const int end = (have >> grp) & 1 ? lim - kt - 4 * h : INT32_MIN;
          if (nb * 32 + 8 * (i / 4) + i % 4 >= end) x[nb][i] = -INFINITY;
        }
    }
    float mt = x[0][0];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mt = fmaxf(mt, x[nb][i]);
    mt = max_halves(mt) * mul;
    if (__any(mt > ref + N::LIM)) {
      const float next = mt > ref + N::LIM ? mt - N::SHIFT : ref;
      const float f = ref == next ? 1.f : __builtin_amdgcn_exp2f(ref - next);
      l *= f;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= f;
      ref = next;
    }
    const float r = ref == -INFINITY ? 0.f : ref;  // no key seen so far
    scores(odd, xn);  // past the last tile: of what the buffer holds, not used
    vec8 pf[2 * NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(x[nb][i], mul, -r));
        l += p;
        pf[2 * nb + i / 8][i % 8] = (T)p;
      }
#pragma unroll
    for (int tt = 0; tt < 2 * NB; ++tt)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) o[db] = N::mfma(read_v(even, tt, db), pf[tt], o[db]);
    have = have_next;
  };
  for (int it = 0; it < iters; it += 2) {
    step(Parity<0>{}, Parity<1>{}, it, xa, xb);
    if (it + 1 < iters) step(Parity<1>{}, Parity<0>{}, it + 1, xb, xa);
  }
  l = sum_halves(l);
  __syncthreads();  // put_back is known
  if (*put_back) {
    for (int it = 0; it < iters; ++it) {
      if (!hides(it, there(page_of(it)))) continue;
      const int kt = (first + it * WK) * KT;
      for (int p = kt; p < kt + KT && p < lim_max && p < k1; ++p) {
        const int id = table[p >> a.page_shift];
        if (id < 0 || id >= a.pages.n_pages) continue;
        const uint16_t* v = (const uint16_t*)vbase + id * page_elems + (int64_t)(p & (ps - 1)) * D + 4 * h;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint16_t y = v[32 * db + 8 * (i / 4) + i % 4];
            if (p < lim && (y & 0x7fff) > N::MAX) o[db][i] += (float)__builtin_bit_cast(T, y);
          }
      }
    }
  }

  float* part = nullptr;
  const bool whole = lim_tile <= L.chunk;  // no other workgroup has keys of this tile
  if (!whole)
    part = L.ws + (((int64_t)slot * Hkv + kvh) * L.splits + split) * part_floats<D>(BM);
  T* const out = (T*)a.out;

  if constexpr (WK == 1) {
    if (w0 + c < m1) {
      if (whole) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* op = out + row * a.ld_out + head * D + 4 * h;
        typedef T vec4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            vec4 w;
            for (int e = 0; e < 4; ++e) w[e] = (T)(l == 0.f ? 0.f : o[db][4 * i + e] * inv);
            *(vec4*)(op + 32 * db + 8 * i) = w;
          }
        if (a.lse && h == 0)
          a.lse[(int64_t)row * a.heads + head] = log_sum<N>(ref, l);
      } else {
        float* pp = part + (32 * wm + c) * D + 4 * h;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            f32x4 w;
            for (int e = 0; e < 4; ++e) w[e] = o[db][4 * i + e];
            *(f32x4*)(pp + 32 * db + 8 * i) = w;
          }
        if (h == 0) {
          part[BM * D + 2 * (32 * wm + c)] = ref;
          part[BM * D + 2 * (32 * wm + c) + 1] = l;
        }
      }
    }
  } else {
    // join the key groups' sums through LDS
    constexpr int LD = D + 4;
    float* const so = (float*)smem;          // [WK][BM][LD]
    float* const sr = so + WK * BM * LD;     // [WK][BM][2]
    __syncthreads();
    {
      float* p = so + (wk * BM + 32 * wm + c) * LD + 4 * h;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x4 w;
          for (int e = 0; e < 4; ++e) w[e] = o[db][4 * i + e];
          *(f32x4*)(p + 32 * db + 8 * i) = w;
        }
      if (h == 0) {
        sr[(wk * BM + 32 * wm + c) * 2] = ref;
        sr[(wk * BM + 32 * wm + c) * 2 + 1] = l;
      }
    }
    __syncthreads();
    constexpr int TPR = 256 / BM, E = D / TPR;  // threads of a row, values each
    const int rr = threadIdx.x / TPR, e0 = (threadIdx.x % TPR) * E;
    if (m0 + rr < m1) {
      float top = -INFINITY, f[WK], sum = 0.f, acc[E];
      for (int k = 0; k < WK; ++k) top = fmaxf(top, sr[(k * BM + rr) * 2]);
      for (int e = 0; e < E; ++e) acc[e] = 0.f;
      for (int k = 0; k < WK; ++k) {
        const float rk = sr[(k * BM + rr) * 2];
        f[k] = rk == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(rk - top);
        // a part without keys has nothing to add (its l is 0, or NaN stays)
        sum += rk == -INFINITY ? sr[(k * BM + rr) * 2 + 1] : f[k] * sr[(k * BM + rr) * 2 + 1];
        for (int e = 0; e < E; e += 4) {
          const f32x4 v = *(const f32x4*)(so + (k * BM + rr) * LD + e0 + e);
          for (int u = 0; u < 4; ++u) acc[e + u] += rk == -INFINITY ? v[u] : f[k] * v[u];
        }
      }
      const int mm = m0 + rr, mq = quotient(mm, L.group);
      if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const int64_t r2 = q.start + mq;
        T* op = out + r2 * a.ld_out + (kvh * G + mm - mq * G) * D + e0;
        for (int e = 0; e < E; e += 8) {
          vec8 w;
          for (int u = 0; u < 8; ++u) w[u] = (T)(sum == 0.f ? 0.f : acc[e + u] * inv);
          *(vec8*)(op + e) = w;
        }
        if (a.lse && e0 == 0)
          a.lse[r2 * a.heads + kvh * G + mm - mq * G] = log_sum<N>(top, sum);
      } else {
        for (int e = 0; e < E; e += 4)
          *(f32x4*)(part + rr * D + e0 + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
        if (e0 == 0) {
          part[BM * D + 2 * rr] = top;
          part[BM * D + 2 * rr + 1] = sum;
        }
      }
    }
  }
}

// Joins the parts of split rows: W wavefronts per (row, query head), D / 4 lanes per part, so
// that 64 / (D / 4) parts are read at a time and wavefront; four such reads are in flight.
struct JoinArgs {
  AttnLaunch l[2];
  int wm[2], n;
};
template <typename T, int D, int W>
__global__ void __launch_bounds__(256) attn_join_kernel(PagedAttnArgs a, JoinArgs j) {
  constexpr int LP = D / 4, AT_ONCE = 64 / LP, UNROLL = 4;
  __shared__ f32x4 so[W > 1 ? W : 1][LP];
  __shared__ float sl[W > 1 ? W : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x, head = W > 1 ? blockIdx.y : blockIdx.y * 4 + wave;
  if (head >= a.heads) return;
  const int s = seq_of_row(a.batch.q_start, a.batch.n_seq, row);
  Seq q;
  if (!read_seq(a, s, q) || row < q.start || row >= q.start + q.n) return;
  const int Hkv = a.pages.kv_heads, G = j.l[0].group.d, kvh = quotient(head, j.l[0].group);
  const int64_t M = (int64_t)q.n * G;
  const int which = j.n > 1 && !(M > j.l[0].m_lo && M <= j.l[0].m_hi);
  const AttnLaunch& L = j.l[which];
  const int lb = 5 + j.wm[which] / 2, bm = 1 << lb;  // 32, 64 or 128 rows
  if (M <= L.m_lo || M > L.m_hi) return;
  const int m = (row - q.start) * G + head - kvh * G, tile = m >> lb, c = m & (bm - 1);
  const int m1 = (int)(M < (int64_t)(tile + 1) * bm ? M : (int64_t)(tile + 1) * bm);
  const int lim = key_limit(q.len - q.n + (int)quotient(m1 - 1, L.group), L.block, q.len);
  if (lim <= L.chunk) return;  // written by its only workgroup
  const int parts = (lim + L.chunk - 1) / L.chunk;
  const int slot = L.single ? s : (int)(((int64_t)q.start * G >> lb) + s) + tile;
  const int64_t stride = part_floats<D>(bm);
  const float* const p0 = L.ws + ((int64_t)slot * Hkv + kvh) * L.splits * stride;
  const float* const refs = p0 + bm * D + 2 * c;
  float top = -INFINITY;
  for (int k = lane; k < parts; k += 64) top = fmaxf(top, refs[k * stride]);
  const int sub = lane % LP, first = (W > 1 ? wave * AT_ONCE : 0) + lane / LP;
  constexpr int STEP = AT_ONCE * W;
  f32x4 acc = {};
  float sum = 0.f;
  for (int base = 0; base < parts; base += STEP * UNROLL) {  // the same for all lanes
    f32x4 v[UNROLL];
    float r[UNROLL], l[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int k = min(base + first + u * STEP, parts - 1);
      v[u] = *(const f32x4*)(p0 + k * stride + c * D + 4 * sub);
      r[u] = refs[k * stride], l[u] = refs[k * stride + 1];
    }
    if (base == 0) top = wave_max(top);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if (base + first + u * STEP >= parts) continue;
      // a part without keys has nothing but zeros (or a NaN that stays); a factor of zero keeps the
      // NaN of a part far below the others (0 x NaN, 0 x infinity)
      const float f = r[u] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(r[u] - top);
      sum += f * l[u];
      for (int e = 0; e < 4; ++e) acc[e] += f * v[u][e];
    }
  }
  for (int o = LP; o < 64; o *= 2) {
    sum += __shfl_xor(sum, o);
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o);
  }
  if constexpr (W > 1) {
    if (lane < LP) so[wave][lane] = acc;
    if (lane == 0) sl[wave] = sum;
    __syncthreads();
    if (wave) return;
    for (int w = 1; w < W; ++w) {
      sum += sl[w];
      for (int e = 0; e < 4; ++e) acc[e] += so[w][sub][e];
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (lane < LP) {
    typedef T vec4 __attribute__((ext_vector_type(4)));
    vec4 w;
    for (int e = 0; e < 4; ++e) w[e] = (T)(sum == 0.f ? 0.f : acc[e] * inv);
    *(vec4*)((T*)a.out + row * a.ld_out + head * D + 4 * sub) = w;
  }
  if (a.lse && lane == 0)
    a.lse[(int64_t)row * a.heads + head] = log_sum<Num<T>>(top, sum);
}

template <typename T, int D, int WM, bool CAP>
hipError_t launch(const PagedAttnArgs& a, const AttnLaunch& L, hipStream_t s) {
  constexpr int WK = Shape<WM>::WK, BM = Shape<WM>::BM, KT = Shape<WM>::KT;
  constexpr int ring = WK * 2 * 2 * KT * D * 2;
  constexpr int join = WK == 1 ? 0 : WK * BM * (D + 4 + 2) * 4;
  constexpr int bytes = ring > join ? ring : join;
  static_assert(bytes <= 160 * 1024, "LDS of one CU");
  const int64_t n = (int64_t)L.slots * L.splits * a.pages.kv_heads;  // <= MAX_GROUPS: plan.fits
  attn_kernel<T, D, WM, CAP><<<dim3((unsigned)n), dim3(256), bytes, s>>>(a, L);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_all(const PagedAttnArgs& a, const PagedPlan& plan, hipStream_t s) {
  char* ws = (char*)a.ws;
  JoinArgs j{};
  int most = 0;
  for (int i = 0; i < plan.n; ++i) {
    const PagedPlan::Part& p = plan.part[i];
    const AttnLaunch L{p.m_lo, p.m_hi, divider(a.heads / a.pages.kv_heads), divider(a.pages.kv_heads),
                       divider(p.splits), divider(a.block), (int)p.slots, p.single, p.splits, p.chunk, (float*)ws};
    ws += p.ws_bytes;
    const bool cap = a.softcap > 0.f;
    hipError_t e;
    if (p.wm == 1)
      e = cap ? launch<T, D, 1, true>(a, L, s) : launch<T, D, 1, false>(a, L, s);
    else if (p.wm == 2)
      e = cap ? launch<T, D, 2, true>(a, L, s) : launch<T, D, 2, false>(a, L, s);
    else
      e = cap ? launch<T, D, 4, true>(a, L, s) : launch<T, D, 4, false>(a, L, s);
    if (e != hipSuccess) return e;
    if (p.splits > 1) {
      j.l[j.n] = L, j.wm[j.n++] = p.wm;
      most = p.splits > most ? p.splits : most;
    }
  }
  if (j.n) {
    // many parts: a workgroup per (row, query head)
    if (most > 16)
      attn_join_kernel<T, D, 4><<<dim3(a.batch.rows, a.heads), dim3(256), 0, s>>>(a, j);
    else
      attn_join_kernel<T, D, 1><<<dim3(a.batch.rows, (a.heads + 3) / 4), dim3(256), 0, s>>>(a, j);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_paged_attention(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  const bool h = a.pages.dtype == LOPA_F16;
  if (a.pages.head_dim == 64) return h ? launch_all<_Float16, 64>(a, p, s) : launch_all<__bf16, 64>(a, p, s);
  return h ? launch_all<_Float16, 128>(a, p, s) : launch_all<__bf16, 128>(a, p, s);
}
