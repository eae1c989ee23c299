// New tokens into a paged K / V cache: per-head RMSNorm, rotate-half rotation and
// the writes, in one pass.
//
// Mathematics: for a head x of d values at position p,
//   y = x / sqrt(mean(x^2) + eps) * w,
//   (y_j, y_{j+h}) -> (y_j c_j - y_{j+h} s_j, y_{j+h} c_j + y_j s_j), h = d / 2,
// with the angle p theta^(-j/h). The turns p theta^(-j/h) / 2 pi are formed and
// reduced to [0, 1) in fp64 (an fp32 product is off by 2^-24 of the angle, 0.04
// rad at position 600,000); the sine and cosine of the reduced turns are fp32.
//
// What bounds it: memory, every value read once and written once. A lane holds 8
// values of a head's first half and the 8 that pair with them, so the rotation
// needs no exchange and the norm one sum over the d / 16 lanes of a head. The
// angles depend on the row and the pair only, and cost more than a head: a
// wavefront computes them once for `per_wave` groups of heads of its row, the next
// group's loads in flight (8192 rows of 28 + 2 x 4 heads of 128, 151 MB: 36 us, 4.2 TB/s;
// with one group a wavefront 55; one row 4.4 us).
#include "paged.h"

#include <algorithm>

namespace {

constexpr int WAVES = 4;

template <typename T, int D>
__global__ void __launch_bounds__(64 * WAVES) paged_append_kernel(AppendArgs a, int groups, int per_wave) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  constexpr int LH = D / 16;   // lanes of a head
  constexpr int HW = 64 / LH;  // heads a wavefront takes at a time
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.batch.rows) return;
  const int Hkv = a.pages.kv_heads, ps = a.pages.page_size, heads = a.heads + 2 * Hkv;
  const int sub = lane % LH, j0 = 8 * sub;
  const T* const q = (const T*)a.q + row * a.ld_q + j0;
  const T* const k = (const T*)a.k + row * a.ld_k + j0;
  const T* const v = (const T*)a.v + row * a.ld_v + j0;
  const auto head_at = [&](int h) {  // a query's, a key's or a value's
    return h < a.heads ? q + h * D : h < a.heads + Hkv ? k + (h - a.heads) * D : v + (h - a.heads - Hkv) * D;
  };
  const int g0 = blockIdx.y * per_wave, g1 = g0 + per_wave < groups ? g0 + per_wave : groups;
  vec8 lo = {}, hi = {};
  const auto load = [&](int g) {
    const int h = g * HW + lane / LH;
    if (h < heads) {
      const T* src = head_at(h);
      lo = *(const vec8*)src, hi = *(const vec8*)(src + D / 2);
    }
  };
  load(g0);

  const int s = seq_of_row(a.batch.q_start, a.batch.n_seq, row);
  if (s < 0) return;
  const int start = a.batch.q_start[s], end = a.batch.q_start[s + 1];
  if (start < 0 || row < start || row >= end || end > a.batch.rows) return;
  const int64_t pos64 = (int64_t)a.batch.kv_len[s] - (end - row);
  const int pos = pos64 < INT32_MIN ? INT32_MIN : (int)pos64;
  // first element of this row's slot in head 0 of its page; < 0: no page
  int64_t slot = -1;
  if (pos >= 0 && pos < a.batch.table_ld * ps) {
    const int page = a.batch.table[(int64_t)s * a.batch.table_ld + (pos >> a.page_shift)];
    if (page >= 0 && page < a.pages.n_pages) slot = ((int64_t)page * Hkv * ps + (pos & (ps - 1))) * D;
  }
  float c[8], sn[8];
  if (a.rotate)
    for (int i = 0; i < 8; ++i) {
      double t = (double)pos * a.turns[j0 + i];
      t -= floor(t);
      sincospif(2.f * (float)t, &sn[i], &c[i]);
    }
  for (int g = g0; g < g1; ++g) {
    const int h = g * HW + lane / LH;
    vec8 x8 = lo, y8 = hi;
    if (g + 1 < g1) load(g + 1);
    const int kind = h < a.heads ? 0 : h < a.heads + Hkv ? 1 : 2;  // query, key, value
    const T* const w = (const T*)(kind == 0 ? a.q_norm : kind == 1 ? a.k_norm : nullptr);
    if (kind < 2) {
      float x[8], y[8];
      for (int i = 0; i < 8; ++i) x[i] = (float)x8[i], y[i] = (float)y8[i];
      if (w) {
        float ss = 0.f;
        for (int i = 0; i < 8; ++i) ss += x[i] * x[i] + y[i] * y[i];
        for (int o = LH / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o);  // the lanes of a head agree on w
        const float r = 1.f / sqrtf(ss * (1.f / D) + a.eps);
        const vec8 wl = *(const vec8*)(w + j0), wh = *(const vec8*)(w + j0 + D / 2);
        for (int i = 0; i < 8; ++i) x[i] *= r * (float)wl[i], y[i] *= r * (float)wh[i];
      }
      if (a.rotate)
        for (int i = 0; i < 8; ++i) {
          const float u = x[i] * c[i] - y[i] * sn[i], z = y[i] * c[i] + x[i] * sn[i];
          x[i] = u, y[i] = z;
        }
      for (int i = 0; i < 8; ++i) x8[i] = (T)x[i], y8[i] = (T)y[i];
    }
    if (h < heads && (kind == 0 || slot >= 0)) {
      T* dst = kind == 0 ? (T*)a.q_out + row * a.ld_out + h * D
                         : (T*)(kind == 1 ? a.pages.k : a.pages.v) + slot +
                               (int64_t)(h - a.heads - (kind == 2 ? Hkv : 0)) * ps * D;
      *(vec8*)(dst + j0) = x8;
      *(vec8*)(dst + j0 + D / 2) = y8;
    }
  }
}

template <typename T, int D>
hipError_t launch(const AppendArgs& a, hipStream_t s) {
  const int heads = a.heads + 2 * a.pages.kv_heads, hw = 64 / (D / 16);
  const int groups = (heads + hw - 1) / hw;
  // as many groups a wavefront as leave 8 wavefronts on every SIMD
  const int64_t waves = (int64_t)a.batch.rows * groups;
  const int per_wave = (int)std::min<int64_t>(groups, std::max<int64_t>(1, waves / (8 * 1024)));
  paged_append_kernel<T, D><<<dim3((a.batch.rows + WAVES - 1) / WAVES, (groups + per_wave - 1) / per_wave),
                              dim3(64 * WAVES), 0, s>>>(a, groups, per_wave);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const AppendArgs& a, hipStream_t s) {
  const bool h = a.pages.dtype == LOPA_F16;
  if (a.pages.head_dim == 64) return h ? launch<_Float16, 64>(a, s) : launch<__bf16, 64>(a, s);
  return h ? launch<_Float16, 128>(a, s) : launch<__bf16, 128>(a, s);
}
