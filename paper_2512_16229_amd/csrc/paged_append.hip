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
// angles depend on the row and the pair only: a wavefront computes them once for
// all the heads it takes of its row.
#include "paged.h"

namespace {

constexpr int WAVES = 4;

template <typename T, int D>
__global__ void __launch_bounds__(64 * WAVES) paged_append_kernel(AppendArgs a, int groups, int per_wave) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  constexpr int LH = D / 16;   // lanes of a head
  constexpr int HW = 64 / LH;  // heads a wavefront takes at a time
  const int lane = threadIdx.x & 63;
  const int parts = (groups + per_wave - 1) / per_wave;
  const int64_t item = (int64_t)blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)(item / parts), part = (int)(item % parts);
  if (row >= a.batch.rows) return;
  const int s = seq_of_row(a.batch.q_start, a.batch.n_seq, row);
  if (s < 0) return;
  const int start = a.batch.q_start[s], end = a.batch.q_start[s + 1];
  if (start < 0 || row >= end || end > a.batch.rows) return;
  const int64_t pos64 = (int64_t)a.batch.kv_len[s] - (end - row);
  const int pos = pos64 < INT32_MIN ? INT32_MIN : (int)pos64;
  const int Hkv = a.pages.kv_heads, ps = a.pages.page_size, heads = a.heads + 2 * Hkv;
  // first element of this row's slot in head 0 of its page; < 0: no page
  int64_t slot = -1;
  if (pos >= 0 && pos < a.batch.table_ld * ps) {
    const int page = a.batch.table[(int64_t)s * a.batch.table_ld + pos / ps];
    if (page >= 0 && page < a.pages.n_pages) slot = ((int64_t)page * Hkv * ps + pos % ps) * D;
  }
  const int sub = lane % LH, j0 = 8 * sub;
  float c[8], sn[8];
  if (a.rotate)
    for (int i = 0; i < 8; ++i) {
      double t = (double)pos * a.turns[j0 + i];
      t -= floor(t);
      sincospif(2.f * (float)t, &sn[i], &c[i]);
    }
  const int first = part * per_wave;
  for (int g = first; g < first + per_wave && g < groups; ++g) {
    const int h = g * HW + lane / LH;
    if (h >= heads) continue;
    const int kind = h < a.heads ? 0 : h < a.heads + Hkv ? 1 : 2;  // query, key, value
    const int hh = h - (kind == 0 ? 0 : kind == 1 ? a.heads : a.heads + Hkv);
    if (kind && slot < 0) continue;
    const T* src = (const T*)(kind == 0 ? a.q : kind == 1 ? a.k : a.v) +
                   row * (kind == 0 ? a.ld_q : kind == 1 ? a.ld_k : a.ld_v) + hh * D + j0;
    T* dst = kind == 0 ? (T*)a.q_out + row * a.ld_out + hh * D
                       : (T*)(kind == 1 ? a.pages.k : a.pages.v) + slot + (int64_t)hh * ps * D;
    vec8 lo = *(const vec8*)src, hi = *(const vec8*)(src + D / 2);
    if (kind < 2) {
      float x[8], y[8];
      for (int i = 0; i < 8; ++i) x[i] = (float)lo[i], y[i] = (float)hi[i];
      const T* w = (const T*)(kind == 0 ? a.q_norm : a.k_norm);
      if (w) {
        float ss = 0.f;
        for (int i = 0; i < 8; ++i) ss += x[i] * x[i] + y[i] * y[i];
        for (int o = LH / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
        const float r = 1.f / sqrtf(ss * (1.f / D) + a.eps);
        const vec8 wl = *(const vec8*)(w + j0), wh = *(const vec8*)(w + j0 + D / 2);
        for (int i = 0; i < 8; ++i) x[i] *= r * (float)wl[i], y[i] *= r * (float)wh[i];
      }
      if (a.rotate)
        for (int i = 0; i < 8; ++i) {
          const float u = x[i] * c[i] - y[i] * sn[i], v = y[i] * c[i] + x[i] * sn[i];
          x[i] = u, y[i] = v;
        }
      for (int i = 0; i < 8; ++i) lo[i] = (T)x[i], hi[i] = (T)y[i];
    }
    *(vec8*)(dst + j0) = lo;
    *(vec8*)(dst + j0 + D / 2) = hi;
  }
}

template <typename T, int D>
hipError_t launch(const AppendArgs& a, hipStream_t s) {
  const int heads = a.heads + 2 * a.pages.kv_heads, hw = 64 / (D / 16);
  const int groups = (heads + hw - 1) / hw;
  const int per_wave = 1;
  const int64_t waves = (int64_t)a.batch.rows * ((groups + per_wave - 1) / per_wave);
  paged_append_kernel<T, D><<<dim3((unsigned)((waves + WAVES - 1) / WAVES)), dim3(64 * WAVES), 0, s>>>(
      a, groups, per_wave);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const AppendArgs& a, hipStream_t s) {
  const bool h = a.pages.dtype == LOPA_F16;
  if (a.pages.head_dim == 64) return h ? launch<_Float16, 64>(a, s) : launch<__bf16, 64>(a, s);
  return h ? launch<_Float16, 128>(a, s) : launch<__bf16, 128>(a, s);
}
