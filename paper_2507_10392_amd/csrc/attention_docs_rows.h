// Attention inside packed documents of ONE row (or key) by one wavefront in fp32 arithmetic, forward and backward: the formulas as
// they stand, for every case.  The matrix-core kernels fall back to it for rows that did not come out finite: there a key that a
// row does not see takes part with weight zero, and 0 * inf and 0 * NaN are NaN; here such keys are not read.
#pragma once
#include "kernels.h"
#include "attention_rows.h"

namespace zs {

// A score from scale * q.k: capped, and biased by the distance of row and key; `slope_of` receives d score / d (scale q.k).
struct DocScore {
  float softcap, slope;
  __device__ __forceinline__ float operator()(float u, int i, int j, float& slope_of) const {
    slope_of = 1.f;
    if (softcap > 0.f) {
      const float t = tanhf(u / softcap);
      slope_of = (1.f - t) * (1.f + t);
      u = softcap * t;
    }
    return u - slope * fabsf((float)(i - j));
  }
};
template <typename T> struct DocRows { const T* p; int64_t ld; __device__ __forceinline__ const T* row(int i) const { return p + i * ld; } };   // of one head

// The wave's row into LDS of its own as floats.
template <typename T> __device__ __forceinline__ void row_to_lds(float* to, const T* row, int d, int lane) {
  for (int c = lane; c < d; c += 64) to[c] = to_f(row[c]);
}

// NaN in all of a row's columns, which lie lane + 64 c over the wave: no further term changes that, so the walks below end there. Where a training
// step has overflowed, most rows are of this kind: one document of 4096 tokens, 32 heads of 128 over 8, forward of q all NaN 39 ms without the ends,
// 1.4 with them, gradient of dout all NaN 101 and 2.4 (0.16 and 0.5 where all is finite). A row that is not NaN throughout walks on: a single inf in
// dout, whose 32 keys are then formed here, 29 ms.
__device__ __forceinline__ bool all_nan(const float (&x)[2], int d, int lane) {
  return __all((lane >= d || x[0] != x[0]) && (64 + lane >= d || x[1] != x[1]));
}

// Row i, which sees the keys lo .. hi - 1: out(c, o[i][c]) for the columns c = lane and lane + 64 below d.  rows: LDS of the wave's own, 128 floats.
template <typename T, typename F>
__device__ __forceinline__ void doc_fwd_row(float* rows, int i, int lo, int hi, int d, DocRows<T> q, DocRows<T> k, DocRows<T> v, float scale, DocScore score,
                                             int lane, F&& out) {
  if (lo >= hi) {
    for (int c = lane; c < d; c += 64) out(c, 0.f);
    return;
  }
  wave_lds_order();
  row_to_lds(rows, q.row(i), d, lane);
  wave_lds_order();
  float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f}, unused;
  for (int j0 = lo; j0 < hi; j0 += 64) {
    const int j = j0 + lane, n = min(64, hi - j0);
    const float s = j < hi ? score(scale * dot_row(rows, k.row(j), d), i, j, unused) : -INFINITY;
    const float mn = fmaxf(m, wave_max(s)), ref = mn == -INFINITY ? 0.f : mn;
    const float p = j < hi ? expf(s - ref) : 0.f, alpha = expf(m - ref);
    l = l * alpha + wave_sum(p);
    m = mn;
#pragma unroll
    for (int c = 0; c < 2; ++c) acc[c] *= alpha;
    for (int jj = 0; jj < n; ++jj) {
      const float pj = __shfl(p, jj, 64);
      const T* vr = v.row(j0 + jj);
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (64 * c + lane < d) acc[c] += pj * to_f(vr[64 * c + lane]);
    }
    if (all_nan(acc, d, lane)) break;
  }
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (64 * c + lane < d) out(64 * c + lane, acc[c] / l);
}

// dq_i = scale sum_j ds_ij k_j,  ds_ij = p_ij (do_i . v_j - delta_i) s'_ij,  p_ij = exp(s_ij - lse_i): out(c, dq[i][c]).
// rows: LDS of the wave's own, 256 floats.
template <typename T, typename F>
__device__ __forceinline__ void doc_dq_row(float* rows, int i, int lo, int hi, int d, DocRows<T> q, DocRows<T> k, DocRows<T> v, DocRows<T> dout, float lse,
                                           float delta, float scale, DocScore score, int lane, F&& out) {
  float acc[2] = {0.f, 0.f};
  if (lo < hi) {
    wave_lds_order();
    row_to_lds(rows, q.row(i), d, lane);
    row_to_lds(rows + 128, dout.row(i), d, lane);
    wave_lds_order();
  }
  for (int j0 = lo; j0 < hi; j0 += 64) {
    const int j = j0 + lane, n = min(64, hi - j0);
    float ds = 0.f;
    if (j < hi) {
      float slope;
      const float s = score(scale * dot_row(rows, k.row(j), d), i, j, slope);
      ds = expf(s - lse) * (dot_row(rows + 128, v.row(j), d) - delta) * slope;
    }
    for (int jj = 0; jj < n; ++jj) {
      const float dsj = __shfl(ds, jj, 64);
      const T* kr = k.row(j0 + jj);
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (64 * c + lane < d) acc[c] += dsj * to_f(kr[64 * c + lane]);
    }
    if (all_nan(acc, d, lane)) break;
  }
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (64 * c + lane < d) out(64 * c + lane, acc[c] * scale);
}

// Adds one query head's part of dk_j / scale and dv_j, from the rows lo .. hi - 1 that see key j, to dk[c] and dv[c] of the columns
// lane + 64 c.  rows: LDS of the wave's own, 256 floats, which holds k_j and, from 128 on, v_j.  delta: the rows' dO . o, or NULL: formed here.
template <typename T>
__device__ __forceinline__ void doc_dkv_head(const float* rows, int j, int lo, int hi, int d, DocRows<T> q, DocRows<T> dout, DocRows<T> o, const float* lse,
                                             const float* delta, float scale, DocScore score, int lane, float (&dk)[2], float (&dv)[2]) {
  for (int i0 = lo; i0 < hi; i0 += 64) {
    const int i = i0 + lane, n = min(64, hi - i0);
    float p = 0.f, ds = 0.f;
    if (i < hi) {
      float slope;
      p = expf(score(scale * dot_row(rows, q.row(i), d), i, j, slope) - lse[i]);
      float di = 0.f;
      if (delta) di = delta[i];
      else
        for (int c = 0; c < d; ++c) di = fmaf(to_f(dout.row(i)[c]), to_f(o.row(i)[c]), di);
      ds = p * (dot_row(rows + 128, dout.row(i), d) - di) * slope;
    }
    for (int ii = 0; ii < n; ++ii) {
      const float pi = __shfl(p, ii, 64), dsi = __shfl(ds, ii, 64);
      const T *qr = q.row(i0 + ii), *dor = dout.row(i0 + ii);
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (64 * c + lane < d) {
          dv[c] += pi * to_f(dor[64 * c + lane]);
          dk[c] += dsi * to_f(qr[64 * c + lane]);
        }
    }
    if (all_nan(dk, d, lane) && all_nan(dv, d, lane)) break;
  }
}

// The ranges of token t, inside [0, T) whatever the table holds: x .. y - 1 the keys that it sees, z .. w - 1 the rows that see it.
__device__ __forceinline__ int4 doc_range(const int4* ranges, int t, int T) {
  const int4 r = ranges[t];
  return make_int4(max(r.x, 0), min(r.y, T), max(r.z, 0), min(r.w, T));
}

}  // namespace zs
