// Attention inside packed documents, one wave per row: see attention_docs_rows.h.
#include "attention_docs_rows.h"

namespace zs {
namespace {

template <typename T> __device__ __forceinline__ DocRows<T> doc_head(const void* p, int64_t ld, int h, int d) { return DocRows<T>{(const T*)p + h * d, ld}; }
__device__ __forceinline__ DocScore doc_score(const DocAttn& a, int h) { return DocScore{a.softcap, a.slopes ? a.slopes[h] : 0.f}; }

// grid: a wave per row and head.
template <typename T> __global__ __launch_bounds__(256) void doc_fwd_rows_kernel(DocAttn a) {
  __shared__ float rows[4][128];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t at = (int64_t)blockIdx.x * 4 + wave;
  if (at >= (int64_t)a.T * a.nh) return;
  const int i = (int)(at / a.nh), h = (int)(at % a.nh), kv = h / (a.nh / a.nkv);
  const int4 r = doc_range((const int4*)a.ranges, i, a.T);
  T* o = (T*)a.o + i * a.ldo + h * a.d;
  const float lse = doc_fwd_row<T>(rows[wave], i, r.x, r.y, a.d, doc_head<T>(a.q, a.ldq, h, a.d), doc_head<T>(a.k, a.ldkv, kv, a.d),
                                   doc_head<T>(a.v, a.ldkv, kv, a.d), a.scale, doc_score(a, h), lane, [&](int c, float x) { o[c] = from_f<T>(x); });
  if (lane == 0) a.lse[(int64_t)h * a.T + i] = lse;
}

template <typename T> __global__ __launch_bounds__(256) void doc_dq_rows_kernel(DocAttn a) {
  __shared__ float rows[4][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t at = (int64_t)blockIdx.x * 4 + wave;
  if (at >= (int64_t)a.T * a.nh) return;
  const int i = (int)(at / a.nh), h = (int)(at % a.nh), kv = h / (a.nh / a.nkv);
  const int4 r = doc_range((const int4*)a.ranges, i, a.T);
  const T *o = (const T*)a.o + i * a.ldo + h * a.d, *dout = (const T*)a.dout + i * a.ldo + h * a.d;
  float delta = 0.f;
  for (int c = lane; c < a.d; c += 64) delta = fmaf(to_f(dout[c]), to_f(o[c]), delta);
  delta = wave_sum(delta);
  if (lane == 0) a.delta[(int64_t)h * a.T + i] = delta;
  T* dq = (T*)a.dq + i * a.lddq + h * a.d;
  doc_dq_row<T>(rows[wave], i, r.x, r.y, a.d, doc_head<T>(a.q, a.ldq, h, a.d), doc_head<T>(a.k, a.ldkv, kv, a.d), doc_head<T>(a.v, a.ldkv, kv, a.d),
                doc_head<T>(a.dout, a.ldo, h, a.d), a.lse[(int64_t)h * a.T + i], delta, a.scale, doc_score(a, h), lane,
                [&](int c, float x) { dq[c] = from_f<T>(x); });
}

// grid: a wave per key and key head, over the query heads that share it.
template <typename T> __global__ __launch_bounds__(256) void doc_dkv_rows_kernel(DocAttn a) {
  __shared__ float rows[4][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t at = (int64_t)blockIdx.x * 4 + wave;
  if (at >= (int64_t)a.T * a.nkv) return;
  const int j = (int)(at / a.nkv), kv = (int)(at % a.nkv), group = a.nh / a.nkv;
  const int4 r = doc_range((const int4*)a.ranges, j, a.T);
  row_to_lds(rows[wave], (const T*)a.k + j * a.ldkv + kv * a.d, a.d, lane);
  row_to_lds(rows[wave] + 128, (const T*)a.v + j * a.ldkv + kv * a.d, a.d, lane);
  wave_lds_order();
  float dk[2] = {0.f, 0.f}, dv[2] = {0.f, 0.f};
  for (int h = kv * group; h < (kv + 1) * group; ++h)
    doc_dkv_head<T>(rows[wave], j, r.z, r.w, a.d, doc_head<T>(a.q, a.ldq, h, a.d), doc_head<T>(a.dout, a.ldo, h, a.d), a.lse + (int64_t)h * a.T,
                    a.delta + (int64_t)h * a.T, a.scale, doc_score(a, h), lane, dk, dv);
  const int64_t to = j * a.lddkv + kv * a.d;
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (64 * c + lane < a.d) {
      ((T*)a.dk)[to + 64 * c + lane] = from_f<T>(dk[c] * a.scale);
      ((T*)a.dv)[to + 64 * c + lane] = from_f<T>(dv[c]);
    }
}

template <typename T> hipError_t fwd_rows(hipStream_t st, const DocAttn& a) {
  hipLaunchKernelGGL(doc_fwd_rows_kernel<T>, dim3((unsigned)cdiv((int64_t)a.T * a.nh, 4)), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <typename T> hipError_t bwd_rows(hipStream_t st, const DocAttn& a) {
  hipLaunchKernelGGL(doc_dq_rows_kernel<T>, dim3((unsigned)cdiv((int64_t)a.T * a.nh, 4)), dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(doc_dkv_rows_kernel<T>, dim3((unsigned)cdiv((int64_t)a.T * a.nkv, 4)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

int64_t attn_docs_bwd_scratch(DType, int T, int nh, int, int) { return cdiv((int64_t)T * nh * 4, 256) * 256; }
hipError_t attn_docs_fwd(hipStream_t st, DType dt, const DocAttn& a) {
  return dt == F32 ? fwd_rows<float>(st, a) : dt == BF16 ? fwd_rows<bf16>(st, a) : fwd_rows<f16>(st, a);
}
hipError_t attn_docs_bwd(hipStream_t st, DType dt, const DocAttn& in, void* scratch) {
  DocAttn a = in;
  a.delta = (float*)scratch;
  return dt == F32 ? bwd_rows<float>(st, a) : dt == BF16 ? bwd_rows<bf16>(st, a) : bwd_rows<f16>(st, a);
}

}  // namespace zs
