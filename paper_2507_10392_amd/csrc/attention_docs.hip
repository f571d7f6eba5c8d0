// Attention inside packed documents: the choice of the element type's kernels (attention_docs_impl.h).
#include "kernels.h"

namespace zs {

hipError_t attn_docs_bf16(hipStream_t st, const DocAttn& a, bool backward);
hipError_t attn_docs_f16(hipStream_t st, const DocAttn& a, bool backward);
hipError_t attn_docs_f32(hipStream_t st, const DocAttn& a, bool backward);

namespace {
hipError_t run(hipStream_t st, DType dt, const DocAttn& a, bool backward) {
  return dt == F32 ? attn_docs_f32(st, a, backward) : dt == BF16 ? attn_docs_bf16(st, a, backward) : attn_docs_f16(st, a, backward);
}
}  // namespace

int doc_dkv_keys(DType dt, int T, int nh, int nkv) {
  const int most = dt == F32 ? 128 : 64;
  if (cdiv(T, most) * nh < 256) return 32;
  return dt == F32 || cdiv(T, 128) * nkv >= 1024 ? 128 : 64;
}
int doc_dkv_parts(DType dt, int T, int nh, int nkv) {
  const int group = nh / nkv;
  const int64_t blocks = cdiv(T, doc_dkv_keys(dt, T, nh, nkv)) * nkv;
  for (int p = 1; p < group; ++p)
    if (group % p == 0 && blocks * p >= 256) return p;
  return group;
}

namespace {
int64_t delta_bytes(DType dt, int T, int nh) { return cdiv((int64_t)T * nh * 4 * (dt == F16 ? 2 : 1), 256) * 256; }
}  // namespace
int64_t attn_docs_bwd_scratch(DType dt, int T, int nh, int nkv, int d) {
  const int parts = doc_dkv_parts(dt, T, nh, nkv);
  return delta_bytes(dt, T, nh) + (parts > 1 ? cdiv(2ll * parts * T * nkv * d * 4, 256) * 256 : 0);
}
hipError_t attn_docs_fwd(hipStream_t st, DType dt, const DocAttn& a) { return run(st, dt, a, false); }
hipError_t attn_docs_bwd(hipStream_t st, DType dt, const DocAttn& in, void* scratch) {
  DocAttn a = in;
  a.delta = (float*)scratch;
  a.partial = (float*)((char*)scratch + delta_bytes(dt, a.T, a.nh));
  a.parts = doc_dkv_parts(dt, a.T, a.nh, a.nkv);
  return run(st, dt, a, true);
}

}  // namespace zs
