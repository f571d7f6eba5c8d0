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

// delta of every row and, in half, its largest |dO|
int64_t attn_docs_bwd_scratch(DType dt, int T, int nh, int, int) { return cdiv((int64_t)T * nh * 4 * (dt == F16 ? 2 : 1), 256) * 256; }
hipError_t attn_docs_fwd(hipStream_t st, DType dt, const DocAttn& a) { return run(st, dt, a, false); }
hipError_t attn_docs_bwd(hipStream_t st, DType dt, const DocAttn& in, void* scratch) {
  DocAttn a = in;
  a.delta = (float*)scratch;
  return run(st, dt, a, true);
}

}  // namespace zs
