// Attention inside packed documents: the choice of the element type's kernels (attention_docs_impl.h).
#include "kernels.h"

#include <algorithm>

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
  const int group = nh / nkv;
  auto need = [&](int t) {
    const int parts = doc_dkv_parts(dt, t, nh, nkv);
    return delta_bytes(dt, t, nh) + (parts > 1 ? cdiv(2ll * parts * t * nkv * d * 4, 256) * 256 : 0);
  };
  // Fewer tokens may share the query heads out over more parts and need more, so this is the most that any length up to T needs: in a range of
  // lengths with the same blocks and parts the need grows, and these ranges end where p parts just do not suffice, or the blocks change.
  int64_t most = need(T);
  auto end = [&](int64_t t) {
    if (t > 0 && t < T) most = std::max(most, need((int)t));
  };
  end((dt == F32 ? 128 : 64) * (255 / nh));
  for (int p = 1; p <= group && p * nkv <= 255; ++p)
    if (group % p == 0)
      for (int keys = 32; keys <= 128; keys *= 2) end(keys * (255 / (nkv * p)));
  return most;
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
