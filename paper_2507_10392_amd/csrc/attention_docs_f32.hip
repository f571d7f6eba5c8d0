// Attention inside packed documents: float.
#include "attention_docs_impl.h"

namespace zs {
hipError_t attn_docs_f32(hipStream_t st, const DocAttn& a, bool backward) { return doc_attention<float>(st, a, backward); }
}  // namespace zs
