// Attention inside packed documents: f16.
#include "attention_docs_impl.h"

namespace zs {
hipError_t attn_docs_f16(hipStream_t st, const DocAttn& a, bool backward) { return doc_attention<f16>(st, a, backward); }
}  // namespace zs
