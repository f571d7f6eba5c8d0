// Attention inside packed documents: bf16.
#include "attention_docs_impl.h"

namespace zs {
hipError_t attn_docs_bf16(hipStream_t st, const DocAttn& a, bool backward) { return doc_attention<bf16>(st, a, backward); }
}  // namespace zs
