// The gated delta rule inside packed documents: bf16.
#include "delta_rule_impl.h"

namespace zs {
hipError_t delta_rule_bf16(hipStream_t st, const DeltaRule& a, bool backward) { return delta_rule_of<bf16>(st, a, backward); }
}  // namespace zs
