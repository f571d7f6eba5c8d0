// The gated delta rule inside packed documents: half.
#include "delta_rule_impl.h"

namespace zs {
hipError_t delta_rule_f16(hipStream_t st, const DeltaRule& a, bool backward) { return delta_rule_of<f16>(st, a, backward); }
}  // namespace zs
