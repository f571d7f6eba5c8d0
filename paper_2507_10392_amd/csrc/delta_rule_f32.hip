// The gated delta rule inside packed documents: fp32.
#include "delta_rule_impl.h"

namespace zs {
hipError_t delta_rule_f32(hipStream_t st, const DeltaRule& a, bool backward) { return delta_rule_of<float>(st, a, backward); }
}  // namespace zs
