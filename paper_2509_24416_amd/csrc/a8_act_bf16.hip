// The 8-bit linear with activation, gate and residual: outputs in bf16.
#include "a8_act.h"

namespace clq {

hipError_t launch_a8_act_bf16(const Act8Args &g, hipStream_t stream) { return launch_act_type<MxType::BF16>(g, stream); }

}  // namespace clq
