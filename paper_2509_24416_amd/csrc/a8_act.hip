// W4A8 and W8A8 linear with activation, gate and residual in its epilogue:
//   Y = R + gate[sample] * act(sum * x_scale * w_scale + bias),
// all of it in fp32 on the exact integer sums, rounded once.  Outputs in fp16, and the choice of the type.
#include "a8_act.h"

namespace clq {

hipError_t launch_a8_act(const Act8Args &g, hipStream_t stream) {
    switch (g.type) {
        case MxType::F16: return launch_act_type<MxType::F16>(g, stream);
        case MxType::BF16: return launch_a8_act_bf16(g, stream);
        case MxType::F32: return launch_a8_act_f32(g, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace clq
