// One decode token per row of window attention with a learned bias (bla_bias_step).
#include "bla_window_step.h"

namespace bla {

hipError_t launch_bias_step(int bf16_io, int D, const BiasStepArgs& a, int waves, hipStream_t s)
{
#define BLA_CALL(T, DD) step_d<T, DD, kBias>(a, waves, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

}  // namespace bla
