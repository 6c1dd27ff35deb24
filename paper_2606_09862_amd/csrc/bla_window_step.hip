// One decode token per row of window attention (bla_window_step).
#include "bla_window_step.h"

namespace bla {

hipError_t launch_window_step(int bf16_io, int D, const WindowStepArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) step_d<T, DD, kPlain>(a, 4, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

}  // namespace bla
