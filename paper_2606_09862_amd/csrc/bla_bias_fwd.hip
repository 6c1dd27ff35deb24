// Window attention with a learned bias, over a prompt (bla_bias_forward).
#include "bla_window_fwd.h"

namespace bla {

hipError_t launch_bias_forward(int bf16_io, int D, int waves, const BiasArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) forward_d<T, DD, kBias>(waves, a, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

}  // namespace bla
