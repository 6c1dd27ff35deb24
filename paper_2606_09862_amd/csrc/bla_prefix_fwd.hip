// Window attention behind tokens that every query sees, over a prompt (bla_prefix_forward, bla_evict_forward).
#include "bla_window_fwd.h"

namespace bla {

hipError_t launch_prefix_forward(int bf16_io, int D, int waves, const PrefixArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) forward_d<T, DD, kPrefix>(waves, a, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

}  // namespace bla
