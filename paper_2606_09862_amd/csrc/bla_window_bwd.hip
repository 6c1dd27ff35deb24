// Backward pass of window attention (bla_window_backward).
#include "bla_window_bwd.h"

namespace bla {

int window_bwd_block(int D) { return D == 128 ? BwdGeo<bf16, 128>::NB : BwdGeo<bf16, 64>::NB; }

hipError_t launch_window_backward(int bf16_io, int D, const WindowBwdArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) backward_d<T, DD, kPlain>(a, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

}  // namespace bla
