// Window attention over a prompt (bla_window_forward), and the join of parts of a softmax.
#include "bla_window_fwd.h"

namespace bla {
namespace {

// A wave joins a row: lane s holds the maximum and the sum of part s (at most 64 parts), then groups of D / 4 lanes take every
// 64 / (D / 4)-th part's outputs, four columns to a lane, and are added up.  Parts without a visible key have a sum of zero and are not read.
// (One thread to four columns of a row walked the parts one after the other: 26 us for 16 rows of 33 parts.)
template <typename T, int D> __global__ void __launch_bounds__(256) window_join_kernel(JoinArgs a)
{
    constexpr int LR = D / 4, PG = 64 / LR;
    const long long row = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, c = 4 * (lane % LR), pg = lane / LR;
    if (row >= a.rows) return;
    float m = kNoMax, l = 0.f;
    if (lane < a.nsplit) {
        const float* ml = a.part_ml + 2 * ((size_t)lane * a.rows + row);
        l = ml[1];
        m = l != 0.f ? ml[0] : kNoMax;
    }
    float top = m;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    float w = l != 0.f ? exp2_fast(m - top) : 0.f;
    l *= w;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off);
    floatx4 o = zero4();
    for (int s0 = 0; s0 < a.nsplit; s0 += 8 * PG) {  // eight loads in flight; what a part without keys holds is dropped
        floatx4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            v[k] = ld4f(a.part_o + ((size_t)min(s0 + k * PG + pg, a.nsplit - 1) * a.rows + row) * D + c);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int s = s0 + k * PG + pg;
            float ws = __shfl(w, s & 63);  // lanes past nsplit hold a weight of zero
            ws = s < 64 ? ws : 0.f;
            o += ws * (ws != 0.f ? v[k] : zero4());
        }
    }
#pragma unroll
    for (int off = 32; off >= LR; off >>= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], off);
    const bool some = l != 0.f;
    if (pg == 0) st4((T*)a.o + (size_t)row * D + c, some ? o * (1.f / l) : zero4());
    if (a.lse && lane == 0) a.lse[row] = some ? (top + __log2f(l)) * kLn2 : -INFINITY;
}

template <typename T, int D> hipError_t join_d(const JoinArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((window_join_kernel<T, D>), dim3((unsigned)((a.rows + 3) / 4)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_window_forward(int bf16_io, int D, int waves, const WindowArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) forward_d<T, DD, kPlain>(waves, a, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

hipError_t launch_window_join(int bf16_io, int D, const JoinArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) join_d<T, DD>(a, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

}  // namespace bla
