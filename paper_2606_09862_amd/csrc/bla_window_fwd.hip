// Window attention over a prompt (bla_window_forward), and the join of parts of a softmax.
#include "bla_window_fwd.h"

namespace bla {
namespace {

template <typename T, int D> __global__ void __launch_bounds__(256) window_join_kernel(JoinArgs a) { join_rows<T, D>(a, blockIdx.x); }

// More than 64 parts: a workgroup to a row.  A thread holds a part's maximum and sum, then groups of D / 4 threads take every so-maniest part's outputs,
// eight in flight, and are added up in order (256 rows of 129 parts, d = 128: 5.6 us for 17 MB).
constexpr int kWideParts = 256;
template <typename T, int D> __global__ void __launch_bounds__(256) window_join_wide_kernel(JoinArgs a)
{
    constexpr int LR = D / 4, PG = 256 / LR;
    __shared__ float w[kWideParts], red[2][4];
    __shared__ __attribute__((aligned(16))) float so[PG][D];
    const size_t row = blockIdx.x;
    const int tid = threadIdx.x, wave = tid >> 6, c = 4 * (tid % LR), pg = tid / LR;
    float m = kNoMax, l = 0.f;
    if (tid < a.nsplit) {
        const float* ml = a.part_ml + 2 * ((size_t)tid * a.rows + row);
        l = ml[1];
        m = l != 0.f ? ml[0] : kNoMax;
    }
    float top = m;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    if ((tid & 63) == 0) red[0][wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    const float f = l != 0.f ? exp2_fast(m - top) : 0.f;
    w[tid] = f;
    l *= f;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off);
    if ((tid & 63) == 0) red[1][wave] = l;
    __syncthreads();
    l = red[1][0] + red[1][1] + red[1][2] + red[1][3];
    floatx4 o = zero4();
    for (int s0 = pg; s0 < a.nsplit; s0 += 8 * PG) {
        floatx4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = ld4f(a.part_o + ((size_t)min(s0 + k * PG, a.nsplit - 1) * a.rows + row) * D + c);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float x = s0 + k * PG < a.nsplit ? w[s0 + k * PG] : 0.f;
            o += x * (x != 0.f ? v[k] : zero4());
        }
    }
    st4f(&so[pg][c], o);
    __syncthreads();
    const bool some = l != 0.f;
    if (pg == 0) {
#pragma unroll
        for (int k = 1; k < PG; ++k) o += ld4f(&so[k][c]);
        st4((T*)a.o + row * D + c, some ? o * (1.f / l) : zero4());
    }
    if (a.lse && tid == 0) a.lse[row] = some ? (top + __log2f(l)) * kLn2 : -INFINITY;
}

template <typename T, int D> hipError_t join_d(const JoinArgs& a, hipStream_t s)
{
    if (a.nsplit > 64) {
        if (a.nsplit > kWideParts) return hipErrorInvalidValue;
        hipLaunchKernelGGL((window_join_wide_kernel<T, D>), dim3((unsigned)a.rows), dim3(256), 0, s, a);
        return hipGetLastError();
    }
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
