// Backward pass of window attention with a learned bias (bla_bias_backward).
#include "bla_window_bwd.h"

namespace bla {
namespace {

// dbias: a workgroup adds a head's sums up, in float64: a thread takes a bucket of every sixteenth sum, then sixteen threads' are added in order.
// The workgroups of the keys have the head's sums at (unit, wave, head of the group), unit = (b Hkv + hk) nkb + key block; those of the sinks
// behind them, unit = ((b Hkv + hk) tiles + tile) parts + part.
// Bound: latency (16 heads, 8 rows of 2048 keys: 6 us).
__global__ void __launch_bounds__(1024) bias_bwd_sum_kernel(BiasBwdArgs a)
{
    __shared__ double sum[16][kMaxBuckets];
    const int h = blockIdx.x, grp = a.H / a.Hkv, hk = h / grp, hg = h % grp, u = threadIdx.x & 63, part = threadIdx.x >> 6, n = a.spec.buckets;
    const int each = a.s_units ? (int)(a.s_units / ((unsigned)a.B * a.Hkv)) : 0;  // the sinks' workgroups of a key head
    double x = 0.0;
    if (u < n) {
        const auto add = [&](size_t first, int units) {  // units of each row, four waves' sums of each
            const int m = 4 * units;
            for (int b = 0; b < a.B; ++b) {
                const float* p = a.db_part + (((first + ((size_t)b * a.Hkv + hk) * units) * 4) * grp + hg) * n + u;
#pragma unroll 4
                for (int i = part; i < m; i += 16) x += p[(size_t)i * grp * n];
            }
        };
        add(0, a.nkb);
        if (each) add((size_t)a.k_units, each);
    }
    sum[part][u] = x;
    __syncthreads();
    if (part == 0 && u < n) {
        for (int i = 1; i < 16; ++i) x += sum[i][u];
        a.dbias[(size_t)h * n + u] = (float)x;
    }
}

}  // namespace

hipError_t launch_bias_backward(int bf16_io, int D, const BiasBwdArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) backward_d<T, DD, kBias>(a, s)
    const auto passes = [&]() -> hipError_t { BLA_BY_TYPE(BLA_CALL) };
#undef BLA_CALL
    const hipError_t e = passes();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(bias_bwd_sum_kernel, dim3((unsigned)a.H), dim3(1024), 0, s, a);
    return hipGetLastError();
}

}  // namespace bla
