// One decode token per row over a cache of bounded size (bla_evict_step).
#include "bla_evict.h"

namespace bla {
namespace {

// The sums of the weights where several workgroups share a key head's slots or heads: a workgroup takes 256 slots; the maxima and sums of
// up to 64 heads at a time are joined from their parts (a wave to a head, a part to a lane), then each thread adds its slot's weights up, head by head.
__global__ void __launch_bounds__(256) evict_finish_kernel(EvictStepArgs a)
{
    __shared__ float sm[64], sinv[64];
    const int blocks = (a.W + 255) / 256, grp = a.H / a.Hkv;
    const size_t bh = blockIdx.x / blocks;
    const int i = (int)(blockIdx.x % blocks) * 256 + threadIdx.x;
    const int hk = (int)(bh % a.Hkv), b = (int)(bh / a.Hkv);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int64_t pos;
    const bool some = row_tokens(nullptr, a.pos, a.t0, b, 1, pos) != 0;
    const int n = some ? (int)min(pos + 1, (int64_t)a.W) : 0, mine = some ? a.mine[bh] : -1;
    const size_t rows = (size_t)a.B * a.H, row0 = (size_t)b * a.H + (size_t)hk * grp;
    float w = 0.f;
    for (int h0 = 0; some && h0 < grp; h0 += 64) {
        const int nh = min(64, grp - h0);
        for (int h = wave; h < nh; h += 4) {
            float m = kNoMax, l = 0.f;
            if (lane < a.nsplit) {
                const float* ml = a.part_ml + 2 * ((size_t)lane * rows + row0 + h0 + h);
                m = ml[0], l = ml[1];
            }
            float top = m;
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
            l = l != 0.f ? l * exp2_fast(m - top) : 0.f;
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off);
            if (lane == 0) sm[h] = top, sinv[h] = 1.f / l;
        }
        __syncthreads();
        if (i < n)
            for (int h = 0; h < nh; ++h) w += exp2_fast(a.z[(row0 + h0 + h) * a.pitch + i] - sm[h]) * sinv[h];
        __syncthreads();
    }
    if (i < a.W) evict_score_out(a, bh, i, mine, n, pos, w);
}

}  // namespace

hipError_t launch_evict_step(int bf16_io, int D, const EvictStepArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) step_d<T, DD, kEvict>(a, s)
    const auto step = [&]() -> hipError_t { BLA_BY_TYPE(BLA_CALL) };
#undef BLA_CALL
    const hipError_t e = step();
    if (e != hipSuccess || a.fused) return e;
    hipLaunchKernelGGL(evict_finish_kernel, dim3((unsigned)((long long)a.B * a.Hkv * ((a.W + 255) / 256))), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace bla
