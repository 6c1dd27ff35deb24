// One decode token per row over a cache of bounded size (bla_evict_step).
#include "bla_evict.h"

namespace bla {
namespace {

// What is left where several workgroups share a key head's slots or heads.  The first workgroups form the sums of the weights, 256 slots to each: the maxima
// and sums of up to 64 heads at a time are joined from their parts (a wave to a head, a part to a lane), then each thread adds its slot's weights up,
// head by head.  The others join the outputs, four rows to each.
// Bound: latency (16 heads of 4 key heads with 4096 slots, d = 128: 3.9 us behind the 8.4 of the parts; sums and joins in launches of their own 19.3 us a call, so 14.5).
template <typename T, int D> __global__ void __launch_bounds__(256) evict_finish_kernel(EvictStepArgs a)
{
    __shared__ float sm[64], sinv[64];
    const int blocks = (a.W + 255) / 256, grp = a.H / a.Hkv;
    const size_t bh = blockIdx.x / blocks;
    if (bh >= (size_t)a.B * a.Hkv) {
        const JoinArgs j = {a.part_o, a.part_ml, a.o, nullptr, (long long)a.B * a.H, a.nsplit};
        join_rows<T, D>(j, (long long)blockIdx.x - (long long)a.B * a.Hkv * blocks);
        return;
    }
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

template <typename T, int D> hipError_t evict_d(const EvictStepArgs& a, int waves, hipStream_t s)
{
    static_assert(StepGeo<T, D, 4>::LDS + 2 * 4 * 16 * 4 + score_lds(4, sizeof(T) == 2, D) <= 160 * 1024, "the step's LDS");
    static_assert(StepGeo<T, D, 8>::LDS + 2 * 8 * 16 * 4 + score_lds(8, sizeof(T) == 2, D) <= 160 * 1024, "the step's LDS");
    const hipError_t e = step_d<T, D, kEvict>(a, waves, s);
    if (e != hipSuccess || a.fused) return e;
    const long long sums = (long long)a.B * a.Hkv * ((a.W + 255) / 256), joins = ((long long)a.B * a.H + 3) / 4;
    hipLaunchKernelGGL((evict_finish_kernel<T, D>), dim3((unsigned)(sums + joins)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_evict_step(int bf16_io, int D, const EvictStepArgs& a, int waves, hipStream_t s)
{
#define BLA_CALL(T, DD) evict_d<T, DD>(a, waves, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

}  // namespace bla
