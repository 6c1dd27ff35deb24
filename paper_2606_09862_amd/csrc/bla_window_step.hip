// One decode token per row of window attention (bla_window_step).
#include "bla_window.h"

namespace bla {
namespace {

// A workgroup of four waves takes up to 16 query heads of one key head and a part of the ring: the heads are the
// columns of S^T = K Q^T, so a key is read once for all of them.  Wave w walks blocks of 32 slots, four blocks apart, with a
// running maximum and sum of its own; K fragments come straight from memory (a lane's 16 bytes of a row), V rows go through
// a tile of LDS that only the wave touches, to be read transposed.  The waves' results are joined through LDS, the
// parts' by window_join_kernel.  The token's own key and value are taken from k and v wherever its slot is met, so no
// workgroup reads the slot that one of them writes.  Bound: the ring's bytes (512 rows, four key heads of 1028 slots, d = 64, bf16: 76-81 us
// for 408 MB, 5.2 TB/s); of one row, latency (4 key heads of 4100 slots, d = 128: 6 us in 33 parts and 5 us for their join, which
// took 26 us with a thread to four columns of a row).
template <typename T, int D>
__global__ void __launch_bounds__(256) window_step_kernel(WindowStepArgs a)
{
    typedef typename Frag<T>::type F;
    constexpr int PE = 16 / (int)sizeof(T), CH = D / PE, LV = red_ld<T>(D);
    constexpr int NV = 32 * CH / 64;  // 16-byte pieces of V of a lane
    constexpr int LO = D + 4;
    constexpr size_t VB = sizeof(T) * 4 * 32 * LV, OB = sizeof(float) * 4 * 16 * LO;
    __shared__ __attribute__((aligned(16))) char raw[VB > OB ? VB : OB];
    __shared__ float sml[2][4][16];

    unsigned u = blockIdx.x;
    const int part = (int)(u % (unsigned)a.nsplit);
    u /= (unsigned)a.nsplit;
    const int gi = (int)(u % (unsigned)a.ngrp);
    u /= (unsigned)a.ngrp;
    const int hk = (int)(u % (unsigned)a.Hkv), b = (int)(u / (unsigned)a.Hkv);
    const int grp = a.H / a.Hkv, h0 = hk * grp + 16 * gi, nh = min(16, grp - 16 * gi);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const size_t qrow = (size_t)b * a.H + h0, rows = (size_t)a.B * a.H;

    int64_t pos;
    if (row_tokens(nullptr, a.pos, a.t0, b, 1, pos) == 0) {  // a row without a token
        for (int i = tid; i < nh * D; i += 256)
            if (a.nsplit == 1) ((T*)a.o)[qrow * D + i] = (T)0.f;
        if (a.nsplit > 1 && tid < nh) {
            const size_t at = (size_t)part * rows + qrow + tid;
            a.part_ml[2 * at] = kNoMax;
            a.part_ml[2 * at + 1] = 0.f;
        }
        return;
    }
    const int slots = a.S + a.W;
    const int n = (int)min(pos + 1, (int64_t)slots);
    const int mine = pos < a.S ? (int)pos : a.S + (int)((pos - a.S) % a.W);  // the token's slot
    const size_t bh = (size_t)b * a.Hkv + hk;
    const T *kn = (const T*)a.k + bh * D, *vn = (const T*)a.v + bh * D;
    T *ck = (T*)a.ck + bh * slots * D, *cv = (T*)a.cv + bh * slots * D;
    if (part == 0 && gi == 0 && tid < 2 * CH) {
        const int ch = tid % CH;
        if (tid < CH)
            *(intx4*)(ck + (size_t)mine * D + ch * PE) = *(const intx4*)(kn + ch * PE);
        else
            *(intx4*)(cv + (size_t)mine * D + ch * PE) = *(const intx4*)(vn + ch * PE);
    }

    const int nblk = (n + 31) / 32, each = (nblk + a.nsplit - 1) / a.nsplit;
    const int bb = part * each, be = min(nblk, bb + each);

    F qf[D / 32];
    {
        const T* q = (const T*)a.q + (qrow + min(r, nh - 1)) * D;
        const float sgn = a.scale < 0.f ? -1.f : 1.f;
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) {
            qf[kb] = ld_nat(q, kb, g);
            if (a.scale < 0.f)
#pragma unroll
                for (int e = 0; e < 8; ++e) qf[kb][e] = (T)(sgn * (float)qf[kb][e]);
        }
    }
    const float sc = fabsf(a.scale) * kLog2e;

    T* sV = (T*)raw + wave * 32 * LV;
    F kf[2][D / 32];
    intx4 vr[NV];
    auto load = [&](int blk) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const int i = min(32 * blk + 16 * kt + r, n - 1);
            const T* row = i == mine ? kn : ck + (size_t)i * D;
#pragma unroll
            for (int kb = 0; kb < D / 32; ++kb) kf[kt][kb] = ld_nat(row, kb, g);
        }
#pragma unroll
        for (int x = 0; x < NV; ++x) {
            const int i = min(32 * blk + (x * 64 + lane) / CH, n - 1);
            const T* row = i == mine ? vn : cv + (size_t)i * D;
            vr[x] = *(const intx4*)(row + ((x * 64 + lane) % CH) * PE);
        }
    };

    floatx4 acc[D / 16];
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc[dt] = zero4();
    float mx = kNoMax, sum = 0.f;
    int blk = bb + wave;
    if (blk < be) load(blk);
    for (; blk < be; blk += 4) {
#pragma unroll
        for (int x = 0; x < NV; ++x)
            *(intx4*)(sV + ((x * 64 + lane) / CH) * LV + ((x * 64 + lane) % CH) * PE) = vr[x];
        floatx4 s[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            s[kt] = zero4();
#pragma unroll
            for (int kb = 0; kb < D / 32; ++kb) s[kt] = mma(kf[kt][kb], qf[kb], s[kt]);
        }
        if (blk + 4 < be) load(blk + 4);
        if (32 * blk + 32 > n) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[kt][e] = 32 * blk + 16 * kt + 4 * g + e < n ? s[kt][e] : -INFINITY;
        }
        float m = kNoMax;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) m = fmaxf(m, fmaxf(fmaxf(s[kt][0], s[kt][1]), fmaxf(s[kt][2], s[kt][3])));
        m = fmaxf(mx, rows_max(m));
        const float al = exp2_fast((mx - m) * sc), nm = -m * sc;
        mx = m;
        sum *= al;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[kt][e] = exp2_fast(__builtin_fmaf(s[kt][e], sc, nm));
                sum += s[kt][e];
            }
        const F pf = frag_from_acc<T>(s[0], s[1]);
        // the wave's own stores above, read by its other lanes (LDS serves a wave in order)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
            acc[dt] *= al;
            acc[dt] = mma(ld_red(sV, LV, 16 * dt, 0, g, r), pf, acc[dt]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    sum = rows_sum(sum);

    __syncthreads();
    float* sO = (float*)raw;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) st4f(sO + (wave * 16 + r) * LO + 16 * dt + 4 * g, acc[dt]);
    if (g == 0) {
        sml[0][wave][r] = mx * sc;
        sml[1][wave][r] = sum;
    }
    __syncthreads();
    for (int i = tid; i < nh * (D / 4); i += 256) {
        const int hq = i / (D / 4), c = 4 * (i % (D / 4));
        float m = kNoMax * sc;
#pragma unroll
        for (int w = 0; w < 4; ++w) m = fmaxf(m, sml[0][w][hq]);
        float l = 0.f;
        floatx4 o = zero4();
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = exp2_fast(sml[0][w][hq] - m);
            l += f * sml[1][w][hq];
            o += f * ld4f(sO + (w * 16 + hq) * LO + c);
        }
        if (a.nsplit == 1) {
            st4((T*)a.o + (qrow + hq) * D + c, o * (1.f / l));
        } else {
            const size_t at = (size_t)part * rows + qrow + hq;
            st4f(a.part_o + at * D + c, o);
            if (c == 0) {
                a.part_ml[2 * at] = m;
                a.part_ml[2 * at + 1] = l;
            }
        }
    }
}

template <typename T, int D> hipError_t step_d(const WindowStepArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((window_step_kernel<T, D>), dim3((unsigned)((long long)a.B * a.Hkv * a.ngrp * a.nsplit)), dim3(256), 0,
                       s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_window_step(int bf16_io, int D, const WindowStepArgs& a, hipStream_t s)
{
    if (bf16_io) {
        if (D == 32) return step_d<bf16, 32>(a, s);
        if (D == 64) return step_d<bf16, 64>(a, s);
        if (D == 128) return step_d<bf16, 128>(a, s);
    } else {
        if (D == 32) return step_d<float, 32>(a, s);
        if (D == 64) return step_d<float, 64>(a, s);
        if (D == 128) return step_d<float, 128>(a, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace bla
