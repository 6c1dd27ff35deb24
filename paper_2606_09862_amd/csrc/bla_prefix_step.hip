// One decode token per row of window attention behind a prefix that rows share (bla_prefix_step).
#include "bla_window_step.h"

namespace bla {
namespace {

// The rows that share a prefix, with the query heads of a key head, are one matrix of queries: its products with the prefix are matrix products
// without a mask.  A workgroup of four waves takes 64 QT queries (wave w the 16 QT from 16 QT w on) and a part of the prefix, in tiles of 64 tokens that pass
// through two LDS buffers, one barrier per tile, as in window_forward_kernel; each fragment read from LDS serves QT products.  Its result is a part,
// joined with the ring's parts by window_join_kernel.
template <typename T, int D> struct PrefixGeo {
    static constexpr int NT = 256, PE = 16 / (int)sizeof(T), CH = D / PE, RPP = NT / CH, NP = (64 + RPP - 1) / RPP;
    static constexpr int QT = 2, NB = 64 * QT;
    static constexpr int LK = nat_ld<T>(D), LV = red_ld<T>(D), BUF = kWinKeys * (LK + LV);
};

template <typename T, int D> __device__ __forceinline__ void prefix_part(const PrefixStepArgs& a, long long u, T* lds)
{
    typedef PrefixGeo<T, D> G;
    typedef typename Frag<T>::type F;
    constexpr int QT = G::QT;
    const int grp = a.H / a.Hkv, each_row = a.B / a.G;
    const int blk = (int)(u % a.nqb);
    u /= a.nqb;
    const int part = (int)(u % a.npart);
    u /= a.npart;
    const int hk = (int)(u % a.Hkv), gi = (int)(u / a.Hkv);
    const int nq = each_row * grp, q0 = blk * G::NB;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const int np = a.plen ? min(max(a.plen[gi], 0), a.P) : a.P;
    const int ntile = (np + kWinKeys - 1) / kWinKeys, each = (ntile + a.npart - 1) / a.npart;
    const int tb = part * each, te = min(ntile, tb + each);

    const int ch = tid % G::CH, lrow = tid / G::CH;
    const size_t pre = ((size_t)gi * a.Hkv + hk) * a.P * D + ch * G::PE;
    const T *kp = (const T*)a.pk + pre, *vp = (const T*)a.pv + pre;
    intx4 kr[G::NP], vr[G::NP];
    auto load = [&](int tile) {
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            if (G::RPP > 64 && lrow >= kWinKeys) continue;
            const size_t at = (size_t)min(tile * kWinKeys + ps * G::RPP + lrow, np - 1) * D;
            kr[ps] = *(const intx4*)(kp + at);
            vr[ps] = *(const intx4*)(vp + at);
        }
    };

    F qf[QT][D / 32];
    size_t row[QT];
    bool real[QT];
    const int a0 = q0 + 16 * QT * wave;
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int i = min(a0 + 16 * qt + r, nq - 1), b = gi * each_row + i / grp;
        row[qt] = (size_t)b * a.H + hk * grp + i % grp;
        int64_t pos;
        real[qt] = a0 + 16 * qt + r < nq && row_tokens(nullptr, a.pos, a.t0, b, 1, pos) != 0;
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) {
            qf[qt][kb] = ld_nat((const T*)a.q + row[qt] * D, kb, g);
            if (a.scale < 0.f)
#pragma unroll
                for (int e = 0; e < 8; ++e) qf[qt][kb][e] = (T)(-(float)qf[qt][kb][e]);
        }
    }
    const float sc = fabsf(a.scale) * kLog2e, lag = kLag / sc;
    floatx4 acc[QT][D / 16];
    float mx[QT], sum[QT], limit[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        mx[qt] = limit[qt] = kNoMax, sum[qt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) acc[qt][dt] = zero4();
    }

    if (tb < te) load(tb);
    for (int t = tb; t < te; ++t) {
        T *sK = lds + (t & 1) * G::BUF, *sV = sK + kWinKeys * G::LK;
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            const int i = ps * G::RPP + lrow;
            if (G::RPP > 64 && lrow >= kWinKeys) continue;
            *(intx4*)(sK + i * G::LK + ch * G::PE) = kr[ps];
            *(intx4*)(sV + i * G::LV + ch * G::PE) = vr[ps];
        }
        __syncthreads();
        if (t + 1 < te) load(t + 1);
        if (a0 >= nq) continue;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int left = np - t * kWinKeys - 32 * hf;
            if (left <= 0) continue;
            floatx4 s[QT][2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) s[qt][kt] = zero4();
#pragma unroll
                for (int kb = 0; kb < D / 32; ++kb) {
                    const F kf = ld_nat(sK + (32 * hf + 16 * kt + r) * G::LK, kb, g);
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) s[qt][kt] = mma(kf, qf[qt][kb], s[qt][kt]);
                }
            }
            if (left < 32) {
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        s[qt][e >> 2][e & 3] = 4 * g + 16 * (e >> 2) + (e & 3) < left ? s[qt][e >> 2][e & 3] : -INFINITY;
            }
            F pf[QT];
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                floatx4(&x)[2] = s[qt];
                float m = max3(max3(x[0][0], x[0][1], x[0][2]), max3(x[0][3], x[1][0], x[1][1]), max3(x[1][2], x[1][3], x[1][3]));
                if (__any(m > limit[qt])) {  // as in window_forward_kernel
                    m = fmaxf(mx[qt], rows_max(m));
                    const float al = exp2_fast((mx[qt] - m) * sc);
                    sum[qt] *= al;
#pragma unroll
                    for (int dt = 0; dt < D / 16; ++dt) acc[qt][dt] *= al;
                    mx[qt] = m;
                    limit[qt] = m == kNoMax ? kNoMax : m + lag;
                }
                const float nm = -mx[qt] * sc;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[kt][e] = exp2_fast(__builtin_fmaf(x[kt][e], sc, nm));
                        sum[qt] += x[kt][e];
                    }
                pf[qt] = frag_from_acc<T>(x[0], x[1]);
            }
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                const F vf = ld_red(sV, G::LV, 16 * dt, hf, g, r);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) acc[qt][dt] = mma(vf, pf[qt], acc[qt][dt]);
            }
        }
    }
    const size_t rows = (size_t)a.B * a.H;
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const float l = rows_sum(sum[qt]);
        if (a0 + 16 * qt + r >= nq) continue;
        const size_t at = (size_t)part * rows + row[qt];
        if (real[qt])
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) st4f(a.pre_o + at * D + 16 * dt + 4 * g, acc[qt][dt]);
        if (g == 0) {
            a.pre_ml[2 * at] = real[qt] ? mx[qt] * sc : kNoMax;
            a.pre_ml[2 * at + 1] = real[qt] ? l : 0.f;
        }
    }
}

// The prefix's workgroups, then the rings' (which fill the compute units that run out of prefix): one launch.
template <typename T, int D> __global__ void __launch_bounds__(256) prefix_step_kernel(PrefixStepArgs a)
{
    typedef PrefixGeo<T, D> G;
    constexpr size_t PB = sizeof(T) * 2 * G::BUF, LDS = PB > StepGeo<T, D>::LDS ? PB : StepGeo<T, D>::LDS;
    __shared__ __attribute__((aligned(16))) char raw[LDS];
    __shared__ float sml[2][4][16];
    if (blockIdx.x < 8 * (unsigned)a.per) {
        const long long u = xcd_unit(blockIdx.x, a.per);
        if (u < a.units) prefix_part<T, D>(a, u, (T*)raw);
        return;
    }
    window_step_part<T, D, kPrefix>(a, blockIdx.x - 8 * (unsigned)a.per, raw, sml);
}

template <typename T, int D> hipError_t prefix_d(const PrefixStepArgs& a, hipStream_t s)
{
    const long long rings = (long long)a.B * a.Hkv * a.ngrp * a.nsplit;
    hipLaunchKernelGGL((prefix_step_kernel<T, D>), dim3((unsigned)(8 * a.per + rings)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

int prefix_step_block() { return PrefixGeo<bf16, 64>::NB; }

hipError_t launch_prefix_step(int bf16_io, int D, const PrefixStepArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) prefix_d<T, DD>(a, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

}  // namespace bla
