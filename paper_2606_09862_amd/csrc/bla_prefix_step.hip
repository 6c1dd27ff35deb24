// One decode token per row of window attention behind a prefix that rows share (bla_prefix_step).
#include "bla_window_step.h"

namespace bla {
namespace {

// The rows that share a prefix, with the query heads of a key head, are one matrix of queries: its products with the prefix are matrix products
// without a mask.  A workgroup takes 64 QT queries and a part of the prefix, in tiles of 64 tokens that pass through two LDS buffers, one barrier per
// tile, as in window_forward_kernel; each fragment read from LDS serves QT products.  KG groups of four waves take every KG-th tile, wave w of a group the
// 16 QT queries from 16 QT w on, and are joined through LDS, so that a workgroup fills half a compute unit and leaves one part for as many waves.  The parts are
// joined with the ring's by window_join_kernel.  Bound: for one prefix of many tokens neither its bytes nor issue: a group walks four tiles or so, one ahead, so that
// starting and ending weigh as much as the stream (16 rows x 16 heads on 2 behind 65536 tokens, d = 128, bf16: 26 us for 67 MB read and 17 MB of parts, 3.2 TB/s, with 128
// parts; 44 in all with 48 parts of one group, 29 now); with as many rows as fill the device also the rings' (256 rows x 16 heads on 4
// behind 8192, rings of 512, d = 64: 33 us for 110 MB and 9 GFLOP).
// Few queries (kFewQueries) leave most of such a workgroup idle: they go as the heads of a ring do, in window_step_part.  Where prefix and ring are short as well
// (short_ring), a workgroup of eight waves takes both for its key head's heads of one row: one launch, without parts, though each row reads the
// prefix for itself (3 rows of float32 behind 777 tokens, d = 32: 14.3 us a call with parts, 9.5 without; the kernel takes 8.8).
template <typename T, int D> struct PrefixGeo {
    static constexpr int NT = 256, PE = 16 / (int)sizeof(T), CH = D / PE, RPP = NT / CH, NP = (64 + RPP - 1) / RPP;  // of a group
    static constexpr int QT = 2, NB = 64 * QT;
    static constexpr int LK = nat_ld<T>(D), LV = red_ld<T>(D), BUF = kWinKeys * (LK + LV);
    static constexpr size_t ONE = sizeof(T) * 2 * BUF;  // LDS of a group
    static constexpr int KG = ONE > 64 * 1024 && ONE <= 80 * 1024 ? 2 : 1, NW = 4 * KG;
    static constexpr size_t TILES = KG * ONE, RING = StepGeo<T, D, NW>::LDS, LDS = TILES > RING ? TILES : RING;
    static_assert(KG == 1 || sizeof(float) * 4 * 64 * QT * (D / 4 + 2) <= TILES, "the join's LDS");
};

template <typename T, int D> __device__ __forceinline__ void prefix_part(const PrefixStepArgs& a, long long u, char* raw)
{
    typedef PrefixGeo<T, D> G;
    typedef typename Frag<T>::type F;
    constexpr int QT = G::QT, KG = G::KG;
    const int grp = a.H / a.Hkv, each_row = a.B / a.G;
    const int blk = (int)(u % a.nqb);
    u /= a.nqb;
    const int part = (int)(u % a.npart);
    u /= a.npart;
    const int hk = (int)(u % a.Hkv), gi = (int)(u / a.Hkv);
    const int nq = each_row * grp, q0 = blk * G::NB;
    const int kg = KG > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0, tid = threadIdx.x & 255;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    T* const lds = (T*)raw + kg * 2 * G::BUF;
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

    if (tb + kg < te) load(tb + kg);
    int buf = 0;
    for (int t = tb + kg; t - kg < te; t += KG, buf ^= 1) {  // as many rounds in every group
        T *sK = lds + buf * G::BUF, *sV = sK + kWinKeys * G::LK;
        if (t < te)
#pragma unroll
            for (int ps = 0; ps < G::NP; ++ps) {
                const int i = ps * G::RPP + lrow;
                if (G::RPP > 64 && lrow >= kWinKeys) continue;
                *(intx4*)(sK + i * G::LK + ch * G::PE) = kr[ps];
                *(intx4*)(sV + i * G::LV + ch * G::PE) = vr[ps];
            }
        __syncthreads();
        if (t + KG < te) load(t + KG);
        if (a0 >= nq || t >= te) continue;
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
    if constexpr (KG > 1) {
        float* const join = (float*)raw + (size_t)wave * 64 * QT * (D / 4 + 2);
        __syncthreads();
        if (kg == 1) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                float* x = join + qt * 64 * (D / 4 + 2);
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) st4f(x + (dt * 64 + lane) * 4, acc[qt][dt]);
                x[64 * (D / 4) + lane] = mx[qt];
                x[64 * (D / 4 + 1) + lane] = sum[qt];
            }
        }
        __syncthreads();
        if (kg == 1) return;
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const float* x = join + qt * 64 * (D / 4 + 2);
            const float m1 = x[64 * (D / 4) + lane], m = fmaxf(mx[qt], m1), f0 = exp2_fast((mx[qt] - m) * sc), f1 = exp2_fast((m1 - m) * sc);
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) acc[qt][dt] = acc[qt][dt] * f0 + ld4f(x + (dt * 64 + lane) * 4) * f1;
            sum[qt] = sum[qt] * f0 + x[64 * (D / 4 + 1) + lane] * f1;
            mx[qt] = m;
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
template <typename T, int D> __global__ void __launch_bounds__((64 * PrefixGeo<T, D>::NW)) prefix_step_kernel(PrefixStepArgs a)
{
    typedef PrefixGeo<T, D> G;
    __shared__ __attribute__((aligned(16))) char raw[G::LDS];
    __shared__ float sml[2][G::NW][16];
    if (blockIdx.x < 8 * (unsigned)a.per) {
        const long long u = xcd_unit(blockIdx.x, a.per);
        if (u < a.units) prefix_part<T, D>(a, u, raw);
        return;
    }
    window_step_part<T, D, kPrefix, G::NW>(a, blockIdx.x - 8 * (unsigned)a.per, raw, sml);
}

template <typename T, int D> __global__ void __launch_bounds__(256) prefix_few_kernel(PrefixStepArgs a)
{
    __shared__ __attribute__((aligned(16))) char raw[StepGeo<T, D>::LDS];
    __shared__ float sml[2][4][16];
    if (blockIdx.x < 8 * (unsigned)a.per) {
        const long long u = xcd_unit(blockIdx.x, a.per);
        if (u < a.units) window_step_part<T, D, kFew>(a, (unsigned)u, raw, sml);
        return;
    }
    window_step_part<T, D, kPrefix>(a, blockIdx.x - 8 * (unsigned)a.per, raw, sml);
}

template <typename T, int D> __global__ void __launch_bounds__(512) prefix_both_kernel(PrefixStepArgs a)
{
    __shared__ __attribute__((aligned(16))) char raw[StepGeo<T, D, 8>::LDS];
    __shared__ float sml[2][8][16];
    window_step_part<T, D, kBoth, 8>(a, blockIdx.x, raw, sml);
}

template <typename T, int D> hipError_t prefix_d(const PrefixStepArgs& a, PrefixForm form, hipStream_t s)
{
    if (form == kFormBoth) {
        hipLaunchKernelGGL((prefix_both_kernel<T, D>), dim3((unsigned)((long long)a.B * a.Hkv * a.ngrp)), dim3(512), 0, s, a);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)(8 * a.per + (long long)a.B * a.Hkv * a.ngrp * a.nsplit));
    if (form == kFormFew)
        hipLaunchKernelGGL((prefix_few_kernel<T, D>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((prefix_step_kernel<T, D>), grid, dim3(64 * PrefixGeo<T, D>::NW), 0, s, a);
    return hipGetLastError();
}

constexpr int FILL = 256;
template <typename T, int D> PrefixShape shape_d() { return {PrefixGeo<T, D>::NB, PrefixGeo<T, D>::KG, 64 * PrefixGeo<T, D>::NW, FILL}; }

}  // namespace

PrefixShape prefix_shape(int bf16_io, int D)
{
    if (bf16_io) return D == 32 ? shape_d<bf16, 32>() : D == 64 ? shape_d<bf16, 64>() : shape_d<bf16, 128>();
    return D == 32 ? shape_d<float, 32>() : D == 64 ? shape_d<float, 64>() : shape_d<float, 128>();
}

hipError_t launch_prefix_step(int bf16_io, int D, const PrefixStepArgs& a, PrefixForm form, hipStream_t s)
{
#define BLA_CALL(T, DD) prefix_d<T, DD>(a, form, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

}  // namespace bla
