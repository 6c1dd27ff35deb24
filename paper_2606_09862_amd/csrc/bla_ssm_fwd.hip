// The selective scan over a prompt and for single tokens (bla_ssm_forward, bla_ssm_step).
#include "bla_ssm.h"

namespace bla {
namespace {

// A workgroup of four waves walks the chunks of one segment of one head with the state in registers.
//
// Wave w owns 16 tokens of a chunk (columns t of every tile) and NP / 4 rows n of the state, held transposed (accumulator rows d,
// columns n) in float32.  Per chunk:
//   G^T = B C^T (rows u, columns t; tiles u <= t only), weighted by e^{s_t - s_u} dt_u: the operand of the second product;
//   Y^T = h^T C^T scaled by e^{s_t}, plus X^T (weighted G)^T: h is published in LDS in the operand type;
//   h^T <- e^{s_c} h^T + X^T (w B)^T with w_u = e^{s_c - s_u} dt_u: the transposed fragments of X serve both products.
// In bf16 the weighted G and the published h are rounded by 2^-8 relative at most, as y is.  The weights of the state's update keep float32's
// precision (Split) in every segment: the state is a float32 result that is carried on, and y is the same whether it is asked for or not.
// (Weights rounded once in the segments whose state only enters y: 77 us instead of 95 on the shape below.)
// SUM: the segment's own state from zero and its decay, for the scan over the segments; no outputs.
// Bound: the waits between a chunk's two barriers at two waves to a SIMD (in both forms the matrix pipes are busy 17-19 % of the cycles and vector
// instructions issue in 40 %; two workgroups on a compute unit, 8 x 16 heads x 4096 tokens, d = 64, N = 128, bf16, four
// segments: 95-102 us and 43-46 us of SUM for 157 MB; 16 heads x 16411 tokens in float32, d = N = 64, 29 segments: 96 and 33 us).  Waves that own
// columns d and put the weights on X halve the splitting at N = 128 (82 and 40 us), and lose as much where N = 64 or d = 32 (d = 128, N = 64: 106 us
// instead of 82; float32, d = 32, N = 128: 188 instead of 118), since every wave then reads all of B and C from LDS.
template <typename T, int D, int NP> struct SsmGeo {
    static constexpr int PE = 16 / (int)sizeof(T);
    static constexpr int CHX = D / PE, CHB = NP / PE;        // 16-byte pieces of a row
    static constexpr int PX = 64 * CHX / 256, PB = 64 * CHB / 256;
    static constexpr int LX = red_ld<T>(D), LB = nat_ld<T>(NP), LH = red_ld<T>(D);
    static constexpr int TNW = NP / 64, TD = D / 16;
};

template <typename T, int D, int NP, bool SUM>
__global__ void __launch_bounds__(256) ssm_forward_kernel(SsmArgs a)
{
    typedef SsmGeo<T, D, NP> G;
    typedef typename Frag<T>::type F;
    __shared__ __attribute__((aligned(16))) T sX[64 * G::LX];
    __shared__ __attribute__((aligned(16))) T sB[64 * G::LB];
    __shared__ __attribute__((aligned(16))) T sH[SUM ? 8 : NP * G::LH];
    __shared__ __attribute__((aligned(16))) float sS[2][64], sSl[2][64], sDt[2][64], sE[2][64], sW[2][64];
    __shared__ float sTot[2];

    long long u = xcd_unit(blockIdx.x, a.per);
    if (u >= a.units) return;
    const int h = (int)(u % a.H);
    u /= a.H;
    const int nsg = SUM ? a.sub * (a.nseg - 1) : a.nseg;
    const int item = (int)(u % nsg), seg = SUM ? item / a.sub : item, b = (int)(u / nsg);
    const int bh = b * a.H + h, grp = h / (a.H / a.G);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const int len = ssm_length(a.lengths, b, a.L);
    const T* x = (const T*)a.x + (size_t)bh * a.L * D;
    const T* Bm = (const T*)a.Bm + ((size_t)b * a.G + grp) * a.L * a.N;
    const T* Cm = (const T*)a.Cm + ((size_t)b * a.G + grp) * a.L * a.N;
    T* y = SUM ? nullptr : (T*)a.y + (size_t)bh * a.L * D;
    const float* dt = a.dt + (size_t)bh * a.L;
    const double rate = ssm_rate(a.A[h]);
    const float skip = a.Dm ? a.Dm[h] : 0.f;
    const int psz = SUM ? (a.cps + a.sub - 1) / a.sub : a.cps;  // chunks of a part
    const int c0 = seg * a.cps + (SUM ? item % a.sub * psz : 0), c1 = min(min(a.nch, (seg + 1) * a.cps), c0 + psz);
    const int cend = min(c1, (len + 63) / 64);  // chunks past it are padding
    const size_t BH = (size_t)a.B * a.H;

    floatx4 hs[G::TNW][G::TD];  // h[n = 16 (TNW wave + nt) + r][d = 16 dt + 4g ..]
    const float* from = SUM ? nullptr : seg == 0 ? (a.state_in ? a.state_in + (size_t)bh * a.N * D : nullptr)
                                                 : a.seg_state + ((size_t)(a.sub * seg - 1) * BH + bh) * a.N * D;
#pragma unroll
    for (int nt = 0; nt < G::TNW; ++nt) {
        const int n = 16 * (G::TNW * wave + nt) + r;
#pragma unroll
        for (int d = 0; d < G::TD; ++d)
            hs[nt][d] = from && n < a.N ? ld4f(from + (size_t)n * D + 16 * d + 4 * g) : zero4();
    }

    intx4 xr[G::PX], br[G::PB];
    F cf[NP / 32], cn[NP / 32];
    auto load = [&](int c) {
        const int n = min(64, len - 64 * c);
        if (n == 64 && a.N == NP) {  // whole tiles lie in one piece: no arithmetic on the lanes
            const T *xc = x + (size_t)(64 * c) * D, *bc = Bm + (size_t)(64 * c) * NP, *cc = Cm + (size_t)(64 * c) * NP;
#pragma unroll
            for (int i = 0; i < G::PX; ++i) xr[i] = *(const intx4*)(xc + (unsigned)((i * 256 + tid) * G::PE));
#pragma unroll
            for (int i = 0; i < G::PB; ++i) br[i] = *(const intx4*)(bc + (unsigned)((i * 256 + tid) * G::PE));
            if (!SUM)
#pragma unroll
                for (int kb = 0; kb < NP / 32; ++kb) {
                    const T* p = cc + (unsigned)((16 * wave + r) * NP + 32 * kb + 4 * g);
                    cn[kb] = join(ld4<T>(p), ld4<T>(p + 16));
                }
            return;
        }
#pragma unroll
        for (int i = 0; i < G::PX; ++i) {
            const int row = (i * 256 + tid) / G::CHX, ch = (i * 256 + tid) % G::CHX;
            xr[i] = intx4{0, 0, 0, 0};
            if (row < n) xr[i] = *(const intx4*)(x + (size_t)(64 * c + row) * D + ch * G::PE);
        }
#pragma unroll
        for (int i = 0; i < G::PB; ++i) {
            const int row = (i * 256 + tid) / G::CHB, ch = (i * 256 + tid) % G::CHB;
            br[i] = intx4{0, 0, 0, 0};
            if (row < n && ch * G::PE < a.N) br[i] = *(const intx4*)(Bm + (size_t)(64 * c + row) * a.N + ch * G::PE);
        }
        if (!SUM) {
            const int t = 16 * wave + r;
#pragma unroll
            for (int kb = 0; kb < NP / 32; ++kb)
                cn[kb] = t < n ? ld_acc_row<T>(Cm + (size_t)(64 * c + t) * a.N, kb, g, a.N) : zero_frag<T>();
        }
    };
    double decay = 0.0;
    float dtr = 0.f;
    auto load_dt = [&](int c) { dtr = c < cend && lane < len - 64 * c ? dt[64 * c + lane] : 0.f; };
    auto exponents = [&](int buf) {  // of the chunk whose dt is loaded
        const double s = wave_scan(ssm_exponent(dtr, rate)), tot = wave_last(s);
        decay += tot;
        if (!SUM) {
            sS[buf][lane] = (float)s;
            sSl[buf][lane] = (float)(s - (double)(float)s);
            sDt[buf][lane] = dtr;
            sE[buf][lane] = exp2_f64(s);
        }
        sW[buf][lane] = exp2_f64(tot - s) * dtr;
        if (lane == 0) sTot[buf] = exp2_f64(tot);
    };

    if (c0 < cend) load(c0);
    if (wave == 0) {
        load_dt(c0);
        exponents(0);
        load_dt(c0 + 1);
    }
    for (int c = c0, buf = 0; c < cend; ++c, buf ^= 1) {
#pragma unroll
        for (int i = 0; i < G::PX; ++i) {
            const int row = (i * 256 + tid) / G::CHX, ch = (i * 256 + tid) % G::CHX;
            *(intx4*)(sX + row * G::LX + ch * G::PE) = xr[i];
        }
#pragma unroll
        for (int i = 0; i < G::PB; ++i) {
            const int row = (i * 256 + tid) / G::CHB, ch = (i * 256 + tid) % G::CHB;
            *(intx4*)(sB + row * G::LB + ch * G::PE) = br[i];
        }
        if (!SUM) {
#pragma unroll
            for (int kb = 0; kb < NP / 32; ++kb) cf[kb] = cn[kb];
#pragma unroll
            for (int nt = 0; nt < G::TNW; ++nt)
#pragma unroll
                for (int d = 0; d < G::TD; ++d)
                    st4(sH + (16 * (G::TNW * wave + nt) + r) * G::LH + 16 * d + 4 * g, hs[nt][d]);
        }
        __syncthreads();
        if (c + 1 < cend) load(c + 1);

        F pf[2] = {zero_frag<T>(), zero_frag<T>()};
        if (!SUM) {
            const int t = 16 * wave + r;
            const float st = sS[buf][t], stl = sSl[buf][t];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {  // 32 tokens u
                if (hf == 1 && wave < 2) continue;
                floatx4 p[2] = {zero4(), zero4()};
#pragma unroll
                for (int kb = 0; kb < NP / 32; ++kb)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        p[i] = mma(ld_acc(sB, G::LB, 32 * hf + 16 * i, kb, g, r), cf[kb], p[i]);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int u0 = 32 * hf + 16 * i + 4 * g;
                    const floatx4 su = ld4f(sS[buf] + u0), sl = ld4f(sSl[buf] + u0), du = ld4f(sDt[buf] + u0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[i][e] *= exp2_fast((st - su[e]) + (stl - sl[e])) * du[e];
                    if (2 * hf + i >= wave)  // the tile on the diagonal, or the one past it
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[i][e] = u0 + e <= t ? p[i][e] : 0.f;
                }
                pf[hf] = frag_from_acc<T>(p[0], p[1]);
            }
        }
        Split<T> wb[G::TNW][2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const floatx8 w = join(ld4f(sW[buf] + 32 * kb + 4 * g), ld4f(sW[buf] + 32 * kb + 16 + 4 * g));
#pragma unroll
            for (int nt = 0; nt < G::TNW; ++nt)
                wb[nt][kb].set(w * to_f8(ld_red(sB, G::LB, 16 * (G::TNW * wave + nt), kb, g, r)));
        }
        const float es = SUM ? 0.f : sE[buf][16 * wave + r], tot = sTot[buf];
#pragma unroll
        for (int nt = 0; nt < G::TNW; ++nt)
#pragma unroll
            for (int d = 0; d < G::TD; ++d) hs[nt][d] *= tot;
        // the columns d in pairs of tiles, whose products alternate
#pragma unroll
        for (int d = 0; d < G::TD; d += 2) {
            F xf[2][2];  // [kb][tile]
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 2; ++i) xf[kb][i] = ld_red(sX, G::LX, 16 * (d + i), kb, g, r);
            if (!SUM) {
                floatx4 o[2] = {zero4(), zero4()};
#pragma unroll
                for (int kb = 0; kb < NP / 32; ++kb)
#pragma unroll
                    for (int i = 0; i < 2; ++i) o[i] = mma(ld_red(sH, G::LH, 16 * (d + i), kb, g, r), cf[kb], o[i]);
                const int t = 64 * c + 16 * wave + r;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    o[i] = mma(xf[0][i], pf[0], o[i] * es);
                    if (wave >= 2) o[i] = mma(xf[1][i], pf[1], o[i]);
                    const floatx4 xt = to_f4(ld4<T>(sX + (16 * wave + r) * G::LX + 16 * (d + i) + 4 * g));
                    o[i] += skip * xt;
                    T* to = y + (size_t)(64 * c) * D + (unsigned)((16 * wave + r) * D + 16 * (d + i) + 4 * g);
                    if (64 * c + 64 <= len)
                        st4(to, o[i]);
                    else if (t < a.L)
                        st4(to, t < len ? o[i] : zero4());
                }
            }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int nt = 0; nt < G::TNW; ++nt) {
                    floatx4 hd[2] = {hs[nt][d], hs[nt][d + 1]};
                    mma_split(xf[kb], wb[nt][kb], hd);
                    hs[nt][d] = hd[0];
                    hs[nt][d + 1] = hd[1];
                }
        }
        if (wave == 0) {  // the wave with the fewest products
            exponents(buf ^ 1);
            load_dt(c + 2);
        }
        __syncthreads();
    }

    if (!SUM) {  // padding
        const int t0 = 64 * max(c0, cend), t1 = min(a.L, 64 * c1);
        for (int i = tid; i < (t1 - t0) * G::CHX; i += 256) *(intx4*)(y + (size_t)t0 * D + (size_t)i * G::PE) = intx4{0, 0, 0, 0};
    }
    float* to = SUM ? a.seg_state + ((size_t)item * BH + bh) * a.N * D
                    : seg == a.nseg - 1 && a.state_out ? a.state_out + (size_t)bh * a.N * D : nullptr;
    if (to) {
#pragma unroll
        for (int nt = 0; nt < G::TNW; ++nt) {
            const int n = 16 * (G::TNW * wave + nt) + r;
            if (n < a.N)
#pragma unroll
                for (int d = 0; d < G::TD; ++d) st4f(to + (size_t)n * D + 16 * d + 4 * g, hs[nt][d]);
        }
    }
    if (SUM && tid == 0) a.seg_decay[(size_t)item * BH + bh] = exp2_f64(decay);
}

// States entering segments 1 .. in place of the segments' own states: four elements of a head's state per lane.
__global__ void __launch_bounds__(256) ssm_scan_kernel(SsmArgs a, int D)
{
    const size_t n4 = (size_t)a.N * D / 4, BH = (size_t)a.B * a.H;
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= BH * n4) return;
    const size_t bh = i / n4;
    floatx4 c = a.state_in ? ld4f(a.state_in + 4 * i) : zero4();
    const int n = a.sub * (a.nseg - 1);
    for (int s0 = 0; s0 < n; s0 += 8) {  // eight segments' states in flight (one at a time: 11 us for 29 segments of 16 heads, now 7)
        floatx4 v[8];
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int s = min(s0 + k, n - 1);
            v[k] = ld4f(a.seg_state + ((size_t)s * BH * n4 + i) * 4);
            w[k] = a.seg_decay[s * BH + bh];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (s0 + k < n) {
                c = c * w[k] + v[k];
                if ((s0 + k) % a.sub == a.sub - 1) st4f(a.seg_state + ((size_t)(s0 + k) * BH * n4 + i) * 4, c);
            }
    }
}

// One token: a workgroup reads and writes a head's state once, four columns of a row per lane; y is summed over the row groups through LDS.
// Bound: the state's bytes (512 x 16 heads, d = 64, N = 128: 100-104 us for 539 MB, 5.3 TB/s).
template <typename T, int D, int PASSES> __global__ void __launch_bounds__(256) ssm_step_kernel(SsmStepArgs a)
{
    constexpr int NQ = D / 4, RPP = 256 / NQ;
    __shared__ __attribute__((aligned(16))) float red[RPP * D];
    const int bh = blockIdx.x, h = bh % a.H, b = bh / a.H, grp = h / (a.H / a.G);
    const int tid = threadIdx.x, qd = tid % NQ, rg = tid / NQ;
    const float* in = a.state_in + (size_t)bh * a.N * D;
    float* out = a.state_out + (size_t)bh * a.N * D;
    floatx4 s[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p)  // a lane reads the rows that it writes, no other: the state may be updated in place
        s[p] = p * RPP + rg < a.N ? ld4f(in + (size_t)(p * RPP + rg) * D + 4 * qd) : zero4();
    const T* Bm = (const T*)a.Bm + ((size_t)b * a.G + grp) * a.N;
    const T* Cm = (const T*)a.Cm + ((size_t)b * a.G + grp) * a.N;
    const float dt = a.dt[bh];
    const float keep = exp2_f64(ssm_exponent(dt, ssm_rate(a.A[h])));
    const floatx4 x = to_f4(ld4<T>((const T*)a.x + (size_t)bh * D + 4 * qd)), xd = dt * x;
    floatx4 y = zero4();
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int n = p * RPP + rg;
        if (n < a.N) {
            const floatx4 v = keep * s[p] + (float)Bm[n] * xd;
            st4f(out + (size_t)n * D + 4 * qd, v);
            y += (float)Cm[n] * v;
        }
    }
    st4f(red + rg * D + 4 * qd, y);
    __syncthreads();
    if (tid < NQ) {
        floatx4 o = (a.Dm ? a.Dm[h] : 0.f) * x;
        for (int i = 0; i < RPP; ++i) o += ld4f(red + i * D + 4 * tid);
        st4((T*)a.y + (size_t)bh * D + 4 * tid, o);
    }
}

template <typename T, int D, int NP> hipError_t forward_n(const SsmArgs& a, hipStream_t s)
{
    if (a.nseg > 1) {
        SsmArgs z = a;
        z.units = (long long)a.B * a.H * a.sub * (a.nseg - 1);
        z.per = (z.units + 7) / 8;
        hipLaunchKernelGGL((ssm_forward_kernel<T, D, NP, true>), dim3((unsigned)(8 * z.per)), dim3(256), 0, s, z);
        const size_t n = (size_t)a.B * a.H * a.N * D / 4;
        hipLaunchKernelGGL(ssm_scan_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a, D);
    }
    hipLaunchKernelGGL((ssm_forward_kernel<T, D, NP, false>), dim3((unsigned)(8 * a.per)), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T, int D> hipError_t forward_d(const SsmArgs& a, hipStream_t s)
{
    return a.N <= 64 ? forward_n<T, D, 64>(a, s) : forward_n<T, D, 128>(a, s);
}

template <typename T, int D> hipError_t step_d(const SsmStepArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)(a.B * a.H));
    constexpr int RPP = 256 / (D / 4);
    const int passes = (a.N + RPP - 1) / RPP;
#define BLA_STEP(P)                                                                            \
    if constexpr (P * RPP < 256) {                                                             \
        if (passes <= P) {                                                                     \
            hipLaunchKernelGGL((ssm_step_kernel<T, D, P>), grid, dim3(256), 0, s, a);          \
            return hipGetLastError();                                                          \
        }                                                                                      \
    }
    BLA_STEP(1)
    BLA_STEP(2)
    BLA_STEP(4)
    BLA_STEP(8)
    BLA_STEP(16)
#undef BLA_STEP
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_ssm_forward(int bf16_io, int D, const SsmArgs& a, hipStream_t s)
{
    if (bf16_io) {
        if (D == 32) return forward_d<bf16, 32>(a, s);
        if (D == 64) return forward_d<bf16, 64>(a, s);
        if (D == 128) return forward_d<bf16, 128>(a, s);
    } else {
        if (D == 32) return forward_d<float, 32>(a, s);
        if (D == 64) return forward_d<float, 64>(a, s);
        if (D == 128) return forward_d<float, 128>(a, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_ssm_step(int bf16_io, int D, const SsmStepArgs& a, hipStream_t s)
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
