// Backward pass of window attention (bla_window_backward).
//
// With P = exp(scale q k - lse) on the visible pairs and delta_i = sum_c dO_ic o_ic:
//   dS = P (dO v^T - delta),   dq = scale dS k,   dk = scale dS^T q,   dv = P^T dO.
// Two passes recompute P from lse, one per query block (dq, and delta for the other) and one per key block (dk, dv, summed over the
// heads that share the key head and over the queries that see the block), so that every gradient has one
// owner and a fixed order of sums, without atomics.  P and dS are rounded to the operand type before their second
// products (2^-9 relative in bf16, as the results are); sums and row terms are float32.
#include "bla_window.h"

namespace bla {
namespace {

template <typename T, int D> struct BwdGeo {
    static constexpr int CH = D * (int)sizeof(T) / 16, RPP = 256 / CH, NP = 64 / RPP, PE = 16 / (int)sizeof(T);
    static constexpr int QT = D == 128 ? 1 : 2;  // query tiles of a wave in the query pass
    static constexpr int KT = D == 128 ? 1 : 2;  // key tiles of a wave in the key pass
    static constexpr int BQ = 64 * QT, NK = 64 * KT;
    static constexpr int LD = dual_ld<T>(D), LN = nat_ld<T>(D);
};

// Query pass: as the forward kernel, S^T and dP^T tiles (rows: keys) whose dS^T is the operand of dQ^T = K^T dS^T.
template <typename T, int D>
__global__ void __launch_bounds__(256) window_bwd_q_kernel(WindowBwdArgs a)
{
    typedef BwdGeo<T, D> G;
    typedef typename Frag<T>::type F;
    constexpr int QT = G::QT, BUF = 64 * (G::LD + G::LN);
    __shared__ __attribute__((aligned(16))) T lds[2 * BUF];

    long long u = xcd_unit(blockIdx.x, a.q_per);
    if (u >= a.q_units) return;
    const int grp = a.H / a.Hkv;
    const int hg = (int)(u % grp);
    u /= grp;
    const int q0 = (int)(u % a.nqb) * G::BQ;
    u /= a.nqb;
    const int hk = (int)(u % a.Hkv), b = (int)(u / a.Hkv);
    const int h = hk * grp + hg;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const int len = a.lengths ? min(max(a.lengths[b], 0), a.L) : a.L;
    const int nq = min(G::BQ, len - q0);
    const size_t row0 = ((size_t)b * a.H + h) * a.L + q0;
    T* const out = (T*)a.dq + row0 * D;
    const int ch = tid % G::CH, lrow = tid / G::CH;
    if (nq <= 0) {
        const int rows = min(G::BQ, a.L - q0);
        for (int i = tid; i < rows * G::CH; i += 256) *(intx4*)(out + (size_t)i * G::PE) = intx4{0, 0, 0, 0};
        return;
    }
    const int lo = q0 - (a.W - 1) > 0 ? q0 - (a.W - 1) : 0;
    const int ns = min(a.S, lo), c = q0 - lo, total = ns + c + nq, sb = max(0, a.S - lo);
    const size_t kvrow = ((size_t)b * a.Hkv + hk) * a.L;
    const int ntile = (total + 63) / 64;

    intx4 kr[G::NP], vr[G::NP];
    auto load = [&](int tile) {
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            const int i = tile * 64 + ps * G::RPP + lrow;
            kr[ps] = vr[ps] = intx4{0, 0, 0, 0};
            if (i < total) {
                const size_t at = (kvrow + (i < ns ? i : lo + i - ns)) * D + ch * G::PE;
                kr[ps] = *(const intx4*)((const T*)a.k + at);
                vr[ps] = *(const intx4*)((const T*)a.v + at);
            }
        }
    };

    const int a0 = 16 * QT * wave;
    F qf[QT][D / 32], df[QT][D / 32];
    float lse2[QT], delta[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int i = min(a0 + 16 * qt + r, nq - 1);
        const size_t at = (row0 + i) * D;
        float x = 0.f;
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) {
            qf[qt][kb] = ld_nat((const T*)a.q + at, kb, g);
            df[qt][kb] = ld_nat((const T*)a.dO + at, kb, g);
            const F of = ld_nat((const T*)a.o + at, kb, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) x = __builtin_fmaf((float)df[qt][kb][e], (float)of[e], x);
        }
        delta[qt] = rows_sum(x);
        lse2[qt] = a.lse[row0 + i] * kLog2e;
        if (g == 0 && a0 + 16 * qt + r < nq) a.delta[row0 + i] = delta[qt];
    }
    const float sc = a.scale * kLog2e;
    floatx4 acc[QT][D / 16];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt)
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) acc[qt][dt] = zero4();

    const int aend = min(a0 + 16 * QT, nq) - 1;
    load(0);
    for (int t = 0; t < ntile; ++t) {
        T *sK = lds + (t & 1) * BUF, *sV = sK + 64 * G::LD;
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            const int i = ps * G::RPP + lrow;
            *(intx4*)(sK + i * G::LD + dual_col<T>(i, ch * G::PE)) = kr[ps];
            *(intx4*)(sV + i * G::LN + ch * G::PE) = vr[ps];
        }
        __syncthreads();
        if (t + 1 < ntile) load(t + 1);
        const int j0 = t * 64 - ns, j1 = j0 + 63;
        if (a0 >= nq || j0 > c + aend || (j0 >= sb && j1 <= c + a0 - a.W)) continue;
        const bool whole = j1 < 0 || (j0 >= 0 && j1 <= c + a0 && (c + aend - j0 < a.W || j1 < sb));
#pragma unroll
        for (int kb2 = 0; kb2 < 2; ++kb2) {
            floatx4 s[QT][2], dp[QT][2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) s[qt][kt] = dp[qt][kt] = zero4();
#pragma unroll
                for (int kb = 0; kb < D / 32; ++kb) {
                    const F kf = ld_nat_dual(sK, G::LD, 32 * kb2 + 16 * kt, kb, g, r);
                    const F vf = ld_nat(sV + (32 * kb2 + 16 * kt + r) * G::LN, kb, g);
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) {
                        s[qt][kt] = mma(kf, qf[qt][kb], s[qt][kt]);
                        dp[qt][kt] = mma(vf, df[qt][kb], dp[qt][kt]);
                    }
                }
            }
            F sf[QT];
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                const int ca = c + a0 + 16 * qt + r;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float p = exp2_fast(__builtin_fmaf(s[qt][kt][e], sc, -lse2[qt])) * (dp[qt][kt][e] - delta[qt]);
                        if (!whole) {
                            const int j = j0 + 32 * kb2 + 16 * kt + 4 * g + e;
                            p = (j < 0) | ((j <= ca) & ((ca - j < a.W) | (j < sb))) ? p : 0.f;
                        }
                        s[qt][kt][e] = p;
                    }
                sf[qt] = frag_from_acc<T>(s[qt][0], s[qt][1]);
            }
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                const F kf = ld_red_dual(sK, G::LD, 16 * dt, kb2, g, r);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) acc[qt][dt] = mma(kf, sf[qt], acc[qt][dt]);
            }
        }
    }
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int i = a0 + 16 * qt + r;
        if (i >= min(G::BQ, a.L - q0)) continue;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt)
            st4(out + (size_t)i * D + 16 * dt + 4 * g, i < nq ? acc[qt][dt] * a.scale : zero4());
    }
}

// Key pass.  Wave w owns 16 KT keys: their K and V are operands in registers for the whole walk, and S = Q K^T and
// dP = dO V^T (accumulator rows: queries) give P and dS as operands of dV^T = dO^T P and dK^T = Q^T dS.  The walk goes over the
// heads of the group and the 64-query tiles that see the block.  Keys that are sinks are seen by every later
// query, so the blocks that hold some are split over the queries into parts of about a plain block's work, whose
// float32 results window_bwd_sum_kernel adds up in order.
template <typename T, int D>
__global__ void __launch_bounds__(256) window_bwd_k_kernel(WindowBwdArgs a)
{
    typedef BwdGeo<T, D> G;
    typedef typename Frag<T>::type F;
    constexpr int KT = G::KT, BUF = 64 * 2 * G::LD;
    __shared__ __attribute__((aligned(16))) T lds[2 * BUF];
    __shared__ __attribute__((aligned(16))) float sStat[2][2][64];

    long long u = xcd_unit(blockIdx.x, a.k_per);
    if (u >= a.k_units) return;
    const int grp = a.H / a.Hkv;
    const int jobs = a.nsb * a.ssplit + a.nkb - a.nsb;  // of one key head
    const int job = (int)(u % jobs);
    u /= jobs;
    const int hk = (int)(u % a.Hkv), b = (int)(u / a.Hkv);
    const bool sink = job < a.nsb * a.ssplit;
    const int nb = sink ? job / a.ssplit : job - a.nsb * a.ssplit + a.nsb, part = sink ? job % a.ssplit : 0;
    const int n0 = nb * G::NK;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const int len = a.lengths ? min(max(a.lengths[b], 0), a.L) : a.L;
    const size_t kvrow = ((size_t)b * a.Hkv + hk) * a.L;
    const int ch = tid % G::CH, lrow = tid / G::CH;

    // 64-query tiles of the walk, from query n0 on
    const int qend = sink ? len : (int)min((long long)len, (long long)n0 + G::NK - 1 + a.W);
    int tb = 0, te = qend > n0 ? (qend - n0 + 63) / 64 : 0;
    if (sink) {
        const int each = (te + a.ssplit - 1) / a.ssplit;
        tb = part * each;
        te = min(te, tb + each);
    }
    const int nt = max(0, te - tb), steps = nt * grp;

    const int k0 = n0 + 16 * KT * wave;  // the wave's first key
    F kf[KT][D / 32], vf[KT][D / 32];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        const size_t at = (kvrow + min(k0 + 16 * kt + r, a.L - 1)) * D;
        const bool in = k0 + 16 * kt + r < len;
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) {
            kf[kt][kb] = in ? ld_nat((const T*)a.k + at, kb, g) : zero_frag<T>();
            vf[kt][kb] = in ? ld_nat((const T*)a.v + at, kb, g) : zero_frag<T>();
        }
    }
    floatx4 dk[KT][D / 16], dv[KT][D / 16];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) dk[kt][dt] = dv[kt][dt] = zero4();
    const float sc = a.scale * kLog2e;

    intx4 qr[G::NP], dr[G::NP];
    float st = 0.f;
    auto load = [&](int step) {
        const int hg = step / nt, q0 = n0 + 64 * (tb + step % nt);
        const size_t row0 = ((size_t)b * a.H + hk * grp + hg) * a.L + q0;
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            const int i = ps * G::RPP + lrow;
            qr[ps] = dr[ps] = intx4{0, 0, 0, 0};
            if (q0 + i < len) {
                const size_t at = (row0 + i) * D + ch * G::PE;
                qr[ps] = *(const intx4*)((const T*)a.q + at);
                dr[ps] = *(const intx4*)((const T*)a.dO + at);
            }
        }
        if (tid < 128) {
            const int i = tid & 63;
            st = q0 + i < len ? (tid < 64 ? a.lse[row0 + i] * kLog2e : a.delta[row0 + i]) : 0.f;
        }
    };

    if (steps > 0) load(0);
    for (int step = 0; step < steps; ++step) {
        T *sQ = lds + (step & 1) * BUF, *sD = sQ + 64 * G::LD;
        float(*stat)[64] = sStat[step & 1];
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            const int i = ps * G::RPP + lrow, at = i * G::LD + dual_col<T>(i, ch * G::PE);
            *(intx4*)(sQ + at) = qr[ps];
            *(intx4*)(sD + at) = dr[ps];
        }
        if (tid < 128) stat[tid >> 6][tid & 63] = st;
        __syncthreads();
        if (step + 1 < steps) load(step + 1);
        const int q0 = n0 + 64 * (tb + step % nt), q1 = min(q0 + 63, len - 1);
        const int kend = k0 + 16 * KT - 1;
        if (k0 > q1 || (k0 >= a.S && q0 - kend >= a.W)) continue;
        const bool whole = kend <= q0 && q0 + 63 < len && (q0 + 63 - k0 < a.W || kend < a.S);
#pragma unroll
        for (int kb2 = 0; kb2 < 2; ++kb2) {
            floatx4 s[KT][2], dp[KT][2];
#pragma unroll
            for (int qt = 0; qt < 2; ++qt) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) s[kt][qt] = dp[kt][qt] = zero4();
#pragma unroll
                for (int kb = 0; kb < D / 32; ++kb) {
                    const F qf = ld_nat_dual(sQ, G::LD, 32 * kb2 + 16 * qt, kb, g, r);
                    const F df = ld_nat_dual(sD, G::LD, 32 * kb2 + 16 * qt, kb, g, r);
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) {
                        s[kt][qt] = mma(qf, kf[kt][kb], s[kt][qt]);
                        dp[kt][qt] = mma(df, vf[kt][kb], dp[kt][qt]);
                    }
                }
            }
            F pf[KT], sf[KT];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
                for (int qt = 0; qt < 2; ++qt) {
                    const floatx4 lse2 = ld4f(stat[0] + 32 * kb2 + 16 * qt + 4 * g);
                    const floatx4 delta = ld4f(stat[1] + 32 * kb2 + 16 * qt + 4 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float p = exp2_fast(__builtin_fmaf(s[kt][qt][e], sc, -lse2[e]));
                        if (!whole) {
                            const int q = q0 + 32 * kb2 + 16 * qt + 4 * g + e, j = k0 + 16 * kt + r;
                            p = (q < len) & (j <= q) & ((q - j < a.W) | (j < a.S)) ? p : 0.f;
                        }
                        s[kt][qt][e] = p;
                        dp[kt][qt][e] = p * (dp[kt][qt][e] - delta[e]);
                    }
                }
                pf[kt] = frag_from_acc<T>(s[kt][0], s[kt][1]);
                sf[kt] = frag_from_acc<T>(dp[kt][0], dp[kt][1]);
            }
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                const F df = ld_red_dual(sD, G::LD, 16 * dt, kb2, g, r), qf = ld_red_dual(sQ, G::LD, 16 * dt, kb2, g, r);
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    dv[kt][dt] = mma(df, pf[kt], dv[kt][dt]);
                    dk[kt][dt] = mma(qf, sf[kt], dk[kt][dt]);
                }
            }
        }
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        const int key = k0 + 16 * kt + r;
        if (sink) {
            float* to = a.part + ((((size_t)part * a.B + b) * a.Hkv + hk) * a.nsb * G::NK + key) * 2 * D;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                st4f(to + 16 * dt + 4 * g, dk[kt][dt]);
                st4f(to + D + 16 * dt + 4 * g, dv[kt][dt]);
            }
        } else if (key < a.L) {
            const size_t at = (kvrow + key) * D;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                st4((T*)a.dk + at + 16 * dt + 4 * g, dk[kt][dt] * a.scale);
                st4((T*)a.dv + at + 16 * dt + 4 * g, dv[kt][dt]);
            }
        }
    }
}

// dk and dv of the keys of the blocks with sinks: the parts, added in order.
template <typename T, int D> __global__ void __launch_bounds__(256) window_bwd_sum_kernel(WindowBwdArgs a)
{
    const int keys = a.nsb * BwdGeo<T, D>::NK;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int c = 4 * (int)(i % (2 * D / 4));
    const long long row = i / (2 * D / 4);  // (b, hk, key)
    if (row >= (long long)a.B * a.Hkv * keys) return;
    const int key = (int)(row % keys);
    if (key >= a.L) return;
    floatx4 x = zero4();
    for (int s = 0; s < a.ssplit; ++s) x += ld4f(a.part + ((size_t)s * a.B * a.Hkv * keys + row) * 2 * D + c);
    const size_t at = ((size_t)(row / keys) * a.L + key) * D;
    if (c < D)
        st4((T*)a.dk + at + c, x * a.scale);
    else
        st4((T*)a.dv + at + c - D, x);
}

template <typename T, int D> hipError_t backward_d(const WindowBwdArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((window_bwd_q_kernel<T, D>), dim3((unsigned)(8 * a.q_per)), dim3(256), 0, s, a);
    hipLaunchKernelGGL((window_bwd_k_kernel<T, D>), dim3((unsigned)(8 * a.k_per)), dim3(256), 0, s, a);
    if (a.nsb > 0) {
        const long long n = (long long)a.B * a.Hkv * a.nsb * BwdGeo<T, D>::NK * (2 * D / 4);
        hipLaunchKernelGGL((window_bwd_sum_kernel<T, D>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace

int window_bwd_keys(int, int D) { return D == 128 ? BwdGeo<bf16, 128>::NK : BwdGeo<bf16, 64>::NK; }
int window_bwd_queries(int, int D) { return D == 128 ? BwdGeo<bf16, 128>::BQ : BwdGeo<bf16, 64>::BQ; }

hipError_t launch_window_backward(int bf16_io, int D, const WindowBwdArgs& a, hipStream_t s)
{
    if (bf16_io) {
        if (D == 32) return backward_d<bf16, 32>(a, s);
        if (D == 64) return backward_d<bf16, 64>(a, s);
        if (D == 128) return backward_d<bf16, 128>(a, s);
    } else {
        if (D == 32) return backward_d<float, 32>(a, s);
        if (D == 64) return backward_d<float, 64>(a, s);
        if (D == 128) return backward_d<float, 128>(a, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace bla
