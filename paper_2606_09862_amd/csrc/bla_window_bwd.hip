// Backward pass of window attention (bla_window_backward).
//
// With P = exp(scale q k - lse) on the visible pairs and delta_i = sum_c dO_ic o_ic:
//   dS = P (dO v^T - delta),   dq = scale dS k,   dk = scale dS^T q,   dv = P^T dO.
// Two passes recompute P from lse, one per query block (dq, and delta for the other) and one per key block (dk, dv, summed over the
// heads that share the key head and over the queries whose windows reach the block; the sinks' other queries have
// workgroups of their own), so that every gradient has a fixed order of sums, without atomics.  P and dS are rounded to the operand type before their second
// products (2^-8 relative at most in bf16, as the results are); sums and row terms are float32.
#include <algorithm>

#include "bla_window.h"

namespace bla {
namespace {

// Tiles of 16 queries (query pass) or keys (key pass) that a wave owns: two where the registers hold them, so that each fragment read
// from LDS serves two products.
template <typename T, int D> constexpr int bwd_tiles() { return D == 128 ? 1 : 2; }
// Four waves to a workgroup: with eight one workgroup fills a compute unit and its waves wait for each other at every tile (128 x 4096 tokens,
// d = 64, window 511: query pass 229 us with eight waves, 167 with four; key pass 310 and 259).
template <typename T, int D> struct BwdGeo {
    static constexpr int NT = 256, PE = 16 / (int)sizeof(T), CH = D / PE, RPP = NT / CH, NP = 64 / RPP;
    static constexpr int XT = bwd_tiles<T, D>(), NB = 64 * XT;
    static constexpr int LD = nat_ld<T>(D);
};

// Query pass: as the forward kernel, S^T and dP^T tiles (rows: keys) whose dS^T is the operand of dQ^T = K^T dS^T.
// Bound: issue, as the forward kernel (8 x 16 heads x 4096 queries, four heads to a key head, d = 64, window 511, bf16: 160-168 us).
//
// EXACT: delta is formed from outputs that were rounded to bf16, which adds 2^-9 |dO| |o| or so to each dP - delta.  That is lost among dS's own
// rounding where many keys share a row, and as large as it where few do.  The sum of the dS of a row is what delta is off by (the exact
// ones sum to zero), so the row's dq is put right by that sum times sum_j P_j k_j, a third product, and delta goes on to the key pass without the error.
template <typename T, int D, bool EXACT>
__global__ void __launch_bounds__(256) window_bwd_q_kernel(WindowBwdArgs a)
{
    typedef BwdGeo<T, D> G;
    typedef typename Frag<T>::type F;
    constexpr int QT = G::XT, BUF = 64 * 2 * G::LD;
    __shared__ __attribute__((aligned(16))) T lds[2 * BUF];

    long long u = xcd_unit(blockIdx.x, a.q_per);
    if (u >= a.q_units) return;
    const int grp = a.H / a.Hkv;
    const int hg = (int)(u % grp);
    u /= grp;
    const int q0 = (int)(u % a.nqb) * G::NB;
    u /= a.nqb;
    const int hk = (int)(u % a.Hkv), b = (int)(u / a.Hkv);
    const int h = hk * grp + hg;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const int len = a.lengths ? min(max(a.lengths[b], 0), a.L) : a.L;
    const int nq = min(G::NB, len - q0);
    const size_t row0 = ((size_t)b * a.H + h) * a.L + q0;
    T* const out = (T*)a.dq + row0 * D;
    const int ch = tid % G::CH, lrow = tid / G::CH;
    if (nq <= 0) {
        const int rows = min(G::NB, a.L - q0);
        for (int i = tid; i < rows * G::CH; i += G::NT) *(intx4*)(out + (size_t)i * G::PE) = intx4{0, 0, 0, 0};
        return;
    }
    const int lo = q0 - (a.W - 1) > 0 ? q0 - (a.W - 1) : 0;
    const int ns = min(a.S, lo), c = q0 - lo, total = ns + c + nq, sb = max(0, a.S - lo);
    const size_t kvrow = ((size_t)b * a.Hkv + hk) * a.L;
    const T *kp = (const T*)a.k + kvrow * D + ch * G::PE, *vp = (const T*)a.v + kvrow * D + ch * G::PE;
    const int ntile = (total + 63) / 64;

    intx4 kr[G::NP], vr[G::NP];
    auto load = [&](int tile) {
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            const int i = min(tile * 64 + ps * G::RPP + lrow, total - 1);
            const size_t at = (size_t)(i < ns ? i : lo + i - ns) * D;
            kr[ps] = *(const intx4*)(kp + at);
            vr[ps] = *(const intx4*)(vp + at);
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
        if (!EXACT && g == 0 && a0 + 16 * qt + r < nq) a.delta[row0 + i] = delta[qt];
    }
    const float sc = a.scale * kLog2e;
    floatx4 acc[QT][D / 16], pk[EXACT ? QT : 1][D / 16];
    float off[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        off[qt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) acc[qt][dt] = pk[EXACT ? qt : 0][dt] = zero4();
    }

    const int aend = min(a0 + 16 * QT, nq) - 1;
    load(0);
    for (int t = 0; t < ntile; ++t) {
        T *sK = lds + (t & 1) * BUF, *sV = sK + 64 * G::LD;
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            const int i = ps * G::RPP + lrow;
            *(intx4*)(sK + i * G::LD + ch * G::PE) = kr[ps];
            *(intx4*)(sV + i * G::LD + ch * G::PE) = vr[ps];
        }
        __syncthreads();
        if (t + 1 < ntile) load(t + 1);
        if (a0 >= nq) continue;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int i0 = t * 64 - ns + 32 * hf, i1 = i0 + 31;  // window keys (negative: sinks)
            if (i0 > c + aend || (i0 >= sb && i1 <= c + a0 - a.W)) continue;
            floatx4 s[QT][2], dp[QT][2];  // scores, then dS; dP, then P where it is wanted
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) s[qt][kt] = dp[qt][kt] = zero4();
#pragma unroll
                for (int kb = 0; kb < D / 32; ++kb) {
                    const F kf = ld_nat(sK + (32 * hf + 16 * kt + r) * G::LD, kb, g);
                    const F vf = ld_nat(sV + (32 * hf + 16 * kt + r) * G::LD, kb, g);
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) {
                        s[qt][kt] = mma(kf, qf[qt][kb], s[qt][kt]);
                        dp[qt][kt] = mma(vf, df[qt][kb], dp[qt][kt]);
                    }
                }
            }
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = exp2_fast(__builtin_fmaf(s[qt][kt][e], sc, -lse2[qt]));
                        s[qt][kt][e] = p * (dp[qt][kt][e] - delta[qt]);
                        dp[qt][kt][e] = p;
                    }
            if (i1 > c + a0 || (i0 <= c + aend - a.W && i1 >= sb)) {  // some pair is not visible (selects without branches, as in the forward kernel)
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) {
                    const int jhi = c + a0 + 16 * qt + r, jlo = jhi - (a.W - 1), j = i0 + 4 * g;
                    if (i0 >= sb) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const bool seen = (unsigned)(j + 16 * (e >> 2) + (e & 3) - jlo) < (unsigned)a.W;
                            s[qt][e >> 2][e & 3] = seen ? s[qt][e >> 2][e & 3] : 0.f;
                            if (EXACT) dp[qt][e >> 2][e & 3] = seen ? dp[qt][e >> 2][e & 3] : 0.f;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int k = j + 16 * (e >> 2) + (e & 3);
                            const bool seen = (k <= jhi) & ((k >= jlo) | (k < sb));
                            s[qt][e >> 2][e & 3] = seen ? s[qt][e >> 2][e & 3] : 0.f;
                            if (EXACT) dp[qt][e >> 2][e & 3] = seen ? dp[qt][e >> 2][e & 3] : 0.f;
                        }
                    }
                }
            }
            F sf[QT], pf[QT];
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                sf[qt] = frag_from_acc<T>(s[qt][0], s[qt][1]);
                if (EXACT) {
                    pf[qt] = frag_from_acc<T>(dp[qt][0], dp[qt][1]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) off[qt] += s[qt][e >> 2][e & 3];
                }
            }
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                const F kf = ld_red(sK, G::LD, 16 * dt, hf, g, r);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) {
                    acc[qt][dt] = mma(kf, sf[qt], acc[qt][dt]);
                    if (EXACT) pk[qt][dt] = mma(kf, pf[qt], pk[qt][dt]);
                }
            }
        }
    }
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int i = a0 + 16 * qt + r;
        if (EXACT) {
            off[qt] = rows_sum(off[qt]);
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) acc[qt][dt] -= off[qt] * pk[qt][dt];
            if (g == 0 && i < nq) a.delta[row0 + i] = delta[qt] + off[qt];
        }
        if (i >= min(G::NB, a.L - q0)) continue;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt)
            st4(out + (size_t)i * D + 16 * dt + 4 * g, i < nq ? acc[qt][dt] * a.scale : zero4());
    }
}

// The pairs of sinks and the queries that see them from beyond their windows.  A wave takes 16 sinks and every so-maniest 32 queries of every head of
// the group, on its own: rows of Q and dO come from memory as operands of S and dP, and through LDS that only the wave touches
// as the transposed operands of dV^T and dK^T.  The four waves are added up in LDS, a workgroup writes one part.  Bound: the bytes of Q
// and dO (128 x 4096 tokens at d = 64, window 511, 4 sinks: 117 MB).  As part of the key walk these queries took a fifth of the
// workgroups for one wave's work each: 251 us with them, 204 without.
template <typename T, int D> __device__ __forceinline__ void window_bwd_sinks(const WindowBwdArgs& a, unsigned u, char* raw)
{
    typedef typename Frag<T>::type F;
    constexpr int LD = nat_ld<T>(D), LO = D + 4;
    constexpr size_t QB = sizeof(T) * 4 * 2 * 32 * LD, OB = sizeof(float) * 4 * 16 * LO;
    static_assert(QB <= sizeof(T) * 256 * BwdGeo<T, D>::LD && OB <= QB, "the key kernel's LDS");
    const int part = (int)(u % (unsigned)a.ssplit);
    u /= (unsigned)a.ssplit;
    const int nst = (a.ns + 15) / 16, st = (int)(u % (unsigned)nst);
    u /= (unsigned)nst;
    const int hk = (int)(u % (unsigned)a.Hkv), b = (int)(u / (unsigned)a.Hkv);
    const int grp = a.H / a.Hkv;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const int len = a.lengths ? min(max(a.lengths[b], 0), a.L) : a.L;
    const int j = 16 * st + r;                                                // the lane's sink
    const long long first = (long long)16 * st + a.W;                        // the first query past a window that holds one
    const int q_first = (int)min(first, (long long)len), blocks = (len - q_first + 31) / 32;

    F kf[D / 32], vf[D / 32];
    {
        const size_t at = (((size_t)b * a.Hkv + hk) * a.L + min(j, a.L - 1)) * D;
        const bool in = j < a.ns && j < len;
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) {
            kf[kb] = in ? ld_nat((const T*)a.k + at, kb, g) : zero_frag<T>();
            vf[kb] = in ? ld_nat((const T*)a.v + at, kb, g) : zero_frag<T>();
        }
    }
    // the lane's sink is seen from beyond its window by the queries from j + W on
    const int q_sink = j < a.ns && j < len ? (int)min((long long)j + a.W, (long long)len) : len;
    floatx4 dk[D / 16], dv[D / 16];
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) dk[dt] = dv[dt] = zero4();
    const float sc = a.scale * kLog2e;
    T *sQ = (T*)raw + wave * 2 * 32 * LD, *sD = sQ + 32 * LD;

    for (long long it = part * 4 + wave; it < (long long)grp * blocks; it += a.ssplit * 4) {
        const int hg = (int)(it / blocks), q0 = q_first + 32 * (int)(it % blocks);
        const size_t row0 = ((size_t)b * a.H + hk * grp + hg) * a.L;
        floatx4 s[2], dp[2];
#pragma unroll
        for (int qt = 0; qt < 2; ++qt) {
            const size_t at = (row0 + min(q0 + 16 * qt + r, len - 1)) * D;
            s[qt] = dp[qt] = zero4();
#pragma unroll
            for (int kb = 0; kb < D / 32; ++kb) {
                const F qf = ld_nat((const T*)a.q + at, kb, g), df = ld_nat((const T*)a.dO + at, kb, g);
                *(F*)(sQ + (16 * qt + r) * LD + 32 * kb + 8 * g) = qf;
                *(F*)(sD + (16 * qt + r) * LD + 32 * kb + 8 * g) = df;
                s[qt] = mma(qf, kf[kb], s[qt]);
                dp[qt] = mma(df, vf[kb], dp[qt]);
            }
        }
#pragma unroll
        for (int qt = 0; qt < 2; ++qt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int q = q0 + 16 * qt + 4 * g + e;
                const size_t at = row0 + min(q, len - 1);
                const float p = exp2_fast(__builtin_fmaf(s[qt][e], sc, -a.lse[at] * kLog2e));
                const bool seen = (q >= q_sink) & (q < len);  // no branch: see the forward kernel's masks
                s[qt][e] = seen ? p : 0.f;
                dp[qt][e] = seen ? p * (dp[qt][e] - a.delta[at]) : 0.f;
            }
        const F pf = frag_from_acc<T>(s[0], s[1]), sf = frag_from_acc<T>(dp[0], dp[1]);
        // the wave's own stores above, read by its other lanes (LDS serves a wave in order)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
            dv[dt] = mma(ld_red(sD, LD, 16 * dt, 0, g, r), pf, dv[dt]);
            dk[dt] = mma(ld_red(sQ, LD, 16 * dt, 0, g, r), sf, dk[dt]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    float* sO = (float*)raw;
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st4f(sO + (wave * 16 + r) * LO + 16 * dt + 4 * g, which ? dv[dt] : dk[dt]);
        __syncthreads();
        for (int i = tid; i < 16 * (D / 4); i += 256) {
            const int key = i / (D / 4), c = 4 * (i % (D / 4));
            if (16 * st + key >= a.ns) continue;
            floatx4 x = ld4f(sO + key * LO + c);
#pragma unroll
            for (int w = 1; w < 4; ++w) x += ld4f(sO + (w * 16 + key) * LO + c);
            st4f(a.part + (((((size_t)part * a.B + b) * a.Hkv + hk) * a.ns + 16 * st + key) * 2 + which) * D + c, x);
        }
    }
}

// Key pass.  Wave w owns 16 KT keys: their K and V are operands in registers for the whole walk, and S = Q K^T and
// dP = dO V^T (accumulator rows: queries) give P and dS as operands of dV^T = dO^T P and dK^T = Q^T dS.  The walk goes over the
// heads of the group and the 64-query tiles whose windows hold keys of the block.  Later queries see sinks as well: those pairs
// are window_bwd_sinks', and the sinks' gradients go out in float32 for window_bwd_sum_kernel to add up.
// Bound: issue (the query pass's shape: 203-215 us of keys; with the sinks' workgroups 221-235, which took 31 us in a launch of their own and 340
// us in all where they were spread among the keys').
template <typename T, int D>
__global__ void __launch_bounds__(256) window_bwd_k_kernel(WindowBwdArgs a)
{
    typedef BwdGeo<T, D> G;
    typedef typename Frag<T>::type F;
    constexpr int KT = G::XT, BUF = 64 * 2 * G::LD;
    __shared__ __attribute__((aligned(16))) T lds[2 * BUF];
    __shared__ __attribute__((aligned(16))) float sStat[2][2][64];

    if (blockIdx.x >= 8 * a.k_per) {  // last: they fill the compute units that run out of keys
        window_bwd_sinks<T, D>(a, blockIdx.x - (unsigned)(8 * a.k_per), (char*)lds);
        return;
    }
    long long u = xcd_unit(blockIdx.x, a.k_per);
    if (u >= a.k_units) return;
    const int grp = a.H / a.Hkv;
    const int nb = (int)(u % a.nkb);
    u /= a.nkb;
    const int hk = (int)(u % a.Hkv), b = (int)(u / a.Hkv);
    const int n0 = nb * G::NB;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const int len = a.lengths ? min(max(a.lengths[b], 0), a.L) : a.L;
    const size_t kvrow = ((size_t)b * a.Hkv + hk) * a.L;
    const int ch = tid % G::CH, lrow = tid / G::CH;

    // 64-query tiles of the walk, from query n0 on
    const int qend = (int)min((long long)len, (long long)n0 + G::NB - 1 + a.W);
    const int nt = qend > n0 ? (qend - n0 + 63) / 64 : 0;

    const int k0 = n0 + 16 * KT * wave, kend = k0 + 16 * KT - 1;  // the wave's keys
    F kf[KT][D / 32], vf[KT][D / 32];
    unsigned span[KT];                                            // key j is seen by the queries j .. j + span - 1
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        const int j = k0 + 16 * kt + r;
        const size_t at = (kvrow + min(j, a.L - 1)) * D;
        const bool in = j < len;
        span[kt] = in ? (unsigned)min(len - j, a.W) : 0u;
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
    const T *qp = (const T*)a.q + ch * G::PE, *dp_ = (const T*)a.dO + ch * G::PE;
    auto load = [&](int hg, int t) {  // queries past the row's last repeat it: the masks hide them
        const size_t row0 = ((size_t)b * a.H + hk * grp + hg) * a.L;
        const int q0 = n0 + 64 * t;
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            const size_t at = (row0 + min(q0 + ps * G::RPP + lrow, len - 1)) * D;
            qr[ps] = *(const intx4*)(qp + at);
            dr[ps] = *(const intx4*)(dp_ + at);
        }
        if (tid < 128) {
            const size_t at = row0 + min(q0 + (tid & 63), len - 1);
            st = tid < 64 ? a.lse[at] * kLog2e : a.delta[at];
        }
    };

    if (nt > 0) load(0, 0);
    int buf = 0;
    for (int hg = 0; hg < grp; ++hg)
        for (int t = 0; t < nt; ++t, buf ^= 1) {
            T *sQ = lds + buf * BUF, *sD = sQ + 64 * G::LD;
            float(*stat)[64] = sStat[buf];
#pragma unroll
            for (int ps = 0; ps < G::NP; ++ps) {
                    const int i = ps * G::RPP + lrow, at = i * G::LD + ch * G::PE;
                *(intx4*)(sQ + at) = qr[ps];
                *(intx4*)(sD + at) = dr[ps];
            }
            if (tid < 128) stat[tid >> 6][tid & 63] = st;
            __syncthreads();
            if (t + 1 < nt)
                load(hg, t + 1);
            else if (hg + 1 < grp)
                load(hg + 1, 0);
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const int q0 = n0 + 64 * t + 32 * hf, q1 = q0 + 31;
                if (q0 >= len || k0 > q1 || q0 - kend >= a.W) continue;
                floatx4 s[KT][2], dp[KT][2];
#pragma unroll
                for (int qt = 0; qt < 2; ++qt) {
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) s[kt][qt] = dp[kt][qt] = zero4();
#pragma unroll
                    for (int kb = 0; kb < D / 32; ++kb) {
                        const F qf = ld_nat(sQ + (32 * hf + 16 * qt + r) * G::LD, kb, g);
                        const F df = ld_nat(sD + (32 * hf + 16 * qt + r) * G::LD, kb, g);
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt) {
                            s[kt][qt] = mma(qf, kf[kt][kb], s[kt][qt]);
                            dp[kt][qt] = mma(df, vf[kt][kb], dp[kt][qt]);
                        }
                    }
                }
#pragma unroll
                for (int qt = 0; qt < 2; ++qt) {
                    const floatx4 lse2 = ld4f(stat[0] + 32 * hf + 16 * qt + 4 * g);
                    const floatx4 delta = ld4f(stat[1] + 32 * hf + 16 * qt + 4 * g);
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[kt][qt][e] = exp2_fast(__builtin_fmaf(s[kt][qt][e], sc, -lse2[e]));
                            dp[kt][qt][e] = s[kt][qt][e] * (dp[kt][qt][e] - delta[e]);
                        }
                }
                if (kend > q0 || q1 >= len || q1 - k0 >= a.W) {  // some pair is not visible (selects without branches, as in the forward kernel)
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) {
                        const int q = q0 + 4 * g - (k0 + 16 * kt + r);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const bool seen = (unsigned)(q + 16 * (e >> 2) + (e & 3)) < span[kt];
                            s[kt][e >> 2][e & 3] = seen ? s[kt][e >> 2][e & 3] : 0.f;
                            dp[kt][e >> 2][e & 3] = seen ? dp[kt][e >> 2][e & 3] : 0.f;
                        }
                    }
                }
                F pf[KT], sf[KT];
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    pf[kt] = frag_from_acc<T>(s[kt][0], s[kt][1]);
                    sf[kt] = frag_from_acc<T>(dp[kt][0], dp[kt][1]);
                }
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) {
                    const F df = ld_red(sD, G::LD, 16 * dt, hf, g, r), qf = ld_red(sQ, G::LD, 16 * dt, hf, g, r);
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
        if (key < a.S && key < a.L) {
            float* to = a.near + (((size_t)b * a.Hkv + hk) * a.ns + key) * 2 * D;
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

// dk and dv of the sinks: the key kernel's and the parts, added in order.
template <typename T, int D> __global__ void __launch_bounds__(256) window_bwd_sum_kernel(WindowBwdArgs a)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int c = 4 * (int)(i % (2 * D / 4));
    const long long row = i / (2 * D / 4), rows = (long long)a.B * a.Hkv * a.ns;  // (b, hk, key)
    if (row >= rows) return;
    floatx4 x = ld4f(a.near + row * 2 * D + c);
#pragma unroll 8
    for (int s = 0; s < a.ssplit; ++s) x += ld4f(a.part + ((size_t)s * rows + row) * 2 * D + c);
    const size_t at = ((size_t)(row / a.ns) * a.L + row % a.ns) * D;
    if (c < D)
        st4((T*)a.dk + at + c, x * a.scale);
    else
        st4((T*)a.dv + at + c - D, x);
}

// Most keys of a row for which delta's error is taken out in the query pass (bf16).  Relative error of dq without it (dk a little less), at d = 64: sequences of
// 16 tokens 0.0032, 8 keys a row 0.0030, 16 keys 0.0028, 64 keys 0.0026, 511 keys 0.0025; with it 0.0024 everywhere (dS and dq rounded; dq alone: 0.0017).
// Time without it and with it, 8 x 16 heads x 4096 tokens on 4 key heads: d = 64, 8 keys 131 and 137 us, 64 keys 173 and 185; d = 32, 64 keys 100 and 112; d =
// 64, 515 keys 340 and 390, which is why long windows go without.
constexpr int kExactKeys = 64;

template <typename T, int D> hipError_t backward_d(const WindowBwdArgs& a, hipStream_t s)
{
    typedef BwdGeo<T, D> G;
    if (std::min((long long)a.W + a.S, (long long)a.L) <= kExactKeys)
        hipLaunchKernelGGL((window_bwd_q_kernel<T, D, sizeof(T) == 2>), dim3((unsigned)(8 * a.q_per)), dim3(G::NT), 0, s, a);
    else
        hipLaunchKernelGGL((window_bwd_q_kernel<T, D, false>), dim3((unsigned)(8 * a.q_per)), dim3(G::NT), 0, s, a);
    hipLaunchKernelGGL((window_bwd_k_kernel<T, D>), dim3((unsigned)(8 * a.k_per) + a.s_units), dim3(G::NT), 0, s, a);
    if (a.ns > 0) {
        const long long n = (long long)a.B * a.Hkv * a.ns * (2 * D / 4);
        hipLaunchKernelGGL((window_bwd_sum_kernel<T, D>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace

int window_bwd_block(int D) { return D == 128 ? BwdGeo<bf16, 128>::NB : BwdGeo<bf16, 64>::NB; }

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
