// Backward pass of the selective scan (bla_ssm_backward).
//
// In a chunk, with L_tu = e^{s_t - s_u} for u <= t, Q = dY X^T, K = C B^T, the entering state h and the gradient g of the
// leaving one:
//   dx_u = dt_u (sum_t L K dy_t + e^{s_c - s_u} g^T B_u) + D dy_u
//   dC_t = sum_u L Q dt_u B_u + e^{s_t} h dy_t                (summed over the heads of the group)
//   dB_u = dt_u (sum_t L Q C_t + e^{s_c - s_u} g x_u)         (likewise)
// and through the exponents, with M = L K Q:
//   p_u   = sum_t M_tu + e^{s_c - s_u} B_u . g x_u            (the gradient of dt_u as a factor)
//   ds_t  = sum_u M_tu dt_u + e^{s_t} C_t . h dy_t - dt_t p_t
//   da_t  = sum_{t' >= t} ds_t' + sum_u dt_u e^{s_c - s_u} B_u . g x_u + e^{s_c} <g, h>
//   ddt_t = p_t + A da_t,   dA = sum_t dt_t da_t,   dD = sum_t x_t . dy_t.
// Two walks over the chunks leave h and g of every chunk in the workspace; then the chunks are independent.  ddt, dA, dD and the
// state's gradient are float32 results and take no operand rounding: their products of bf16 inputs are exact,
// and h and g enter them as sums of three bf16 (Split).  In da_t the M_t'u of u >= t are in the rows' sums and in the columns' and cancel, so both
// sum the same float32 values in float64 (float32 sums left dA off by up to thirty times what a float32 recurrence leaves).  dx, dB, dC take weights in the operand type.
#include "bla_ssm.h"

namespace bla {
namespace {

// States entering the chunks (from B, x), and in the second half of the grid the gradients of the states leaving them (`back`: from C, dy, chunks in
// reverse): the two walks are independent, and either alone leaves half of the device idle.  The columns d of a
// state are independent too, so a workgroup takes 32 of one head's.  As the state update of ssm_forward_kernel.  Bound: the states' bytes (8 x 16
// heads x 2048 tokens, d = N = 64, bf16: 49-61 us for 134 MB of states and 76 MB of reads, 3.5-4.3 TB/s; in two launches 80).
template <typename T, int D, int NP> __global__ void __launch_bounds__(256) ssm_walk_kernel(SsmBwdArgs a)
{
    typedef typename Frag<T>::type F;
    constexpr int DS = 32, PE = 16 / (int)sizeof(T), CHX = DS / PE, CHB = NP / PE;
    constexpr int NX = 64 * CHX, PB = 64 * CHB / 256, PX = (NX + 255) / 256;
    constexpr int LX = red_ld<T>(DS), LB = nat_ld<T>(NP), TNW = NP / 64, TD = DS / 16;
    __shared__ __attribute__((aligned(16))) T sX[2][64 * LX];
    __shared__ __attribute__((aligned(16))) T sB[2][64 * LB];
    __shared__ __attribute__((aligned(16))) float sW[2][64];
    __shared__ float sTot[2];

    const unsigned half = gridDim.x / 2;
    const bool back = blockIdx.x >= half;
    long long u = xcd_unit(back ? blockIdx.x - half : blockIdx.x, a.walk_per);
    if (u >= a.walk_units) return;
    const int d0 = (int)(u % (D / DS)) * DS;
    u /= D / DS;
    const int h = (int)(u % a.H), b = (int)(u / a.H);
    const int bh = b * a.H + h, grp = h / (a.H / a.G);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const int len = ssm_length(a.lengths, b, a.L);
    const T* x = (const T*)(back ? a.dy : a.x) + (size_t)bh * a.L * D + d0;
    const T* Bm = (const T*)(back ? a.Cm : a.Bm) + ((size_t)b * a.G + grp) * a.L * a.N;
    const float* dt = a.dt + (size_t)bh * a.L;
    const double rate = ssm_rate(a.A[h]);
    float* store = (back ? a.leave : a.enter) + (size_t)bh * a.nch * a.N * D + d0;
    const float* from = back ? a.dstate_out : a.state_in;

    floatx4 hs[TNW][TD];
#pragma unroll
    for (int nt = 0; nt < TNW; ++nt) {
        const int n = 16 * (TNW * wave + nt) + r;
#pragma unroll
        for (int d = 0; d < TD; ++d)
            hs[nt][d] = from && n < a.N ? ld4f(from + ((size_t)bh * a.N + n) * D + d0 + 16 * d + 4 * g) : zero4();
    }
    auto put = [&](float* to) {
#pragma unroll
        for (int nt = 0; nt < TNW; ++nt) {
            const int n = 16 * (TNW * wave + nt) + r;
            if (n < a.N)
#pragma unroll
                for (int d = 0; d < TD; ++d) st4f(to + (size_t)n * D + 16 * d + 4 * g, hs[nt][d]);
        }
    };
    intx4 xr[PX], br[PB];
    float dtr = 0.f;
    auto load = [&](int c) {
        const int n = min(64, len - 64 * c);
#pragma unroll
        for (int i = 0; i < PX; ++i) {
            const int k = i * 256 + tid, row = k / CHX, ch = k % CHX;
            xr[i] = intx4{0, 0, 0, 0};
            if (k < NX && row < n) xr[i] = *(const intx4*)(x + (size_t)(64 * c + row) * D + ch * PE);
        }
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const int row = (i * 256 + tid) / CHB, ch = (i * 256 + tid) % CHB;
            br[i] = intx4{0, 0, 0, 0};
            if (row < n && ch * PE < a.N) br[i] = *(const intx4*)(Bm + (size_t)(64 * c + row) * a.N + ch * PE);
        }
        if (wave == 0) dtr = lane < n ? dt[64 * c + lane] : 0.f;
    };
    // the last chunk in the order of the walk is needed only for the gradient of the state before the call
    const int steps = back ? a.nch : a.nch - 1;
    auto chunk = [&](int i) { return back ? a.nch - 1 - i : i; };
    if (steps > 0) load(chunk(0));
    for (int i = 0; i < steps; ++i) {
        const int buf = i & 1;
#pragma unroll
        for (int k = 0; k < PX; ++k) {
            const int q = k * 256 + tid, row = q / CHX, ch = q % CHX;
            if (q < NX) *(intx4*)(sX[buf] + row * LX + ch * PE) = xr[k];
        }
#pragma unroll
        for (int k = 0; k < PB; ++k) {
            const int row = (k * 256 + tid) / CHB, ch = (k * 256 + tid) % CHB;
            *(intx4*)(sB[buf] + row * LB + ch * PE) = br[k];
        }
        if (wave == 0) {
            const double s = wave_scan(ssm_exponent(dtr, rate)), tot = wave_last(s);
            sW[buf][lane] = back ? exp2_f64(s) : exp2_f64(tot - s) * dtr;
            if (lane == 0) sTot[buf] = exp2_f64(tot);
        }
        __syncthreads();
        if (i + 1 < steps) load(chunk(i + 1));
        put(store + (size_t)chunk(i) * a.N * D);
        Split<T> wb[TNW][2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const floatx8 w = join(ld4f(sW[buf] + 32 * kb + 4 * g), ld4f(sW[buf] + 32 * kb + 16 + 4 * g));
#pragma unroll
            for (int nt = 0; nt < TNW; ++nt)
                wb[nt][kb].set(w * to_f8(ld_red(sB[buf], LB, 16 * (TNW * wave + nt), kb, g, r)));
        }
        const float tot = sTot[buf];
#pragma unroll
        for (int nt = 0; nt < TNW; ++nt)
#pragma unroll
            for (int d = 0; d < TD; ++d) hs[nt][d] *= tot;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            F xf[TD];
#pragma unroll
            for (int d = 0; d < TD; ++d) xf[d] = ld_red(sX[buf], LX, 16 * d, kb, g, r);
#pragma unroll
            for (int nt = 0; nt < TNW; ++nt) mma_split(xf, wb[nt][kb], hs[nt]);
        }
    }
    if (!back) put(store + (size_t)(a.nch - 1) * a.N * D);
    if (back && a.dstate_in) put(a.dstate_in + (size_t)bh * a.N * D + d0);
}

// One chunk of a group's heads (or of a part of them).  Wave w owns 16 tokens, first as columns t (dC and the row sums of M), then as columns u
// (dx, dB and the column sums), so that every product's second operand is an accumulator of the wave; dB and dC stay in registers
// over the heads.  Bound: the waits between its phases, for memory and at barriers (8 x 16 heads x 2048 tokens in two groups, d = N = 64, bf16: 85-92 us for 250
// MB, two states of 64 tokens among them: more than half of the waves' cycles are waits, the matrix pipes are busy 12 % and vector instructions issue in 39 %;
// loads a phase ahead cost spills and gained nothing).
template <typename T, int D, int NP>
__global__ void __launch_bounds__(256, sizeof(T) == 2 && NP == 64 ? 2 : 1) ssm_bwd_kernel(SsmBwdArgs a)
{
    typedef typename Frag<T>::type F;
    constexpr bool two = sizeof(T) == 2;
    constexpr int PE = 16 / (int)sizeof(T), LD1 = nat_ld<T>(D), LD2 = nat_ld<T>(NP);
    constexpr int TN = NP / 16, TD = D / 16, SH = NP * LD1;
    constexpr int C1 = D / PE, C2 = NP / PE, P1 = 64 * C1 / 256, P2 = 64 * C2 / 256, PS = NP * D / 4 / 256;
    // States of up to 4096 elements: B and C stay in LDS for all heads, and h waits in registers for its product with g (bf16, d = N = 64: the
    // kernel 98 -> 85 us).  Larger ones have neither the registers nor, at d = 128, the LDS: a workgroup per compute unit would go.
    constexpr bool stay = PS <= 4;
    __shared__ __attribute__((aligned(16))) T s1[64 * LD1];             // x, then dy
    __shared__ __attribute__((aligned(16))) T s2[(stay ? 2 : 1) * 64 * LD2];  // B, then C; or both
    __shared__ __attribute__((aligned(16))) T sH[(two ? 3 : 1) * SH];   // h, then g: rounded, what that leaves, and what that leaves
    __shared__ __attribute__((aligned(16))) float sS[64], sSl[64], sDt[64];
    __shared__ double sDs[64], sLate[64], sDD[4];
    __shared__ float sE[64], sF[64], sP[64], sDot[4];

    long long u = xcd_unit(blockIdx.x, a.per);
    if (u >= a.units) return;
    const int hpart = (int)(u % a.hsplit);
    u /= a.hsplit;
    const int grp = (int)(u % a.G);
    u /= a.G;
    const int c = (int)(u % a.nch), b = (int)(u / a.nch);
    const int rep = a.H / a.G, each = (rep + a.hsplit - 1) / a.hsplit;
    const int h0 = grp * rep + hpart * each, h1 = min((grp + 1) * rep, h0 + each);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const int len = ssm_length(a.lengths, b, a.L), n = min(64, len - 64 * c);  // tokens (none or less: padding)
    const int me = 16 * wave + r;                                              // the lane's token, as t and as u
    const size_t bc = ((size_t)b * a.G + grp) * a.L + 64 * c;
    const T *Bm = (const T*)a.Bm + bc * a.N, *Cm = (const T*)a.Cm + bc * a.N;

    floatx4 dc[TN], db[TN];
#pragma unroll
    for (int i = 0; i < TN; ++i) dc[i] = db[i] = zero4();

    // A phase's tiles: 64 rows of D columns for s1 and a state for sH.  All loads are issued before the first store to LDS (tile by tile
    // each waited for memory anew: 10000 cycles a phase instead of 4000).
    intx4 r1[P1];
    floatx4 rst[PS], held[stay ? PS : 1];
    const intx4 zero = {0, 0, 0, 0};  // rows past n and columns past N
    auto fetch = [&](const T* p1, const float* ps) {
#pragma unroll
        for (int i = 0; i < P1; ++i) {
            const int row = (i * 256 + tid) / C1, k = (i * 256 + tid) % C1 * PE;
            r1[i] = *(const intx4*)(p1 + (unsigned)(min(row, n - 1) * D + k));
        }
#pragma unroll
        for (int i = 0; i < PS; ++i) {
            const int row = (i * 256 + tid) / (D / 4), k = (i * 256 + tid) % (D / 4) * 4;
            rst[i] = ld4f(ps + (unsigned)(min(row, a.N - 1) * D + k));
        }
    };
    auto place = [&] {
#pragma unroll
        for (int i = 0; i < P1; ++i) {
            const int row = (i * 256 + tid) / C1, k = (i * 256 + tid) % C1 * PE;
            *(intx4*)(s1 + row * LD1 + k) = row < n ? r1[i] : zero;
        }
#pragma unroll
        for (int i = 0; i < PS; ++i) {
            const int row = (i * 256 + tid) / (D / 4), k = (i * 256 + tid) % (D / 4) * 4;
            floatx4 v = row < a.N ? rst[i] : zero4();
            T* to = sH + row * LD1 + k;
            st4(to, v);
            if constexpr (two) {
                v -= to_f4(cvt4(v, T()));
                st4(to + SH, v);
                st4(to + 2 * SH, v - to_f4(cvt4(v, T())));
            }
        }
    };
    auto rows_of = [&](const T* p2, T* to) {  // 64 rows of N columns
        intx4 r2[P2];
#pragma unroll
        for (int i = 0; i < P2; ++i) {
            const int row = (i * 256 + tid) / C2, k = (i * 256 + tid) % C2 * PE;
            r2[i] = *(const intx4*)(p2 + (size_t)min(row, n - 1) * a.N + min(k, a.N - PE));
        }
#pragma unroll
        for (int i = 0; i < P2; ++i) {
            const int row = (i * 256 + tid) / C2, k = (i * 256 + tid) % C2 * PE;
            *(intx4*)(to + row * LD2 + k) = row < n && k < a.N ? r2[i] : zero;
        }
    };
    T *tB = s2, *tC = s2 + (stay ? 64 * LD2 : 0);
    auto tokens = [&](const void* p, int h) { return (const T*)p + (((size_t)b * a.H + h) * a.L + 64 * c) * D; };
    auto state = [&](const float* p, int h) { return p + (((size_t)b * a.H + h) * a.nch + c) * a.N * D; };
    if (stay && n > 0 && h0 < h1) {
        rows_of(Bm, tB);
        rows_of(Cm, tC);
    }
    for (int h = h0; h < h1; ++h) {
        const size_t bh = (size_t)b * a.H + h, tok = bh * a.L + 64 * c;
        const T *x = (const T*)a.x + tok * D, *dy = (const T*)a.dy + tok * D;
        if (n <= 0) {
            for (int i = tid; i < min(64, a.L - 64 * c) * (D / PE); i += 256)
                *(intx4*)((T*)a.dx + tok * D + (size_t)i * PE) = intx4{0, 0, 0, 0};
            if (tid < min(64, a.L - 64 * c)) a.ddt[tok + tid] = 0.f;
            if (tid < 2) a.part_head[(bh * a.nch + c) * 2 + tid] = 0.0;
            continue;
        }
        const float skip = a.Dm ? a.Dm[h] : 0.f;
        const double A = a.A[h];

        // four rows n = 16 nt + 4g .. of the state times the lane's token
        auto mma_state = [&](int nt, const F(&f)[D / 32]) {
            floatx4 o = zero4();
#pragma unroll
            for (int kb = 0; kb < D / 32; ++kb) {
                if constexpr (two) {
                    o = mma(ld_nat(sH + 2 * SH + (16 * nt + r) * LD1, kb, g), f[kb], o);
                    o = mma(ld_nat(sH + SH + (16 * nt + r) * LD1, kb, g), f[kb], o);
                }
                o = mma(ld_nat(sH + (16 * nt + r) * LD1, kb, g), f[kb], o);
            }
            return o;
        };
        auto decay = [&](float st, float stl, int i, floatx4& out, bool rows_are_t) {  // e^{s_t - s_u} of four rows
            const floatx4 s = ld4f(sS + i), sl = ld4f(sSl + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = exp2_fast(rows_are_t ? (s[e] - st) + (sl[e] - stl) : (st - s[e]) + (stl - sl[e]));
        };

        // ---- columns t
        float d = 0.f;
        if (wave == 0 && lane < n) d = a.dt[tok + lane];
        F cf[NP / 32], yf[D / 32];
#pragma unroll
        for (int kb = 0; kb < NP / 32; ++kb)
            if (!stay) cf[kb] = me < n ? ld_acc_row<T>(Cm + (size_t)me * a.N, kb, g, a.N) : zero_frag<T>();
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) yf[kb] = me < n ? ld_nat(dy + (size_t)me * D, kb, g) : zero_frag<T>();
        fetch(x, state(a.enter, h));
        if (!stay) rows_of(Bm, tB);
        place();
        if constexpr (stay)
#pragma unroll
            for (int i = 0; i < PS; ++i) held[i] = rst[i];
        if (wave == 0) {
            const double s = wave_scan(ssm_exponent(d, ssm_rate(a.A[h]))), tot = wave_last(s);
            sS[lane] = (float)s;
            sSl[lane] = (float)(s - (double)(float)s);
            sDt[lane] = d;
            sE[lane] = exp2_f64(s);
            sF[lane] = exp2_f64(tot - s);
        }
        __syncthreads();
        if (stay)
#pragma unroll
            for (int kb = 0; kb < NP / 32; ++kb) cf[kb] = ld_acc(tC, LD2, 16 * wave, kb, g, r);
        const float s_me = sS[me], sl_me = sSl[me], dt_me = sDt[me], e_me = sE[me], f_me = sF[me];
        double rs = 0.0;
        {
            float rh = 0.f;
            floatx4 p[4];
#pragma unroll
            for (int ut = 0; ut < 4; ++ut) {
                p[ut] = zero4();
                if (ut <= wave) {
                    floatx4 k = zero4(), q = zero4(), l;
#pragma unroll
                    for (int kb = 0; kb < NP / 32; ++kb) k = mma(ld_acc(tB, LD2, 16 * ut, kb, g, r), cf[kb], k);
#pragma unroll
                    for (int kb = 0; kb < D / 32; ++kb) q = mma(ld_nat(s1 + (16 * ut + r) * LD1, kb, g), yf[kb], q);
                    decay(s_me, sl_me, 16 * ut + 4 * g, l, false);
                    const floatx4 du = ld4f(sDt + 16 * ut + 4 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float w = 16 * ut + 4 * g + e <= me ? l[e] * q[e] : 0.f;
                        p[ut][e] = w * du[e];
                        rs += (double)(w * k[e]) * (double)du[e];
                    }
                }
            }
            const F pf[2] = {frag_from_acc<T>(p[0], p[1]), frag_from_acc<T>(p[2], p[3])};
#pragma unroll
            for (int nt = 0; nt < TN; ++nt) {
                const floatx4 o = mma_state(nt, yf) * e_me;
#pragma unroll
                for (int e = 0; e < 4; ++e) rh += o[e] * (float)cf[nt >> 1][4 * (nt & 1) + e];
                dc[nt] += o;
                dc[nt] = mma(ld_red(tB, LD2, 16 * nt, 0, g, r), pf[0], dc[nt]);
                if (wave >= 2) dc[nt] = mma(ld_red(tB, LD2, 16 * nt, 1, g, r), pf[1], dc[nt]);
            }
            rs = rows_sum_f64(rs) + (double)rows_sum(rh);
        }
        __syncthreads();

        // ---- columns u
        F bf[NP / 32], xf[D / 32];
#pragma unroll
        for (int kb = 0; kb < NP / 32; ++kb)
            if (!stay) bf[kb] = me < n ? ld_acc_row<T>(Bm + (size_t)me * a.N, kb, g, a.N) : zero_frag<T>();
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) xf[kb] = me < n ? ld_nat(x + (size_t)me * D, kb, g) : zero_frag<T>();
        fetch(dy, state(a.leave, h));
        if (!stay) rows_of(Cm, tC);
        place();
        float dot = 0.f;  // <g, h>
#pragma unroll
        for (int i = 0; i < PS; ++i) {
            const int row = (i * 256 + tid) / (D / 4), k = (i * 256 + tid) % (D / 4) * 4;
            floatx4 w;
            if constexpr (stay) w = held[i];
            else w = ld4f(state(a.enter, h) + (unsigned)(min(row, a.N - 1) * D + k));
            const float p = rst[i][0] * w[0] + rst[i][1] * w[1] + rst[i][2] * w[2] + rst[i][3] * w[3];
            dot += row < a.N ? p : 0.f;
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) dot += __shfl_xor(dot, off);
        if (lane == 0) sDot[wave] = dot;
        __syncthreads();
        if (stay)
#pragma unroll
            for (int kb = 0; kb < NP / 32; ++kb) bf[kb] = ld_acc(tB, LD2, 16 * wave, kb, g, r);
        double pu = 0.0;
        float late = 0.f;
        {
            floatx4 pk[4], pq[4];
#pragma unroll
            for (int tt = 0; tt < 4; ++tt) {
                pk[tt] = pq[tt] = zero4();
                if (tt >= wave) {
                    floatx4 k = zero4(), q = zero4(), l;
#pragma unroll
                    for (int kb = 0; kb < NP / 32; ++kb) k = mma(ld_acc(tC, LD2, 16 * tt, kb, g, r), bf[kb], k);
#pragma unroll
                    for (int kb = 0; kb < D / 32; ++kb) q = mma(ld_nat(s1 + (16 * tt + r) * LD1, kb, g), xf[kb], q);
                    decay(s_me, sl_me, 16 * tt + 4 * g, l, true);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int t = 16 * tt + 4 * g + e;
                        const float w = t >= me ? l[e] : 0.f;
                        pk[tt][e] = t >= me ? w * k[e] : 0.f;
                        pq[tt][e] = t >= me ? w * q[e] : 0.f;
                        pu += (double)(pq[tt][e] * k[e]);  // the value that the rows summed
                    }
                }
            }
            const F kf[2] = {frag_from_acc<T>(pk[0], pk[1]), frag_from_acc<T>(pk[2], pk[3])};
            const F qf[2] = {frag_from_acc<T>(pq[0], pq[1]), frag_from_acc<T>(pq[2], pq[3])};
#pragma unroll
            for (int nt = 0; nt < TN; ++nt) {
                floatx4 o = mma_state(nt, xf) * f_me;
#pragma unroll
                for (int e = 0; e < 4; ++e) late += o[e] * (float)bf[nt >> 1][4 * (nt & 1) + e];
                if (wave < 2) o = mma(ld_red(tC, LD2, 16 * nt, 0, g, r), qf[0], o);
                o = mma(ld_red(tC, LD2, 16 * nt, 1, g, r), qf[1], o);
                db[nt] += dt_me * o;
            }
#pragma unroll
            for (int d = 0; d < TD; ++d) {
                floatx4 o = zero4();
#pragma unroll
                for (int kb = 0; kb < NP / 32; ++kb) o = mma(ld_red(sH, LD1, 16 * d, kb, g, r), bf[kb], o);
                o *= f_me;
                if (wave < 2) o = mma(ld_red(s1, LD1, 16 * d, 0, g, r), kf[0], o);
                o = mma(ld_red(s1, LD1, 16 * d, 1, g, r), kf[1], o);
                const floatx4 yt = to_f4(ld4<T>(s1 + me * LD1 + 16 * d + 4 * g));
                if (64 * c + me < a.L) st4((T*)a.dx + (tok + me) * D + 16 * d + 4 * g, me < n ? dt_me * o + skip * yt : zero4());
            }
        }
        // x . dy of the token, a sum that goes on over all tokens of a head: products (exact in bf16) summed in float64
        double xy = 0.0;
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) {
            const floatx8 a8 = to_f8(xf[kb]), b8 = to_f8(ld_nat(s1 + me * LD1, kb, g));
#pragma unroll
            for (int e = 0; e < 8; ++e) xy += (double)(a8[e] * b8[e]);
        }
        late = rows_sum(late);
        pu = rows_sum_f64(pu) + (double)late;
        if (g == 0) {
            sP[me] = (float)pu;
            sDs[me] = rs - (double)dt_me * pu;
            sLate[me] = (double)dt_me * (double)late;
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) xy += __shfl_xor(xy, off);
        if (lane == 0) sDD[wave] = xy;
        __syncthreads();
        if (wave == 0) {
            const double ds = sDs[lane], below = wave_scan(ds), all = wave_last(below);
            const double late_all = wave_last(wave_scan(sLate[lane]));
            const double end = late_all + (double)sE[63] * ((double)sDot[0] + sDot[1] + sDot[2] + sDot[3]);
            const double da = all - below + ds + end;
            if (64 * c + lane < a.L) a.ddt[tok + lane] = lane < n ? (float)((double)sP[lane] + A * da) : 0.f;
            const double dA = wave_last(wave_scan((double)sDt[lane] * da));
            if (lane == 0) {
                a.part_head[(bh * a.nch + c) * 2] = dA;
                a.part_head[(bh * a.nch + c) * 2 + 1] = sDD[0] + sDD[1] + sDD[2] + sDD[3];
            }
        }
    }

    if (64 * c + me >= a.L) return;
    if (a.hsplit == 1) {
        T *oc = (T*)a.dCm + (bc + me) * a.N, *ob = (T*)a.dBm + (bc + me) * a.N;
#pragma unroll
        for (int nt = 0; nt < TN; ++nt)
            if (16 * nt + 4 * g < a.N) {
                st4(oc + 16 * nt + 4 * g, me < n ? dc[nt] : zero4());
                st4(ob + 16 * nt + 4 * g, me < n ? db[nt] : zero4());
            }
    } else {
        float* to = a.part_bc + (((((size_t)hpart * a.B + b) * a.G + grp) * a.nch + c) * 2 * 64 + me) * a.N;
#pragma unroll
        for (int nt = 0; nt < TN; ++nt)
            if (16 * nt + 4 * g < a.N) {
                st4f(to + 16 * nt + 4 * g, me < n ? dc[nt] : zero4());
                st4f(to + (size_t)64 * a.N + 16 * nt + 4 * g, me < n ? db[nt] : zero4());
            }
    }
}

// dB and dC from the parts of the heads, in order.
template <typename T> __global__ void __launch_bounds__(256) ssm_bwd_sum_kernel(SsmBwdArgs a)
{
    const size_t n4 = a.N / 4, all = (size_t)a.B * a.G * a.nch * 2 * 64 * n4;
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= all) return;
    const size_t k = 4 * (i % n4), row = i / n4;  // ((b, g, chunk), which, token)
    const size_t t = row % 64, which = row / 64 % 2, bgc = row / 128;
    const size_t at = 64 * (bgc % a.nch) + t;
    if (at >= (size_t)a.L) return;
    floatx4 s = zero4();
    for (int p = 0; p < a.hsplit; ++p) s += ld4f(a.part_bc + ((size_t)p * all + i) * 4);
    st4((T*)(which ? a.dBm : a.dCm) + (bgc / a.nch * a.L + at) * a.N + k, s);
}

// dA and dD of a head: the chunks' parts, in float64 and in a fixed order.
__global__ void __launch_bounds__(256) ssm_bwd_head_kernel(SsmBwdArgs a)
{
    __shared__ double red[2][256];
    const int h = blockIdx.x;
    double s[2] = {0.0, 0.0};
    for (int i = threadIdx.x; i < a.B * a.nch; i += 256) {
        const double* p = a.part_head + (((size_t)(i / a.nch) * a.H + h) * a.nch + i % a.nch) * 2;
        s[0] += p[0];
        s[1] += p[1];
    }
    red[0][threadIdx.x] = s[0];
    red[1][threadIdx.x] = s[1];
    __syncthreads();
    for (int w = 128; w > 0; w >>= 1) {
        if ((int)threadIdx.x < w) {
            red[0][threadIdx.x] += red[0][threadIdx.x + w];
            red[1][threadIdx.x] += red[1][threadIdx.x + w];
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        a.dA[h] = (float)red[0][0];
        if (a.dD) a.dD[h] = (float)red[1][0];
    }
}

template <typename T, int D, int NP> hipError_t backward_n(const SsmBwdArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((ssm_walk_kernel<T, D, NP>), dim3((unsigned)(16 * a.walk_per)), dim3(256), 0, s, a);
    hipLaunchKernelGGL((ssm_bwd_kernel<T, D, NP>), dim3((unsigned)(8 * a.per)), dim3(256), 0, s, a);
    if (a.hsplit > 1) {
        const size_t n = (size_t)a.B * a.G * a.nch * 2 * 64 * (a.N / 4);
        hipLaunchKernelGGL((ssm_bwd_sum_kernel<T>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
    }
    hipLaunchKernelGGL(ssm_bwd_head_kernel, dim3((unsigned)a.H), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T, int D> hipError_t backward_d(const SsmBwdArgs& a, hipStream_t s)
{
    return a.N <= 64 ? backward_n<T, D, 64>(a, s) : backward_n<T, D, 128>(a, s);
}

}  // namespace

hipError_t launch_ssm_backward(int bf16_io, int D, const SsmBwdArgs& a, hipStream_t s)
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
