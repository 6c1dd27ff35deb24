// Window attention over a prompt (bla_window_forward).
#include "bla_window.h"

namespace bla {
namespace {

// One pass over a query block's keys with the running maximum and sum of the softmax.
//
// A workgroup of four waves takes 64 QT queries of one head (wave w the 16 QT queries from 16 QT w on) and walks
// the keys that any of them sees: first the sinks before the window of its first query, then the window's keys,
// as one row of `total` keys in tiles of 64.  The new tokens' keys are read from k, v and the past's from the ring, so
// that a tile may hold sinks, past and new keys alike.  Tiles are loaded into registers one ahead and pass through two LDS
// buffers, one barrier per tile.
// S^T = K Q^T gives each lane four keys of one query (accumulator rows: keys), so the softmax runs down a column
// (in the lane, then over the four row groups), and the accumulators, rounded to the operand type, are the
// operand of O^T = V^T P without leaving the registers.  In bf16 the weights are rounded to 2^-9 relative, as their
// values are; maxima, sums and outputs are float32.
template <typename T, int D, int QT> struct WinGeo {
    static constexpr int BQ = 64 * QT;
    static constexpr int LK = nat_ld<T>(D), LV = red_ld<T>(D);
    static constexpr int CH = D * (int)sizeof(T) / 16;  // 16-byte pieces of a row
    static constexpr int RPP = 256 / CH;                // rows per pass of the workgroup's loads
    static constexpr int NP = kWinKeys / RPP;
    static constexpr int PE = 16 / (int)sizeof(T);
    static constexpr int BUF = kWinKeys * (LK + LV);    // elements of one buffer
};

template <typename T, int D, int QT>
__global__ void __launch_bounds__(256) window_forward_kernel(WindowArgs a)
{
    typedef WinGeo<T, D, QT> G;
    typedef typename Frag<T>::type F;
    __shared__ __attribute__((aligned(16))) T lds[2 * G::BUF];

    long long u = xcd_unit(blockIdx.x, a.per);
    if (u >= a.units) return;
    const int grp = a.H / a.Hkv;
    const int hg = (int)(u % grp);
    u /= grp;
    const int part = (int)(u % a.nsplit);
    u /= a.nsplit;
    const int q0 = (int)(u % a.nqb) * G::BQ;
    u /= a.nqb;
    const int hk = (int)(u % a.Hkv), b = (int)(u / a.Hkv);
    const int h = hk * grp + hg;

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    int64_t pos;
    const int len = row_tokens(a.lengths, a.pos, a.t0, b, a.L, pos);
    const int nq = min(G::BQ, len - q0);
    const size_t row0 = ((size_t)b * a.H + h) * a.L + q0;  // the block's first row of q, o, lse
    T* const out = (T*)a.o + row0 * D;
    const int a0 = 16 * QT * wave;                         // the wave's first query in the block

    if (nq <= 0) {  // padding: zeros
        const int rows = min(G::BQ, a.L - q0);
        for (int i = tid; i < rows * G::CH; i += 256) {
            if (a.nsplit == 1) *(intx4*)(out + (size_t)i * G::PE) = intx4{0, 0, 0, 0};
        }
        for (int i = tid; i < rows; i += 256) {
            if (a.nsplit == 1) {
                if (a.lse) a.lse[row0 + i] = -INFINITY;
            } else {
                const size_t at = (size_t)part * a.B * a.H * a.L + row0 + i;
                a.part_ml[2 * at] = kNoMax;
                a.part_ml[2 * at + 1] = 0.f;
            }
        }
        return;
    }

    // The block's keys: sinks [s0, s0 + ns), then positions [lo, p0 + nq).
    const int64_t p0 = pos + q0;
    const int64_t first = a.ck ? 0 : pos;                   // the first position whose key exists
    const int64_t lo = max(first, p0 - (a.W - 1));
    const int64_t s0 = min(first, (int64_t)a.S);
    const int ns = (int)(min((int64_t)a.S, lo) > s0 ? min((int64_t)a.S, lo) - s0 : 0);
    const int c = (int)(p0 - lo);                           // window keys before the block's first query
    const int total = ns + c + nq;
    const int sb = (int)min((int64_t)0x40000000, max((int64_t)0, a.S - lo));  // window keys that are sinks too
    const int neu = (int)(pos - lo > 0 ? pos - lo : 0);     // window keys that come from the ring
    const int back = (int)(lo > pos ? lo - pos : 0);        // the new token of window key 0
    const int64_t rlo = max(lo, (int64_t)a.S);              // ring slot of the first window key past the sinks
    const int r0 = (int)((rlo - a.S) % a.W), rj = (int)(rlo - lo < 0x40000000 ? rlo - lo : 0x40000000);
    const size_t kvrow = ((size_t)b * a.Hkv + hk) * a.L, crow = ((size_t)b * a.Hkv + hk) * ((size_t)a.S + a.W);

    const int ntile = (total + kWinKeys - 1) / kWinKeys;
    const int each = (ntile + a.nsplit - 1) / a.nsplit;
    const int tb = part * each, te = min(ntile, tb + each);

    const int ch = tid % G::CH, lrow = tid / G::CH;
    intx4 kr[G::NP], vr[G::NP];
    auto load = [&](int tile) {
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            const int i = tile * kWinKeys + ps * G::RPP + lrow;
            const int j = i - ns;
            kr[ps] = vr[ps] = intx4{0, 0, 0, 0};
            if (i < total) {
                const bool fresh = j >= neu || (j < 0 && s0 + i >= pos);
                if (fresh) {
                    const size_t at = (kvrow + (size_t)(j < 0 ? (int)(s0 + i - pos) : j - neu + back)) * D + ch * G::PE;
                    kr[ps] = *(const intx4*)((const T*)a.k + at);
                    vr[ps] = *(const intx4*)((const T*)a.v + at);
                } else {
                    int slot;
                    if (j < 0) {
                        slot = (int)s0 + i;
                    } else if (j < rj) {
                        slot = (int)lo + j;
                    } else {
                        slot = r0 + (j - rj);
                        slot = a.S + (slot >= a.W ? slot - a.W : slot);
                    }
                    const size_t at = (crow + slot) * D + ch * G::PE;
                    kr[ps] = *(const intx4*)((const T*)a.ck + at);
                    vr[ps] = *(const intx4*)((const T*)a.cv + at);
                }
            }
        }
    };
    auto store = [&](T* buf) {
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            const int i = ps * G::RPP + lrow;
            *(intx4*)(buf + i * G::LK + ch * G::PE) = kr[ps];
            *(intx4*)(buf + kWinKeys * G::LK + i * G::LV + ch * G::PE) = vr[ps];
        }
    };

    // queries, sign of the scale folded in (exact), as the second operand of K Q^T
    F qf[QT][D / 32];
    const float sgn = a.scale < 0.f ? -1.f : 1.f;
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int i = min(a0 + 16 * qt + r, nq - 1);
        const T* qrow = (const T*)a.q + (row0 + i) * D;
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) {
            qf[qt][kb] = ld_nat(qrow, kb, g);
            if (a.scale < 0.f)
#pragma unroll
                for (int e = 0; e < 8; ++e) qf[qt][kb][e] = (T)(sgn * (float)qf[qt][kb][e]);
        }
    }
    const float sc = fabsf(a.scale) * kLog2e;

    floatx4 acc[QT][D / 16];
    float mx[QT], sum[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        mx[qt] = kNoMax;
        sum[qt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) acc[qt][dt] = zero4();
    }

    const int aend = min(a0 + 16 * QT, nq) - 1;  // the wave's last query
    if (tb < te) load(tb);
    for (int t = tb; t < te; ++t) {
        T* buf = lds + (t & 1) * G::BUF;
        store(buf);
        __syncthreads();
        if (t + 1 < te) load(t + 1);
        const int j0 = t * kWinKeys - ns, j1 = j0 + kWinKeys - 1;  // the tile's window keys (negative: sinks)
        // no key of the tile is seen by the wave: past its last query, or before its first window
        if (a0 >= nq || j0 > c + aend || (j0 >= sb && j1 <= c + a0 - a.W)) continue;
        const bool whole = j1 < 0 || (j0 >= 0 && j1 <= c + a0 && (c + aend - j0 < a.W || j1 < sb));
        const T* sK = buf;
        const T* sV = buf + kWinKeys * G::LK;

        floatx4 s[QT][4];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) s[qt][kt] = zero4();
#pragma unroll
            for (int kb = 0; kb < D / 32; ++kb) {
                const F kf = ld_nat(sK + (16 * kt + r) * G::LK, kb, g);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) s[qt][kt] = mma(kf, qf[qt][kb], s[qt][kt]);
            }
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            if (!whole) {
                const int ca = c + a0 + 16 * qt + r;  // the query as a window key
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = j0 + 16 * kt + 4 * g + e;
                        const bool seen = (j < 0) | ((j <= ca) & ((ca - j < a.W) | (j < sb)));  // no branches
                        s[qt][kt][e] = seen ? s[qt][kt][e] : -INFINITY;
                    }
            }
            float m = kNoMax;
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
                m = fmaxf(m, fmaxf(fmaxf(s[qt][kt][0], s[qt][kt][1]), fmaxf(s[qt][kt][2], s[qt][kt][3])));
            m = fmaxf(mx[qt], rows_max(m));
            if (__any(m > mx[qt])) {
                const float al = exp2_fast((mx[qt] - m) * sc);
                sum[qt] *= al;
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) acc[qt][dt] *= al;
                mx[qt] = m;
            }
            const float nm = -m * sc;
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = exp2_fast(__builtin_fmaf(s[qt][kt][e], sc, nm));
                    s[qt][kt][e] = p;
                    sum[qt] += p;
                }
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            F pf[QT];
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) pf[qt] = frag_from_acc<T>(s[qt][2 * kb], s[qt][2 * kb + 1]);
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                const F vf = ld_red(sV, G::LV, 16 * dt, kb, g, r);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) acc[qt][dt] = mma(vf, pf[qt], acc[qt][dt]);
            }
        }
    }

#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int i = a0 + 16 * qt + r;
        const float l = rows_sum(sum[qt]);
        if (i >= min(G::BQ, a.L - q0)) continue;
        const bool real = i < nq;
        if (a.nsplit == 1) {
            const float inv = real ? 1.f / l : 0.f;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) st4(out + (size_t)i * D + 16 * dt + 4 * g, real ? acc[qt][dt] * inv : zero4());
            if (a.lse && g == 0) a.lse[row0 + i] = real ? (mx[qt] * sc + __log2f(l)) * kLn2 : -INFINITY;
        } else {
            const size_t at = (size_t)part * a.B * a.H * a.L + row0 + i;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) st4f(a.part_o + at * D + 16 * dt + 4 * g, acc[qt][dt]);
            if (g == 0) {
                a.part_ml[2 * at] = real ? mx[qt] * sc : kNoMax;
                a.part_ml[2 * at + 1] = real ? l : 0.f;
            }
        }
    }
}

// Four consecutive outputs of one row per lane.  Parts without a visible key have a sum of zero and are not read.
template <typename T, int D> __global__ void __launch_bounds__(256) window_join_kernel(JoinArgs a)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long row = i / (D / 4);
    const int c = 4 * (int)(i % (D / 4));
    if (row >= a.rows) return;
    float m = kNoMax;
    for (int s = 0; s < a.nsplit; ++s) {
        const float* ml = a.part_ml + 2 * ((size_t)s * a.rows + row);
        if (ml[1] != 0.f) m = fmaxf(m, ml[0]);
    }
    float l = 0.f;
    floatx4 o = zero4();
    for (int s = 0; s < a.nsplit; ++s) {
        const size_t at = (size_t)s * a.rows + row;
        const float ls = a.part_ml[2 * at + 1];
        if (ls != 0.f) {
            const float w = exp2_fast(a.part_ml[2 * at] - m);
            l += w * ls;
            o += w * ld4f(a.part_o + at * D + c);
        }
    }
    const bool some = l != 0.f;
    st4((T*)a.o + (size_t)row * D + c, some ? o * (1.f / l) : zero4());
    if (a.lse && c == 0) a.lse[row] = some ? (m + __log2f(l)) * kLn2 : -INFINITY;
}

// The rings after the call: slot s takes the newest token whose place it is, else what it held.
template <typename T, int D> __global__ void __launch_bounds__(256) window_ring_kernel(WindowArgs a)
{
    constexpr int PE = 16 / (int)sizeof(T), CH = D / PE;
    const int slots = a.S + a.W;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long row = i / CH;
    const int ch = (int)(i % CH);
    if (row >= (long long)a.B * a.Hkv * slots) return;
    const long long bh = row / slots;
    const int slot = (int)(row % slots), b = (int)(bh / a.Hkv);
    int64_t pos;
    const int len = row_tokens(a.lengths, a.pos, a.t0, b, a.L, pos);
    int64_t t = -1;  // the new token of the slot
    if (len > 0) {
        const int64_t last = pos + len - 1;
        if (slot < a.S)
            t = slot <= last ? slot - pos : -1;
        else if (slot <= last)
            t = last - (last - slot) % a.W - pos;
    }
    const size_t to = (size_t)row * D + ch * PE;
    intx4 kx = {0, 0, 0, 0}, vx = {0, 0, 0, 0};
    if (t >= 0) {
        const size_t from = ((size_t)bh * a.L + t) * D + ch * PE;
        kx = *(const intx4*)((const T*)a.k + from);
        vx = *(const intx4*)((const T*)a.v + from);
    } else if (a.ck) {
        kx = *(const intx4*)((const T*)a.ck + to);
        vx = *(const intx4*)((const T*)a.cv + to);
    }
    *(intx4*)((T*)a.ck_out + to) = kx;
    *(intx4*)((T*)a.cv_out + to) = vx;
}

template <typename T, int D> hipError_t forward_d(int qt, const WindowArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)(8 * a.per));
    if (qt == 2)
        hipLaunchKernelGGL((window_forward_kernel<T, D, 2>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((window_forward_kernel<T, D, 1>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T, int D> hipError_t join_d(const JoinArgs& a, hipStream_t s)
{
    const long long n = a.rows * (D / 4);
    hipLaunchKernelGGL((window_join_kernel<T, D>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T, int D> hipError_t ring_d(const WindowArgs& a, hipStream_t s)
{
    const long long n = (long long)a.B * a.Hkv * (a.S + a.W) * (D * (int)sizeof(T) / 16);
    hipLaunchKernelGGL((window_ring_kernel<T, D>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

#define BLA_BY_TYPE(CALL)                                      \
    if (bf16_io) {                                             \
        if (D == 32) return CALL(bf16, 32);                    \
        if (D == 64) return CALL(bf16, 64);                    \
        if (D == 128) return CALL(bf16, 128);                  \
    } else {                                                   \
        if (D == 32) return CALL(float, 32);                   \
        if (D == 64) return CALL(float, 64);                   \
        if (D == 128) return CALL(float, 128);                 \
    }                                                          \
    return hipErrorInvalidValue;

hipError_t launch_window_forward(int bf16_io, int D, int qt, const WindowArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) forward_d<T, DD>(qt, a, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

hipError_t launch_window_join(int bf16_io, int D, const JoinArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) join_d<T, DD>(a, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

hipError_t launch_window_ring(int bf16_io, int D, const WindowArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) ring_d<T, DD>(a, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

}  // namespace bla
