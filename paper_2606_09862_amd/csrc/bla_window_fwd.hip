// Window attention over a prompt (bla_window_forward).
#include "bla_window.h"

namespace bla {
namespace {

// The rings after the call: slot s takes the newest token whose place it is, else what it held.  The forward kernel's workgroups past
// its own do it, a piece of 16 bytes to a thread, so that it needs no launch.
template <typename T, int D> __device__ __forceinline__ void window_ring(const WindowArgs& a, long long i)
{
    constexpr int PE = 16 / (int)sizeof(T), CH = D / PE;
    const int slots = a.S + a.W;
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

// One pass over a query block's keys with the running maximum and sum of the softmax.
//
// A workgroup of NW waves takes 16 NW queries of one head (wave w the 16 from 16 w on) and walks the keys that any of them
// sees: first the sinks before the window of its first query, then the window's keys, as one row of `total` keys in tiles of
// 64.  With a ring (RING) the past's keys are read from it and the new tokens' from k, v, so that a tile may hold sinks,
// past and new keys alike.  Tiles are loaded into registers one ahead and pass through two LDS buffers, one
// barrier per tile.
// S^T = K Q^T gives each lane four keys of one query (accumulator rows: keys), so the softmax runs down a column
// (in the lane, then over the four row groups), and the accumulators, rounded to the operand type, are the
// operand of O^T = V^T P without leaving the registers.  In bf16 the weights are rounded to 2^-8 relative at most, as their
// values are; maxima, sums and outputs are float32.
// The maximum that the weights are taken against follows the true one only once that is more than 2^kLag above it: the
// weights stay below 2^kLag, no precision is lost, and a tile needs neither a reduction over the lanes nor a rescaling
// unless some lane has found such a score.
// Bound: issue.  A SIMD's vector and matrix instructions hardly overlap.  Of 32 keys a lane has eight scores: 30 vector instructions for exponentials, sums and
// conversion and 5 for the maximum, then 24 or 40 more if some pair is masked and 32 (d = 64) or 48 (d = 128) if the maximum moves; a tile costs 23 or 46 for
// the next one's addresses, and a workgroup some 300 before its first tile and after its last.  That is 9.6 a visible pair at d = 64 and window 1024, and 19.6 at
// d = 128 and window 255, where a lane has 64 visible pairs in all and a third of its tiles are masked (8 x 16 heads x 4096 queries, four heads to a key head, d = 64, window 1024, bf16:
// 190-220 us, 550-640 TFLOP/s of visible pairs; the first form, a wave to 16 queries of 4-wave groups with a reduction a tile, 337 us.  16 heads x 65536,
// d = 128, window 255: 320-343 us for 1.08 GB, 3.3 TB/s; first form 893).
template <typename T, int D, int NW> struct WinGeo {
    static constexpr int BQ = 16 * NW, NT = 64 * NW;
    static constexpr int LK = nat_ld<T>(D), LV = red_ld<T>(D);
    static constexpr int PE = 16 / (int)sizeof(T), CH = D / PE;  // 16-byte pieces of a row
    static constexpr int NPC = kWinKeys * CH;                    // pieces of a tile
    static constexpr int NP = (NPC + NT - 1) / NT, RPP = NT / CH;
    static constexpr int BUF = kWinKeys * (LK + LV);             // elements of one buffer
};
constexpr float kLag = 8.f;

template <typename T, int D, int NW, bool RING>
__global__ void __launch_bounds__(64 * NW, sizeof(T) == 2 && NW == 8 ? 4 : 1) window_forward_kernel(WindowArgs a)
{
    typedef WinGeo<T, D, NW> G;
    typedef typename Frag<T>::type F;
    __shared__ __attribute__((aligned(16))) T lds[2 * G::BUF];

    if (blockIdx.x >= 8 * (unsigned)a.per) {
        window_ring<T, D>(a, (long long)(blockIdx.x - 8 * (unsigned)a.per) * G::NT + threadIdx.x);
        return;
    }
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
    const int a0 = 16 * wave;                              // the wave's first query in the block

    if (nq <= 0) {  // padding: zeros
        const int rows = min(G::BQ, a.L - q0);
        for (int i = tid; i < rows * G::CH; i += G::NT) {
            if (a.nsplit == 1) *(intx4*)(out + (size_t)i * G::PE) = intx4{0, 0, 0, 0};
        }
        for (int i = tid; i < rows; i += G::NT) {
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
    const int64_t first = RING ? 0 : pos;                   // the first position whose key exists
    const int64_t lo = max(first, p0 - (a.W - 1));
    const int64_t s0 = min(first, (int64_t)a.S);
    const int ns = (int)(min((int64_t)a.S, lo) > s0 ? min((int64_t)a.S, lo) - s0 : 0);
    const int c = (int)(p0 - lo);                           // window keys before the block's first query
    const int total = ns + c + nq;
    const int sb = (int)min((int64_t)0x40000000, max((int64_t)0, a.S - lo));  // window keys that are sinks too
    const int neu = (int)(pos - lo > 0 ? pos - lo : 0);     // window keys that come from the ring
    const int back = (int)(lo > pos ? lo - pos : 0);        // the new token of window key 0
    int r0 = 0, rj = 0;
    if (RING) {                                             // ring slot of the first window key past the sinks
        const int64_t rlo = max(lo, (int64_t)a.S);
        r0 = (int)((rlo - a.S) % a.W);
        rj = (int)(rlo - lo < 0x40000000 ? rlo - lo : 0x40000000);
    }
    const size_t kvrow = ((size_t)b * a.Hkv + hk) * a.L, crow = ((size_t)b * a.Hkv + hk) * ((size_t)a.S + a.W);

    const int ntile = (total + kWinKeys - 1) / kWinKeys;
    const int each = (ntile + a.nsplit - 1) / a.nsplit;
    const int tb = part * each, te = min(ntile, tb + each);

    const int ch = tid % G::CH, lrow = tid / G::CH;
    const T *knew = (const T*)a.k + kvrow * D + ch * G::PE, *vnew = (const T*)a.v + kvrow * D + ch * G::PE;
    const T *kold = (const T*)a.ck + crow * D + ch * G::PE, *vold = (const T*)a.cv + crow * D + ch * G::PE;
    intx4 kr[G::NP], vr[G::NP];
    auto load = [&](int tile) {
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            // rows past the last key repeat it: the mask hides them
            const int i = min(tile * kWinKeys + ps * G::RPP + lrow, total - 1), j = i - ns;
            if (G::NPC < G::NT && lrow >= kWinKeys) continue;
            if (!RING || j >= neu || (j < 0 && s0 + i >= pos)) {
                const size_t at = (size_t)(j < 0 ? (int)(s0 - pos) + i : j - neu + back) * D;
                kr[ps] = *(const intx4*)(knew + at);
                vr[ps] = *(const intx4*)(vnew + at);
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
                const size_t at = (size_t)slot * D;
                kr[ps] = *(const intx4*)(kold + at);
                vr[ps] = *(const intx4*)(vold + at);
            }
        }
    };
    auto store = [&](T* buf) {
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            const int i = ps * G::RPP + lrow;
            if (G::NPC >= G::NT || lrow < kWinKeys) {
                *(intx4*)(buf + i * G::LK + ch * G::PE) = kr[ps];
                *(intx4*)(buf + kWinKeys * G::LK + i * G::LV + ch * G::PE) = vr[ps];
            }
        }
    };

    // queries, sign of the scale folded in (exact), as the second operand of K Q^T
    F qf[D / 32];
    {
        const T* qrow = (const T*)a.q + (row0 + min(a0 + r, nq - 1)) * D;
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) {
            qf[kb] = ld_nat(qrow, kb, g);
            if (a.scale < 0.f)
#pragma unroll
                for (int e = 0; e < 8; ++e) qf[kb][e] = (T)(-(float)qf[kb][e]);
        }
    }
    const float sc = fabsf(a.scale) * kLog2e, lag = kLag / sc;

    floatx4 acc[D / 16];
    float mx = kNoMax, sum = 0.f, limit = kNoMax;           // limit: mx + lag
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc[dt] = zero4();

    const int aend = min(a0 + 16, nq) - 1;  // the wave's last query
    const int jhi = c + a0 + r, jlo = jhi - (a.W - 1);  // the lane's query sees the window keys jlo .. jhi, and those below sb up to jhi
    if (tb < te) load(tb);
    for (int t = tb; t < te; ++t) {
        T* buf = lds + (t & 1) * G::BUF;
        store(buf);
        __syncthreads();
        if (t + 1 < te) load(t + 1);
        const T *sK = buf, *sV = buf + kWinKeys * G::LK;
        if (a0 >= nq) continue;
        // 32 keys at a time: those up to the wave's last query, from its first query's window or a sink on
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int i0 = t * kWinKeys - ns + 32 * hf, i1 = i0 + 31;  // window keys (negative: sinks)
            if (i0 > c + aend || (i0 >= sb && i1 <= c + a0 - a.W)) continue;
            floatx4 s[2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                s[kt] = zero4();
#pragma unroll
                for (int kb = 0; kb < D / 32; ++kb) s[kt] = mma(ld_nat(sK + (32 * hf + 16 * kt + r) * G::LK, kb, g), qf[kb], s[kt]);
            }
            // Masks are selects without branches (& and |, not && and ||, and every element assigned): a form that branched per lane around the
            // products' results was compiled to code with wrong results.
            if (i1 > c + a0 || (i0 <= c + aend - a.W && i1 >= sb)) {  // some pair is not visible
                const int j = i0 + 4 * g;
                if (i0 >= sb) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        s[e >> 2][e & 3] = (unsigned)(j + 16 * (e >> 2) + (e & 3) - jlo) < (unsigned)a.W ? s[e >> 2][e & 3] : -INFINITY;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int k = j + 16 * (e >> 2) + (e & 3);
                        s[e >> 2][e & 3] = (k <= jhi) & ((k >= jlo) | (k < sb)) ? s[e >> 2][e & 3] : -INFINITY;
                    }
                }
            }
            float m = max3(max3(s[0][0], s[0][1], s[0][2]), max3(s[0][3], s[1][0], s[1][1]), max3(s[1][2], s[1][3], s[1][3]));
            if (__any(m > limit)) {
                m = fmaxf(mx, rows_max(m));
                const float al = exp2_fast((mx - m) * sc);
                sum *= al;
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) acc[dt] *= al;
                mx = m;
                limit = m == kNoMax ? kNoMax : m + lag;
            }
            const float nm = -mx * sc;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[kt][e] = exp2_fast(__builtin_fmaf(s[kt][e], sc, nm));
                    sum += s[kt][e];
                }
            const F pf = frag_from_acc<T>(s[0], s[1]);
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) acc[dt] = mma(ld_red(sV, G::LV, 16 * dt, hf, g, r), pf, acc[dt]);
        }
    }

    const int i = a0 + r;
    const float l = rows_sum(sum);
    if (i >= min(G::BQ, a.L - q0)) return;
    const bool real = i < nq;
    if (a.nsplit == 1) {
        const float inv = real ? 1.f / l : 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st4(out + (size_t)i * D + 16 * dt + 4 * g, real ? acc[dt] * inv : zero4());
        if (a.lse && g == 0) a.lse[row0 + i] = real ? (mx * sc + __log2f(l)) * kLn2 : -INFINITY;
    } else {
        const size_t at = (size_t)part * a.B * a.H * a.L + row0 + i;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st4f(a.part_o + at * D + 16 * dt + 4 * g, acc[dt]);
        if (g == 0) {
            a.part_ml[2 * at] = real ? mx * sc : kNoMax;
            a.part_ml[2 * at + 1] = real ? l : 0.f;
        }
    }
}

// A wave joins a row: lane s holds the maximum and the sum of part s (at most 64 parts), then groups of D / 4 lanes take every
// 64 / (D / 4)-th part's outputs, four columns to a lane, and are added up.  Parts without a visible key have a sum of zero and are not read.
// (One thread to four columns of a row walked the parts one after the other: 26 us for 16 rows of 33 parts.)
template <typename T, int D> __global__ void __launch_bounds__(256) window_join_kernel(JoinArgs a)
{
    constexpr int LR = D / 4, PG = 64 / LR;
    const long long row = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, c = 4 * (lane % LR), pg = lane / LR;
    if (row >= a.rows) return;
    float m = kNoMax, l = 0.f;
    if (lane < a.nsplit) {
        const float* ml = a.part_ml + 2 * ((size_t)lane * a.rows + row);
        l = ml[1];
        m = l != 0.f ? ml[0] : kNoMax;
    }
    float top = m;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    float w = l != 0.f ? exp2_fast(m - top) : 0.f;
    l *= w;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off);
    floatx4 o = zero4();
    for (int s0 = 0; s0 < a.nsplit; s0 += 8 * PG) {  // eight loads in flight; what a part without keys holds is dropped
        floatx4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            v[k] = ld4f(a.part_o + ((size_t)min(s0 + k * PG + pg, a.nsplit - 1) * a.rows + row) * D + c);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int s = s0 + k * PG + pg;
            float ws = __shfl(w, s & 63);  // lanes past nsplit hold a weight of zero
            ws = s < 64 ? ws : 0.f;
            o += ws * (ws != 0.f ? v[k] : zero4());
        }
    }
#pragma unroll
    for (int off = 32; off >= LR; off >>= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], off);
    const bool some = l != 0.f;
    if (pg == 0) st4((T*)a.o + (size_t)row * D + c, some ? o * (1.f / l) : zero4());
    if (a.lse && lane == 0) a.lse[row] = some ? (top + __log2f(l)) * kLn2 : -INFINITY;
}

template <typename T, int D, bool RING> hipError_t forward_r(int waves, const WindowArgs& a, hipStream_t s)
{
    const long long pieces = a.ck_out ? (long long)a.B * a.Hkv * (a.S + a.W) * (D * (int)sizeof(T) / 16) : 0;
    const dim3 grid((unsigned)(8 * a.per + (pieces + 64 * waves - 1) / (64 * waves)));
    if (waves == 8)
        hipLaunchKernelGGL((window_forward_kernel<T, D, 8, RING>), grid, dim3(512), 0, s, a);
    else
        hipLaunchKernelGGL((window_forward_kernel<T, D, 4, RING>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T, int D> hipError_t forward_d(int waves, const WindowArgs& a, hipStream_t s)
{
    return a.ck ? forward_r<T, D, true>(waves, a, s) : forward_r<T, D, false>(waves, a, s);
}

template <typename T, int D> hipError_t join_d(const JoinArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((window_join_kernel<T, D>), dim3((unsigned)((a.rows + 3) / 4)), dim3(256), 0, s, a);
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

hipError_t launch_window_forward(int bf16_io, int D, int waves, const WindowArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) forward_d<T, DD>(waves, a, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

hipError_t launch_window_join(int bf16_io, int D, const JoinArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) join_d<T, DD>(a, s)
    BLA_BY_TYPE(BLA_CALL)
#undef BLA_CALL
}

}  // namespace bla
