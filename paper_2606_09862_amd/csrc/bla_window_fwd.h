// Window attention over a prompt: the kernel of bla_window_forward, and of the calls that add a learned bias to its scores (bla_bias_forward)
// or let its queries see a prefix or a cache as a whole (bla_prefix_forward, bla_evict_forward).
#pragma once

#include "bla_bias.h"
#include "bla_window.h"

namespace bla {

constexpr int kPlain = 0, kBias = 1, kPrefix = 2, kEvict = 3, kFew = 4, kBoth = 5;  // what a call adds to window attention

struct BiasArgs : WindowArgs {
    BiasSpec spec;
};
struct PrefixArgs : WindowArgs {
    const void *pk, *pv;    // [G, Hkv, P, D]: the rows b G / B share one, whose tokens every query sees
    const int32_t* plen;    // [G]: its tokens (null: all P)
    int P, G;
    bool by_pos;            // as many tokens as the row's position, P at most

    __device__ __forceinline__ int of_row(int b) const { return b / (B / G); }
    __device__ __forceinline__ int tokens(int b, int64_t pos) const
    {
        return by_pos ? (int)min(pos, (int64_t)P) : plen ? min(max(plen[of_row(b)], 0), P) : P;
    }
};
template <int EXT> struct ExtArgs { typedef WindowArgs type; };
template <> struct ExtArgs<kBias> { typedef BiasArgs type; };
template <> struct ExtArgs<kPrefix> { typedef PrefixArgs type; };

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
template <typename T, int D, int NW, int QT> struct WinGeo {
    static constexpr int BQ = 16 * QT * NW, NT = 64 * NW;
    static constexpr int LK = nat_ld<T>(D), LV = red_ld<T>(D);
    static constexpr int PE = 16 / (int)sizeof(T), CH = D / PE;  // 16-byte pieces of a row
    static constexpr int NPC = kWinKeys * CH;                    // pieces of a tile
    static constexpr int NP = (NPC + NT - 1) / NT, RPP = NT / CH;
    static constexpr int BUF = kWinKeys * (LK + LV);             // elements of one buffer
};
constexpr float kLag = 8.f;

// A bias (EXT = kBias) takes the running maximum into the base-2 domain.  32 keys and 16 queries span 47 distances: where those share a bucket, which
// they do nearly everywhere, the bias is one number beside the maximum in the exponent and costs nothing a pair; of near distances it comes from a table in
// LDS, elsewhere from a selection at each edge.
// A prefix (EXT = kPrefix) has tiles of its own ahead of the others.
// QT tiles of 16 queries to a wave: with two each fragment read from LDS serves two products, and what a tile costs beside its pairs is shared.
// Both are bound by issue as well.  4 x 16 heads x 4096 queries, four heads to a key head, causal, d = 64, bf16, 32 buckets to 128: 186-191 us, 720-740 TFLOP/s of
// visible pairs (208 with a tile to a wave, 235 with the blocks in order of the rows too).  16 rows x 16 heads x 512 queries of which 13 % are padding behind 4096
// tokens: 175 us (650 TFLOP/s over all queries, 754 with 24 whole rows).
template <typename T, int D, int NW, int QT, bool RING, int EXT>
__global__ void __launch_bounds__(64 * NW, sizeof(T) == 2 && NW == 8 ? 4 : 1) window_forward_kernel(typename ExtArgs<EXT>::type a)
{
    typedef WinGeo<T, D, NW, QT> G;
    typedef typename Frag<T>::type F;
    __shared__ __attribute__((aligned(16))) T lds[2 * G::BUF];
    __shared__ float near[EXT == kBias ? kPad + kNear : 1];

    if (blockIdx.x >= 8 * (unsigned)a.per) {
        window_ring<T, D>(a, (long long)(blockIdx.x - 8 * (unsigned)a.per) * G::NT + threadIdx.x);
        return;
    }
    const int grp = a.H / a.Hkv;
    int hg, part, q0, hk, b;
    if constexpr (EXT == kPlain) {
        long long u = xcd_unit(blockIdx.x, a.per);
        if (u >= a.units) return;
        hg = (int)(u % grp);
        u /= grp;
        part = (int)(u % a.nsplit);
        u /= a.nsplit;
        q0 = (int)(u % a.nqb) * G::BQ;
        u /= a.nqb;
        hk = (int)(u % a.Hkv), b = (int)(u / a.Hkv);
    } else {  // windows as long as the rows: the last queries have most keys
        long long u = falling_unit(blockIdx.x, a.units);
        if (u >= a.units) return;
        hk = (int)(u % a.Hkv);
        u /= a.Hkv;
        b = (int)(u % a.B);
        u /= a.B;
        hg = (int)(u % grp);
        u /= grp;
        part = (int)(u % a.nsplit);
        q0 = (a.nqb - 1 - (int)(u / a.nsplit)) * G::BQ;
    }
    const int h = hk * grp + hg;

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    int64_t pos;
    const int len = row_tokens(a.lengths, a.pos, a.t0, b, a.L, pos);
    const int nq = min(G::BQ, len - q0);
    const size_t row0 = ((size_t)b * a.H + h) * a.L + q0;  // the block's first row of q, o, lse
    T* const out = (T*)a.o + row0 * D;
    const int a0 = 16 * QT * wave;                           // the wave's first query in the block

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

    int np = 0, ntp = 0;                                    // the prefix, and its tiles
    const T *kpre = nullptr, *vpre = nullptr;
    if constexpr (EXT == kPrefix) {
        np = a.tokens(b, pos);
        ntp = (np + kWinKeys - 1) / kWinKeys;
        const size_t at = ((size_t)a.of_row(b) * a.Hkv + hk) * a.P * D + (tid % G::CH) * G::PE;
        kpre = (const T*)a.pk + at;
        vpre = (const T*)a.pv + at;
    }
    BiasLanes lanes = {};
    int64_t far = 0;                                        // what a sink is further away than its index says
    if constexpr (EXT == kBias) {
        lanes.set_edges(a.spec, lane);
        lanes.set_head(a.spec, h, lane);
        lanes.table(a.spec, near, wave, NW, lane);
        far = min(lo - s0 - ns, (int64_t)1 << 29);
    }
    const int ntile = ntp + (total + kWinKeys - 1) / kWinKeys;
    const int each = (ntile + a.nsplit - 1) / a.nsplit;
    const int tb = part * each, te = min(ntile, tb + each);

    const int ch = tid % G::CH, lrow = tid / G::CH;
    const T *knew = (const T*)a.k + kvrow * D + ch * G::PE, *vnew = (const T*)a.v + kvrow * D + ch * G::PE;
    const T *kold = (const T*)a.ck + crow * D + ch * G::PE, *vold = (const T*)a.cv + crow * D + ch * G::PE;
    intx4 kr[G::NP], vr[G::NP];
    auto load = [&](int tile) {
        if constexpr (EXT == kPrefix) {
            if (tile < ntp) {
#pragma unroll
                for (int ps = 0; ps < G::NP; ++ps) {
                    if (G::NPC < G::NT && lrow >= kWinKeys) continue;
                    const size_t at = (size_t)min(tile * kWinKeys + ps * G::RPP + lrow, np - 1) * D;
                    kr[ps] = *(const intx4*)(kpre + at);
                    vr[ps] = *(const intx4*)(vpre + at);
                }
                return;
            }
            tile -= ntp;
        }
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
    F qf[QT][D / 32];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const T* qrow = (const T*)a.q + (row0 + min(a0 + 16 * qt + r, nq - 1)) * D;
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) {
            qf[qt][kb] = ld_nat(qrow, kb, g);
            if (a.scale < 0.f)
#pragma unroll
                for (int e = 0; e < 8; ++e) qf[qt][kb][e] = (T)(-(float)qf[qt][kb][e]);
        }
    }
    const float sc = fabsf(a.scale) * kLog2e, lag = EXT == kBias ? kLag : kLag / sc;

    floatx4 acc[QT][D / 16];
    float mx[QT], sum[QT], limit[QT];                       // limit: mx + lag
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        mx[qt] = limit[qt] = kNoMax, sum[qt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) acc[qt][dt] = zero4();
    }

    const int aend = min(a0 + 16 * QT, nq) - 1;  // the wave's last query
    const int jhi0 = c + a0 + r;  // with jhi = jhi0 + 16 qt and jlo = jhi - (W - 1) the lane's query sees the window keys jlo .. jhi, and those below sb up to jhi
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
            const int i0 = (t - ntp) * kWinKeys - ns + 32 * hf, i1 = i0 + 31;  // window keys (negative: sinks)
            const bool pre = EXT == kPrefix && t < ntp;
            const int left = np - t * kWinKeys - 32 * hf;                      // prefix tokens from here on
            if (pre ? left <= 0 : (i0 > c + aend || (i0 >= sb && i1 <= c + a0 - a.W))) continue;
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
            // Masks are selects without branches (& and |, not && and ||, and every element assigned): a form that branched per lane around the
            // products' results was compiled to code with wrong results.
            if (pre) {
                if (left < 32)
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            s[qt][e >> 2][e & 3] = 4 * g + 16 * (e >> 2) + (e & 3) < left ? s[qt][e >> 2][e & 3] : -INFINITY;
            } else if (i1 > c + a0 || (i0 <= c + aend - a.W && i1 >= sb)) {  // some pair is not visible
                const int j = i0 + 4 * g;
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) {
                    const int jhi = jhi0 + 16 * qt, jlo = jhi - (a.W - 1);
                    if (i0 >= sb) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            s[qt][e >> 2][e & 3] = (unsigned)(j + 16 * (e >> 2) + (e & 3) - jlo) < (unsigned)a.W ? s[qt][e >> 2][e & 3] : -INFINITY;
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int k = j + 16 * (e >> 2) + (e & 3);
                            s[qt][e >> 2][e & 3] = (k <= jhi) & ((k >= jlo) | (k < sb)) ? s[qt][e >> 2][e & 3] : -INFINITY;
                        }
                    }
                }
            }
            float sx = sc, bu = 0.f;  // kBias: a score in the base-2 domain is s sx + bu
            if constexpr (EXT == kBias) bias_scores<QT>(s, sx, bu, lanes, near, sc, c + a0, i0, (int)far, g, r);
            F pf[QT];
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                floatx4(&x)[2] = s[qt];
                float m = max3(max3(x[0][0], x[0][1], x[0][2]), max3(x[0][3], x[1][0], x[1][1]), max3(x[1][2], x[1][3], x[1][3]));
                if constexpr (EXT == kBias) m = __builtin_fmaf(m, sx, bu);
                if (__any(m > limit[qt])) {
                    m = fmaxf(mx[qt], rows_max(m));
                    const float al = exp2_fast(EXT == kBias ? mx[qt] - m : (mx[qt] - m) * sc);
                    sum[qt] *= al;
#pragma unroll
                    for (int dt = 0; dt < D / 16; ++dt) acc[qt][dt] *= al;
                    mx[qt] = m;
                    limit[qt] = m == kNoMax ? kNoMax : m + lag;
                }
                const float nm = EXT == kBias ? bu - mx[qt] : -mx[qt] * sc;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[kt][e] = exp2_fast(__builtin_fmaf(x[kt][e], sx, nm));
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

#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int i = a0 + 16 * qt + r;
        const float l = rows_sum(sum[qt]), unit = EXT == kBias ? 1.f : sc;  // mx's, in the base-2 domain
        if (i >= min(G::BQ, a.L - q0)) continue;
        const bool real = i < nq && (EXT != kBias || l > 0.f);  // a bias of minus infinity can leave a row without a key
        if (a.nsplit == 1) {
            const float inv = real ? 1.f / l : 0.f;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) st4(out + (size_t)i * D + 16 * dt + 4 * g, real ? acc[qt][dt] * inv : zero4());
            if (a.lse && g == 0) a.lse[row0 + i] = real ? __builtin_fmaf(mx[qt], unit, __log2f(l)) * kLn2 : -INFINITY;
        } else {
            const size_t at = (size_t)part * a.B * a.H * a.L + row0 + i;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) st4f(a.part_o + at * D + 16 * dt + 4 * g, acc[qt][dt]);
            if (g == 0) {
                a.part_ml[2 * at] = real ? mx[qt] * unit : kNoMax;
                a.part_ml[2 * at + 1] = real ? l : 0.f;
            }
        }
    }
}

// A wave joins a row: lane s holds the maximum and the sum of part s (at most 64 parts), then groups of D / 4 lanes take every
// 64 / (D / 4)-th part's outputs, four columns to a lane, and are added up.  Parts without a visible key have a sum of zero and are not read.
// (One thread to four columns of a row walked the parts one after the other: 26 us for 16 rows of 33 parts.)
// block: of 256 threads, four rows to each.
template <typename T, int D> __device__ __forceinline__ void join_rows(const JoinArgs& a, long long block)
{
    constexpr int LR = D / 4, PG = 64 / LR;
    const long long row = block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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

// waves: of 16 queries in a workgroup, 4 or 8.
template <typename T, int D, bool RING, int EXT> hipError_t forward_r(int waves, const typename ExtArgs<EXT>::type& a, hipStream_t s)
{
    constexpr bool two = EXT != kPlain;
    const int threads = waves == 8 && !two ? 512 : 256;
    const long long pieces = a.ck_out ? (long long)a.B * a.Hkv * (a.S + a.W) * (D * (int)sizeof(T) / 16) : 0;
    const dim3 grid((unsigned)(8 * a.per + (pieces + threads - 1) / threads));
    if (waves != 8)
        hipLaunchKernelGGL((window_forward_kernel<T, D, 4, 1, RING, EXT>), grid, dim3(threads), 0, s, a);
    else if constexpr (two)
        hipLaunchKernelGGL((window_forward_kernel<T, D, 4, 2, RING, EXT>), grid, dim3(threads), 0, s, a);
    else
        hipLaunchKernelGGL((window_forward_kernel<T, D, 8, 1, RING, EXT>), grid, dim3(threads), 0, s, a);
    return hipGetLastError();
}

template <typename T, int D, int EXT> hipError_t forward_d(int waves, const typename ExtArgs<EXT>::type& a, hipStream_t s)
{
    return a.ck ? forward_r<T, D, true, EXT>(waves, a, s) : forward_r<T, D, false, EXT>(waves, a, s);
}

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

}  // namespace bla
