// One decode token per row of window attention: the kernel of bla_window_step, of bla_bias_step and of the rings of bla_prefix_step.
#pragma once

#include "bla_window_fwd.h"

namespace bla {

struct BiasStepArgs : WindowStepArgs {
    BiasSpec spec;
};
// The prefix's parts stand ahead of the rings' in part_o and part_ml.
struct PrefixStepArgs : WindowStepArgs {
    const void *pk, *pv;       // [G, Hkv, P, D]
    const int32_t* plen;       // [G] or null
    int P, G;
    int npart, nqb;            // parts of the prefix, blocks of the queries that share it
    long long units, per;      // workgroups of the prefix, per XCD
    float *pre_o, *pre_ml;     // the prefix's parts
};
// The prefix's workgroups where they take it in tiles: queries, groups of waves, threads, and how many fill the device.
struct PrefixShape {
    int block, groups, threads, fill;
};
PrefixShape prefix_shape(int bf16_io, int D);
// How a step takes the prefix: in tiles, as a ring's heads do, or so together with the ring.
enum PrefixForm { kFormTiles, kFormFew, kFormBoth };
// Slots without order (W of them, S = 0); the scores in the base-2 domain go out for the sums of the weights.
struct EvictStepArgs : WindowStepArgs {
    const float* score_in;     // [B, Hkv, W]
    float* score_out;
    const int64_t* at_in;
    int64_t* at_out;
    int recent;
    int* mine;                 // [B, Hkv]: the token's slot
    float* z;                  // [B, H, pitch]
    int pitch;
    bool fused;                // a workgroup has all slots and heads of its key head: it forms the sums itself
    bool in_lds;               // ... and keeps the scores in LDS
};
template <int EXT> struct ExtStepArgs { typedef WindowStepArgs type; };
template <> struct ExtStepArgs<kBias> { typedef BiasStepArgs type; };
template <> struct ExtStepArgs<kPrefix> { typedef PrefixStepArgs type; };
template <> struct ExtStepArgs<kFew> { typedef PrefixStepArgs type; };
template <> struct ExtStepArgs<kBoth> { typedef PrefixStepArgs type; };
template <> struct ExtStepArgs<kEvict> { typedef EvictStepArgs type; };

// A score's place in the order of scores: NaN above every number, the two zeros as one.
__device__ __forceinline__ unsigned score_key(float x)
{
    if (x != x) return 0xfffffffeu;
    const unsigned u = __float_as_uint(x == 0.f ? 0.f : x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The slot that a token of a full cache takes: of those whose token is older than `old` the one with the least score, the lowest of several.  The workgroup's NW
// waves call it with as many words of LDS; every slot is one of slots whatever `at` holds.
template <int NW> __device__ __forceinline__ int evict_slot(const float* score, const int64_t* at, int slots, int64_t old, uint64_t* lds)
{
    uint64_t best = ~0ull;
    for (int i0 = threadIdx.x; i0 < slots; i0 += 8 * 64 * NW) {  // eight loads in flight; a slot that comes twice changes nothing
        float x[8];
        int64_t p[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = min(i0 + 64 * NW * k, slots - 1);
            x[k] = score[i], p[k] = at[i];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint64_t key = (uint64_t)(p[k] < old ? score_key(x[k]) : 0xffffffffu) << 32 | (unsigned)min(i0 + 64 * NW * k, slots - 1);
            best = key < best ? key : best;
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const uint64_t x = __shfl_xor((unsigned long long)best, off);
        best = x < best ? x : best;
    }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = best;
    __syncthreads();
    best = lds[0];
    for (int i = 1; i < NW; ++i) best = lds[i] < best ? lds[i] : best;
    __syncthreads();  // the caller uses the words again
    const unsigned slot = (unsigned)best;
    return slot < (unsigned)slots ? (int)slot : 0;
}

// Slot i of a cache with n tokens after the call, of which the new one's weight is w as well.  Slots without a token stay as they are.
__device__ __forceinline__ void evict_score_out(const EvictStepArgs& a, size_t bh, int i, int mine, int n, int64_t pos, float w)
{
    const size_t at = bh * a.W + i;
    if (i < n)
        a.score_out[at] = (i == mine ? 0.f : a.score_in[at]) + w;
    else if (a.score_out != a.score_in)
        a.score_out[at] = a.score_in[at];
    if (i == mine)
        a.at_out[at] = pos;
    else if (a.at_out != a.at_in)
        a.at_out[at] = a.at_in[at];
}

// A workgroup of four waves takes up to 16 query heads of one key head and a part of the ring: the heads are the
// columns of S^T = K Q^T, so a key is read once for all of them.  Wave w walks blocks of 32 slots, four blocks apart, with a
// running maximum and sum of its own; K fragments come straight from memory (a lane's 16 bytes of a row), V rows go through
// a tile of LDS that only the wave touches, to be read transposed.  The waves' results are joined through LDS, the
// parts' by window_join_kernel.  The token's own key and value are taken from k and v wherever its slot is met, so no
// workgroup reads the slot that one of them writes.  Bound: the ring's bytes (512 rows, four key heads of 1028 slots, d = 64, bf16: 76-81 us
// for 408 MB, 5.2 TB/s); of one row, latency (4 key heads of 4100 slots, d = 128: 6 us in 33 parts and 5 us for their join, which
// took 26 us with a thread to four columns of a row).
template <typename T, int D, int NW = 4> struct StepGeo {
    static constexpr int LV = red_ld<T>(D), LO = D + 4;
    static constexpr size_t VB = sizeof(T) * NW * 32 * LV, OB = sizeof(float) * NW * 16 * LO;
    static constexpr size_t LDS = VB > OB ? VB : OB;
};

// EXT = kBias: the heads have biases of their own, so a lane, whose query head is r, takes them from a table in LDS; the 32 slots of a block are
// as many distances in a row, but where they hold sinks or the ring's seam.  EXT = kPrefix: the results are parts, to be joined with the prefix's.
// EXT = kEvict: the token's slot is found first, and the scores are kept until the softmax's sum is known.
// EXT = kFew: not the ring but a part of the prefix, for 16 of the few queries that share it (heads of one row or of several).
// EXT = kBoth: the blocks of the prefix, then the ring's, for the heads of one row.
// 256 rows, four key heads of 1028 slots, d = 64, bf16: with a bias 46 us for 204 MB, 4.4 TB/s; 512 rows over caches of 1024 slots with their scores 99 us for 449 MB,
// 4.5 TB/s (111 with the scores in memory, loaded one by one).  What a bias or a score costs a slot hides behind the ring's bytes.
template <typename T, int D, int EXT, int NW = 4>
__device__ __forceinline__ void window_step_part(const typename ExtStepArgs<EXT>::type& a, unsigned u, char* raw, float (&sml)[2][NW][16])
{
    typedef typename Frag<T>::type F;
    constexpr int PE = 16 / (int)sizeof(T), CH = D / PE, LV = red_ld<T>(D);
    constexpr int NV = 32 * CH / 64;  // 16-byte pieces of V of a lane
    constexpr int LO = D + 4;
    __shared__ float sB[EXT == kBias ? kMaxBuckets * 16 : 1];
    __shared__ float sfin[EXT == kEvict ? 32 : 1];
    extern __shared__ __attribute__((aligned(16))) float zlds[];  // kEvict: [heads][pitch]
    constexpr int NT = 64 * NW;
    bool whole = EXT != kPrefix && EXT != kFew && a.nsplit == 1;
    if constexpr (EXT == kEvict) whole = a.fused;

    unsigned nsplit = a.nsplit, ngrp = a.ngrp;
    if constexpr (EXT == kFew) nsplit = a.npart, ngrp = a.nqb;
    const int part = (int)(u % nsplit);
    u /= nsplit;
    const int gi = (int)(u % ngrp);
    u /= ngrp;
    const int hk = (int)(u % (unsigned)a.Hkv), grp = a.H / a.Hkv;
    int b = (int)(u / (unsigned)a.Hkv), queries = grp;  // kFew: the row is the prefix's first
    if constexpr (EXT == kFew) {
        queries *= a.B / a.G;
        b *= a.B / a.G;
    }
    const int h0 = hk * grp + 16 * gi, nh = min(16, queries - 16 * gi);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const size_t qrow = (size_t)b * a.H + h0, rows = (size_t)a.B * a.H;
    const auto row_of = [&](int i) -> size_t {  // of the workgroup's query i
        if constexpr (EXT == kFew) {
            const int x = 16 * gi + i;
            return (size_t)(b + x / grp) * a.H + hk * grp + x % grp;
        }
        return qrow + i;
    };

    int64_t pos = 0;  // kFew: of no row
    if (EXT != kFew && row_tokens(nullptr, a.pos, a.t0, b, 1, pos) == 0) {  // a row without a token
        for (int i = tid; i < nh * D; i += NT)
            if (whole) ((T*)a.o)[qrow * D + i] = (T)0.f;
        if (!whole && tid < nh) {
            const size_t at = (size_t)part * rows + qrow + tid;
            a.part_ml[2 * at] = kNoMax;
            a.part_ml[2 * at + 1] = 0.f;
        }
        if constexpr (EXT == kEvict) {
            const size_t bh = (size_t)b * a.Hkv + hk;
            if (part == 0 && gi == 0 && tid == 0) a.mine[bh] = -1;
            if (a.fused)
                for (int i = tid; i < a.W; i += NT) evict_score_out(a, bh, i, -1, 0, pos, 0.f);
        }
        return;
    }
    const int slots = a.S + a.W;
    int n = (int)min(pos + 1, (int64_t)slots);
    const size_t bh = (size_t)b * a.Hkv + hk;
    int mine;  // the token's slot
    if constexpr (EXT == kFew) {
        const int gx = b / (a.B / a.G);
        n = a.plen ? min(max(a.plen[gx], 0), a.P) : a.P;
        mine = -1;
    } else if constexpr (EXT == kEvict)
        mine = pos < slots ? (int)pos : evict_slot<NW>(a.score_in + bh * slots, a.at_in + bh * slots, slots, pos - a.recent, (uint64_t*)raw);
    else
        mine = pos < a.S ? (int)pos : a.S + (int)((pos - a.S) % a.W);
    const T *kn = (const T*)a.k + bh * D, *vn = (const T*)a.v + bh * D;
    T *ck = (T*)a.ck + bh * slots * D, *cv = (T*)a.cv + bh * slots * D;
    if constexpr (EXT == kFew) {
        const size_t at = ((size_t)(b / (a.B / a.G)) * a.Hkv + hk) * a.P * D;
        ck = (T*)a.pk + at, cv = (T*)a.pv + at;  // only read
    }
    if (EXT != kFew && part == 0 && gi == 0 && tid < 2 * CH) {
        const int ch = tid % CH;
        if (tid < CH)
            *(intx4*)(ck + (size_t)mine * D + ch * PE) = *(const intx4*)(kn + ch * PE);
        else
            *(intx4*)(cv + (size_t)mine * D + ch * PE) = *(const intx4*)(vn + ch * PE);
    }

    int np = 0, pblk = 0;  // kBoth: the prefix's tokens, and their blocks ahead of the ring's
    const T *pk = nullptr, *pv = nullptr;
    if constexpr (EXT == kBoth) {
        const int gx = b / (a.B / a.G);
        np = a.plen ? min(max(a.plen[gx], 0), a.P) : a.P;
        pblk = (np + 31) / 32;
        const size_t at = ((size_t)gx * a.Hkv + hk) * a.P * D;
        pk = (const T*)a.pk + at, pv = (const T*)a.pv + at;
    }
    const int nblk = pblk + (n + 31) / 32, each = (nblk + (int)nsplit - 1) / (int)nsplit;
    const int bb = part * each, be = min(nblk, bb + each);

    F qf[D / 32];
    {
        const T* q = (const T*)a.q + row_of(min(r, nh - 1)) * D;
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

    BiasLanes lanes = {};
    int pm = -1;                            // the token's slot of the ring, counted from its first
    if constexpr (EXT == kBias) {
        lanes.set_edges(a.spec, lane);
        for (int i = tid; i < a.spec.buckets * 16; i += NT) {
            const float x = a.spec.bias[(size_t)(h0 + min(i & 15, nh - 1)) * a.spec.buckets + (i >> 4)];
            sB[i] = x < kBiasNone ? -INFINITY : x * kLog2e;
        }
        if (pos >= a.S) pm = mine - a.S;
        __syncthreads();
    }
    const float sx = EXT == kBias ? 1.f : sc;  // what takes a score to the base-2 domain

    T* sV = (T*)raw + wave * 32 * LV;
    F kf[2][D / 32];
    intx4 vr[NV];
    auto load = [&](int blk) {
        const bool pre = EXT == kBoth && blk < pblk;
        const int first = pre ? 32 * blk : 32 * (blk - pblk), last = (pre ? np : n) - 1;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const int i = min(first + 16 * kt + r, last);
            const T* row = pre ? pk + (size_t)i * D : i == mine ? kn : ck + (size_t)i * D;
#pragma unroll
            for (int kb = 0; kb < D / 32; ++kb) kf[kt][kb] = ld_nat(row, kb, g);
        }
#pragma unroll
        for (int x = 0; x < NV; ++x) {
            const int i = min(first + (x * 64 + lane) / CH, last);
            const T* row = pre ? pv + (size_t)i * D : i == mine ? vn : cv + (size_t)i * D;
            vr[x] = *(const intx4*)(row + ((x * 64 + lane) % CH) * PE);
        }
    };

    floatx4 acc[D / 16];
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) acc[dt] = zero4();
    float mx = kNoMax, sum = 0.f;
    int blk = bb + wave;
    if (blk < be) load(blk);
    for (; blk < be; blk += NW) {
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
        if (blk + NW < be) load(blk + NW);
        if constexpr (EXT == kBias) {
            const int i0 = 32 * blk, i1 = i0 + 31;
            int ulo = 0, uhi = a.spec.buckets - 1;
            if (i1 < a.S) {  // distances past 2^30 are in the last bucket
                ulo = lanes.bucket((int)min(pos - i1, (int64_t)1 << 30));
                uhi = lanes.bucket((int)min(pos - i0, (int64_t)1 << 30));
            } else if (i0 >= a.S && (i1 - a.S <= pm || i0 - a.S > pm)) {
                const int wrap = i0 - a.S > pm ? a.W : 0;
                ulo = lanes.bucket(pm - (i1 - a.S) + wrap);
                uhi = lanes.bucket(pm - (i0 - a.S) + wrap);
            }
            float bv[8];
            const float b0 = sB[ulo * 16 + r];
#pragma unroll
            for (int e = 0; e < 8; ++e) bv[e] = b0;
            if (ulo != uhi) {
                int d[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = i0 + 16 * (e >> 2) + 4 * g + (e & 3), x = pm - (i - a.S);
                    d[e] = i < a.S ? (int)min(pos - i, (int64_t)1 << 30) : x + (x < 0 ? a.W : 0);
                }
                for (int w = ulo + 1; w <= uhi; ++w) {
                    const int edge = lanes.first(w);
                    const float x = sB[w * 16 + r];
#pragma unroll
                    for (int e = 0; e < 8; ++e) bv[e] = d[e] >= edge ? x : bv[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e >> 2][e & 3] = __builtin_fmaf(s[e >> 2][e & 3], sc, bv[e]);
        }
        const int left = EXT == kBoth && blk < pblk ? np - 32 * blk : n - 32 * (blk - pblk);  // tokens from here on
        if (left < 32) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[kt][e] = 16 * kt + 4 * g + e < left ? s[kt][e] : -INFINITY;
        }
        if constexpr (EXT == kEvict) {
            if (r < nh) {
                if (a.in_lds) {
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt) st4f(zlds + r * a.pitch + 32 * blk + 16 * kt + 4 * g, s[kt] * sc);
                } else {
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt) st4f(a.z + (qrow + r) * a.pitch + 32 * blk + 16 * kt + 4 * g, s[kt] * sc);
                }
            }
        }
        float m = kNoMax;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) m = fmaxf(m, fmaxf(fmaxf(s[kt][0], s[kt][1]), fmaxf(s[kt][2], s[kt][3])));
        m = fmaxf(mx, rows_max(m));
        const float al = exp2_fast((mx - m) * sx), nm = -m * sx;
        mx = m;
        sum *= al;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[kt][e] = exp2_fast(__builtin_fmaf(s[kt][e], sx, nm));
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
        sml[0][wave][r] = mx * sx;
        sml[1][wave][r] = sum;
    }
    __syncthreads();
    for (int i = tid; i < nh * (D / 4); i += NT) {
        const int hq = i / (D / 4), c = 4 * (i % (D / 4));
        float m = kNoMax * sx;
#pragma unroll
        for (int w = 0; w < NW; ++w) m = fmaxf(m, sml[0][w][hq]);
        float l = 0.f;
        floatx4 o = zero4();
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = exp2_fast(sml[0][w][hq] - m);
            l += f * sml[1][w][hq];
            o += f * ld4f(sO + (w * 16 + hq) * LO + c);
        }
        if (EXT == kEvict && c == 0) {
            sfin[hq] = m;
            sfin[16 + hq] = 1.f / l;
        }
        if (whole) {
            st4((T*)a.o + (qrow + hq) * D + c, EXT != kBias || l > 0.f ? o * (1.f / l) : zero4());
        } else {
            const size_t at = (size_t)part * rows + row_of(hq);
            float *to = a.part_o, *ml = a.part_ml;
            if constexpr (EXT == kFew) {
                to = a.pre_o, ml = a.pre_ml;
                int64_t at_row;
                if (row_tokens(nullptr, a.pos, a.t0, b + (16 * gi + hq) / grp, 1, at_row) == 0) l = 0.f;
            }
            st4f(to + at * D + c, o);
            if (c == 0) {
                ml[2 * at] = m;
                ml[2 * at + 1] = l;
            }
        }
    }
    if constexpr (EXT == kEvict) {
        if (!a.fused) {
            if (part == 0 && gi == 0 && tid == 0) a.mine[bh] = mine;
            return;
        }
        __syncthreads();  // sfin, and the scores that the waves have written
        for (int i = tid; i < slots; i += NT) {
            float w = 0.f;
            if (i < n) {
                if (a.in_lds)
                    for (int h = 0; h < nh; ++h) w += exp2_fast(zlds[h * a.pitch + i] - sfin[h]) * sfin[16 + h];
                else
                    for (int h = 0; h < nh; ++h) w += exp2_fast(a.z[(qrow + h) * a.pitch + i] - sfin[h]) * sfin[16 + h];
            }
            evict_score_out(a, bh, i, mine, n, pos, w);
        }
    }
}

template <typename T, int D, int EXT, int NW> __global__ void __launch_bounds__(64 * NW) window_step_kernel(typename ExtStepArgs<EXT>::type a)
{
    __shared__ __attribute__((aligned(16))) char raw[StepGeo<T, D, NW>::LDS];
    __shared__ float sml[2][NW][16];
    window_step_part<T, D, EXT, NW>(a, blockIdx.x, raw, sml);
}

// waves: of a workgroup, 4, or 8 where the call adds to window attention.
template <typename T, int D, int EXT> hipError_t step_d(const typename ExtStepArgs<EXT>::type& a, int waves, hipStream_t s)
{
    size_t more = 0;
    if constexpr (EXT == kEvict)
        if (a.in_lds) more = sizeof(float) * (a.H / a.Hkv) * a.pitch;
    const dim3 grid((unsigned)((long long)a.B * a.Hkv * a.ngrp * a.nsplit));
    if constexpr (EXT != kPlain)
        if (waves == 8) {
            hipLaunchKernelGGL((window_step_kernel<T, D, EXT, 8>), grid, dim3(512), more, s, a);
            return hipGetLastError();
        }
    hipLaunchKernelGGL((window_step_kernel<T, D, EXT, 4>), grid, dim3(256), more, s, a);
    return hipGetLastError();
}

}  // namespace bla
