// The weight that each token of a cache and of a call gets from the call's queries (bla_evict_forward), and the tokens that stay
// (bla_evict_select).
#include "bla_evict.h"

namespace bla {
namespace {

// Sums over the queries of P = exp(scale q k - lse).  Every lse has to be known first, so the scores are formed again, once for each head.  Wave w of a
// workgroup owns 32 keys of one head's key block, whose K are operands in registers for the whole walk over 64-query tiles; S = Q K^T (accumulator rows:
// queries) leaves each lane four queries of a key, whose weights it adds up in float32.  The heads of a group are added up by evict_sum_out_kernel, in order.
// Bound: issue, of one product instead of two and as many exponentials as attention itself (2 x 16 heads x 4096 queries over themselves, d = 64, bf16: 57 us beside
// 102 for the attention; the heads' sum 5).
template <typename T, int D> struct SumGeo {
    static constexpr int NT = 256, PE = 16 / (int)sizeof(T), CH = D / PE, RPP = NT / CH, NP = (64 + RPP - 1) / RPP;
    static constexpr int KT = 2, LD = nat_ld<T>(D);
};

template <typename T, int D> __global__ void __launch_bounds__(256) evict_sum_kernel(EvictSumArgs a)
{
    typedef SumGeo<T, D> G;
    typedef typename Frag<T>::type F;
    constexpr int KT = G::KT, BUF = 64 * G::LD;
    static_assert(64 * KT == kEvictKeys, "keys of a workgroup");
    __shared__ __attribute__((aligned(16))) T lds[2 * BUF];
    __shared__ __attribute__((aligned(16))) float sl[2][64];

    const long long u = falling_unit(blockIdx.x, a.units);  // the first keys have most queries
    if (u >= a.units) return;
    const long long bh = u % ((long long)a.B * a.H);
    const int nb = (int)(u / ((long long)a.B * a.H)), h = (int)(bh % a.H), b = (int)(bh / a.H), hk = h / (a.H / a.Hkv);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    int64_t pos;
    const int len = row_tokens(a.lengths, a.pos, a.t0, b, a.L, pos);
    const bool old = nb < a.ncb;
    const int k0 = (old ? nb : nb - a.ncb) * kEvictKeys + 16 * KT * wave, kend = k0 + 16 * KT - 1;  // the wave's keys
    const int there = old ? (len > 0 ? (int)min(pos, (int64_t)a.slots) : 0) : len;                // keys of the cache or of the call
    const int n0 = old ? 0 : (nb - a.ncb) * kEvictKeys;                                            // the walk's first query
    const int nt = len > n0 && there > k0 - 16 * KT * wave ? (len - n0 + 63) / 64 : 0;

    const T* kp = old ? (const T*)a.ck + ((size_t)b * a.Hkv + hk) * a.slots * D : (const T*)a.k + ((size_t)b * a.Hkv + hk) * a.L * D;
    F kf[KT][D / 32];
    float run[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        run[kt] = 0.f;
        const int j = k0 + 16 * kt + r;
#pragma unroll
        for (int kb = 0; kb < D / 32; ++kb) kf[kt][kb] = j < there ? ld_nat(kp + (size_t)j * D, kb, g) : zero_frag<T>();
    }
    const float sc = a.scale * kLog2e;
    const int ch = tid % G::CH, lrow = tid / G::CH;
    const size_t row0 = ((size_t)b * a.H + h) * a.L;
    const T* qp = (const T*)a.q + row0 * D + ch * G::PE;
    intx4 qr[G::NP];
    float st = 0.f;
    auto load = [&](int t) {  // queries past the row's last repeat it: the masks hide them
        const int q0 = n0 + 64 * t;
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            if (G::RPP > 64 && lrow >= 64) continue;
            qr[ps] = *(const intx4*)(qp + (size_t)min(q0 + ps * G::RPP + lrow, len - 1) * D);
        }
        if (tid < 64) st = a.lse[row0 + min(q0 + tid, len - 1)] * kLog2e;
    };
    if (nt > 0) load(0);
    for (int t = 0; t < nt; ++t) {
        T* sQ = lds + (t & 1) * BUF;
        float* stat = sl[t & 1];
#pragma unroll
        for (int ps = 0; ps < G::NP; ++ps) {
            if (G::RPP > 64 && lrow >= 64) continue;
            *(intx4*)(sQ + (ps * G::RPP + lrow) * G::LD + ch * G::PE) = qr[ps];
        }
        if (tid < 64) stat[tid] = st;
        __syncthreads();
        if (t + 1 < nt) load(t + 1);
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int q0 = n0 + 64 * t + 32 * hf, q1 = q0 + 31;
            if (q0 >= len || (!old && k0 > q1) || k0 >= there) continue;
            floatx4 s[KT][2];
#pragma unroll
            for (int qt = 0; qt < 2; ++qt) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) s[kt][qt] = zero4();
#pragma unroll
                for (int kb = 0; kb < D / 32; ++kb) {
                    const F qf = ld_nat(sQ + (32 * hf + 16 * qt + r) * G::LD, kb, g);
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) s[kt][qt] = mma(qf, kf[kt][kb], s[kt][qt]);
                }
                const floatx4 lse2 = ld4f(stat + 32 * hf + 16 * qt + 4 * g);
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[kt][qt][e] = exp2_fast(__builtin_fmaf(s[kt][qt][e], sc, -lse2[e]));
            }
            if ((!old && kend > q0) || q1 >= len) {  // some pair is not visible (selects without branches, as in window_forward_kernel)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    const int from = old ? 0 : k0 + 16 * kt + r, q = q0 + 4 * g;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int x = q + 16 * (e >> 2) + (e & 3);
                        s[kt][e >> 2][e & 3] = ((x >= from) & (x < len)) ? s[kt][e >> 2][e & 3] : 0.f;
                    }
                }
            }
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                float x = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) x += s[kt][e >> 2][e & 3];
                run[kt] += x;
            }
        }
    }
    const size_t to = ((size_t)b * a.H + h) * ((size_t)a.slots + a.L) + (old ? 0 : a.slots);
    const int most = old ? a.slots : a.L;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        const float x = rows_sum(run[kt]);
        const int j = k0 + 16 * kt + r;
        if (g == 0 && j < most) a.part[to + j] = j < there ? x : 0.f;
    }
}

// score_out = score_in + the heads' sums, in the order of the heads; zeros where there is no token.
__global__ void __launch_bounds__(256) evict_sum_out_kernel(EvictSumArgs a)
{
    const size_t n = (size_t)a.slots + a.L, i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (size_t)a.B * a.Hkv * n) return;
    const size_t bh = i / n, e = i % n;
    const int grp = a.H / a.Hkv, b = (int)(bh / a.Hkv), hk = (int)(bh % a.Hkv);
    int64_t pos;
    const int len = row_tokens(a.lengths, a.pos, a.t0, b, a.L, pos);
    const bool idle = pos < 0 || pos > kMaxPos;  // such a row's cache stays as it is, its scores with it
    float x = 0.f;
    if (e >= (size_t)a.slots || (a.ck && (idle || (int64_t)e < pos))) {
        if (len > 0 || e >= (size_t)a.slots)
            for (int h = 0; h < grp; ++h) x += a.part[((size_t)b * a.H + hk * grp + h) * n + e];
        if (e < (size_t)a.slots) x += a.score_in[bh * a.slots + e];
    }
    a.score_out[i] = x;
}

// Which entries stay, and their way to the cache.  A workgroup of 16 waves takes one key head of one row and moves a slice of the slots: several find the
// same in parallel, which costs nothing where the key heads do not fill the device, and a second launch would cost more.  An entry's key is its score's place in the order of scores, the
// largest of all for the newest `recent` tokens; counts of its upper 11, next 11 and last 10 bits (by integer atomics in LDS, whose order does not
// matter) find the key of the last entry that stays, of which the lowest entries fill the slots.  Once all entries with the bits found so far stay, no further bits are
// looked at.  Then each wave walks a sixteenth of the entries in order, first to count, then to number those that stay.
// Bound: latency: two or three counts, as many scans and two dependent loads (1024 of 4096 entries for 32 key heads, d = 64: 12.4 us, 1.5 TB/s; a launch to choose and one
// to move 18.7; loads one by one and always three counts 14.1).  With as many key heads as compute units it is bound by memory (32 rows of 8, d = 128: 53 us, 5.1 TB/s).
__device__ __forceinline__ void move_slice(const EvictSelectArgs& a, size_t bh, int64_t pos, int s0, int s1, const int* index)
{
    const intx4 *ck = (const intx4*)a.ck + bh * a.slots * a.pieces, *cv = (const intx4*)a.cv + bh * a.slots * a.pieces;
    const intx4 *k = (const intx4*)a.k + bh * a.L * a.pieces, *v = (const intx4*)a.v + bh * a.L * a.pieces;
    const size_t to = bh * a.slots + s0;
    const int shift = __builtin_ctz(a.pieces);  // 4, 8, 16 or 32
    for (int i = threadIdx.x; i < (s1 - s0) << shift; i += 1024) {  // a piece of 16 bytes of a key and of a value to a thread
        const int e = index[i >> shift], c = i & (a.pieces - 1);
        intx4 kx = {0, 0, 0, 0}, vx = {0, 0, 0, 0};
        if (e >= a.slots) {
            kx = k[((size_t)(e - a.slots) << shift) + c];
            vx = v[((size_t)(e - a.slots) << shift) + c];
        } else if (e >= 0) {
            kx = ck[((size_t)e << shift) + c];
            vx = cv[((size_t)e << shift) + c];
        }
        ((intx4*)a.ck_out)[(to << shift) + i] = kx;
        ((intx4*)a.cv_out)[(to << shift) + i] = vx;
    }
    for (int i = threadIdx.x; i < s1 - s0; i += 1024) {
        const int e = index[i];
        a.score_out[to + i] = e >= 0 ? a.score[bh * ((size_t)a.slots + a.L) + e] : 0.f;
        a.at_out[to + i] = e >= a.slots ? pos + (e - a.slots) : e >= 0 ? a.at_in[bh * a.slots + e] : -1;
    }
}

constexpr int kSelWaves = 16, kSelLds = 24 * 1024;  // entries whose keys are kept in LDS; those beyond are formed anew

__global__ void __launch_bounds__(1024) evict_select_kernel(EvictSelectArgs a)
{
    __shared__ unsigned keys[kSelLds];
    __shared__ int hist[3][2048];
    __shared__ int wsum[2][kSelWaves];
    __shared__ int found[3][3];
    __shared__ int index[kSliceSlots];  // the slice's entries
    const size_t bh = blockIdx.x / a.slices;
    const int slice = (int)(blockIdx.x % a.slices), each_slice = (a.slots + a.slices - 1) / a.slices;
    const int s0 = slice * each_slice, s1 = min(a.slots, s0 + each_slice);
    const int b = (int)(bh / a.Hkv), tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    int64_t pos;
    const int len = row_tokens(a.lengths, a.pos, a.t0, b, a.L, pos);
    const bool idle = pos < 0 || pos > kMaxPos;
    const int n = a.ck && !idle ? (int)min(pos, (int64_t)a.slots) : 0, total = n + len;
    if (idle || total <= a.slots) {  // everything stays
        for (int i = s0 + tid; i < s1; i += 1024)
            index[i - s0] = idle ? (a.ck ? i : -1) : i < n ? i : i < total ? a.slots + i - n : -1;
        __syncthreads();
        move_slice(a, bh, pos, s0, s1, index);
        return;
    }
    const float* score = a.score + bh * ((size_t)a.slots + a.L);
    const int64_t* at = a.at_in ? a.at_in + bh * a.slots : nullptr;
    const int64_t late = pos + len - a.recent;  // the first position that stays in any case
    float es[4];
    int64_t ep[4];
    auto fetch = [&](int i0) {  // four entries, all loads in flight; one past the last is the last again
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = min(i0 + 1024 * k, total - 1);
            es[k] = score[i < n ? i : a.slots + i - n];
            ep[k] = pos + (i - n);
        }
        if (n > 0)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t old = at[min(i0 + 1024 * k, n - 1)];
                ep[k] = i0 + 1024 * k < n ? old : ep[k];
            }
    };
    auto fetched = [&](int k) { return ep[k] >= late ? 0xffffffffu : score_key(es[k]); };
    auto key = [&](int i) {
        if (i < kSelLds) return keys[i];
        const int64_t p = i < n ? at[i] : pos + (i - n);
        return p >= late ? 0xffffffffu : score_key(score[i < n ? i : a.slots + i - n]);
    };
    fetch(tid);
    for (int i = tid; i < 3 * 2048; i += 1024) (&hist[0][0])[i] = 0;
    __syncthreads();
    for (int i0 = tid; i0 < total;) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + 1024 * k;
            if (i >= total) continue;
            const unsigned x = fetched(k);
            if (i < kSelLds) keys[i] = x;
            atomicAdd(&hist[0][x >> 21], 1);
        }
        i0 += 4096;
        if (i0 < total) fetch(i0);
    }

    unsigned prefix = 0;    // the upper bits of the last key that stays
    int need = a.slots;     // entries that stay among those with these bits
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
        if (pass > 0)
            for (int i = tid; i < total; i += 1024) {
                const unsigned x = key(i);
                if (x >> (pass == 1 ? 21 : 10) == prefix) atomicAdd(&hist[pass][(x >> shift) & (bins - 1)], 1);
            }
        __syncthreads();
        // the bin in which the count from above passes `need`: two bins a thread, the highest first
        const int t0 = bins - 1 - 2 * tid, c0 = t0 >= 0 ? hist[pass][t0] : 0, c1 = t0 >= 1 ? hist[pass][t0 - 1] : 0;
        int x = c0 + c1;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int y = __shfl_up(x, off);
            if (lane >= off) x += y;
        }
        if (lane == 63) wsum[0][wave] = x;
        __syncthreads();
        int above = x - c0 - c1;
        for (int w = 0; w < wave; ++w) above += wsum[0][w];
        if (above < need && above + c0 + c1 >= need) {
            const bool first = above + c0 >= need;
            found[pass][0] = first ? t0 : t0 - 1;
            found[pass][1] = need - above - (first ? 0 : c0);
            found[pass][2] = first ? c0 : c1;
        }
        __syncthreads();
        prefix = pass == 2 ? prefix << 10 | (unsigned)found[pass][0] : pass == 1 ? prefix << 11 | (unsigned)found[pass][0] : (unsigned)found[pass][0];
        need = found[pass][1];
        if (pass < 2 && need == found[pass][2]) {  // every key with these bits stays, some below them do not, so the bits are not zeros
            prefix = (prefix << shift) - 1, need = 0;
            break;
        }
    }
    const int each = ((total + kSelWaves - 1) / kSelWaves + 63) & ~63, i0 = wave * each, i1 = min(total, i0 + each);
    int more = 0, same = 0;
    for (int i = i0; i < i1; i += 64) {
        const unsigned x = i + lane < i1 ? key(i + lane) : 0u;
        more += __popcll(__ballot(i + lane < i1 && x > prefix));
        same += __popcll(__ballot(i + lane < i1 && x == prefix));
    }
    if (lane == 0) wsum[0][wave] = more, wsum[1][wave] = same;
    __syncthreads();
    more = same = 0;
    for (int w = 0; w < wave; ++w) more += wsum[0][w], same += wsum[1][w];
    int out = more + min(same, need);
    const unsigned long long below = (1ull << lane) - 1;
    for (int i = i0; i < i1; i += 64) {
        const bool in = i + lane < i1;
        const unsigned x = in ? key(i + lane) : 0u;
        const unsigned long long eq = __ballot(in && x == prefix);
        const bool stay = in && (x > prefix || (x == prefix && same + __popcll(eq & below) < need));
        const unsigned long long kept = __ballot(stay);
        const int slot = out + __popcll(kept & below);
        if (stay && slot >= s0 && slot < s1) index[slot - s0] = i + lane < n ? i + lane : a.slots + i + lane - n;
        same += __popcll(eq);
        out += __popcll(kept);
    }
    __syncthreads();
    move_slice(a, bh, pos, s0, s1, index);
}

template <typename T, int D> hipError_t sum_d(const EvictSumArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((evict_sum_kernel<T, D>), dim3((unsigned)(8 * a.per)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_evict_sum(int bf16_io, int D, const EvictSumArgs& a, hipStream_t s)
{
#define BLA_CALL(T, DD) sum_d<T, DD>(a, s)
    const auto sum = [&]() -> hipError_t { BLA_BY_TYPE(BLA_CALL) };
#undef BLA_CALL
    if (a.units > 0)
        if (const hipError_t e = sum(); e != hipSuccess) return e;
    const long long n = (long long)a.B * a.Hkv * ((long long)a.slots + a.L);
    hipLaunchKernelGGL(evict_sum_out_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_evict_select(const EvictSelectArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)((long long)a.B * a.Hkv * a.slices)), dim3(1024), 0, s, a);
    return hipGetLastError();
}

}  // namespace bla
