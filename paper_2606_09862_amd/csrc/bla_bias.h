// A learned bias of each head and bucket of distance: what the kernels that add it share.
//
// Bucket n of a distance is the number of edges at or below it: bucket u holds the distances edges[u - 1] .. edges[u] - 1.  There are at most 64
// buckets, so a wave holds them in two registers, an edge and a bias to each lane: a distance that is the same in every lane finds its
// bucket with a comparison and a count of the lanes.
#pragma once

#include "bla_seq.h"

namespace bla {

constexpr int kMaxBuckets = 64;
constexpr int kNear = 1024;          // distances that have a table in LDS
constexpr int kPad = 64;             // places before them, for pairs of later keys in a tile that the masks hide
// A bias below it counts as minus infinity: its pairs have no weight.  Past 2^20 or so a score's last bits are gone in float32, and the maximum that a kernel
// forms from a tile's largest product would be off by more than its exponentials bear.
constexpr float kBiasNone = -1e6f;

// The least and the largest distance between 32 keys and a wave's queries.  Keys and queries have indices whose difference is their distance, but for
// keys at negative indices (sinks ahead of the window), which are `far` further away.  qi: the first query, i0: the first key.
struct BiasSpan {
    int lo, hi;
};
__host__ __device__ inline BiasSpan bias_span(int qi, int queries, int i0, int far)
{
    const int i1 = i0 + 31;
    return {qi - i1 + (i1 < 0 ? far : 0), qi + queries - 1 - i0 + (i0 < 0 ? far : 0)};
}
// Whether a span whose ends have different buckets takes its biases from the table: keys on both sides of index 0 are not one run of distances.
__host__ __device__ inline bool bias_near(BiasSpan d, int i0) { return d.hi < kNear && (i0 >= 0 || i0 + 31 < 0); }
// How far the table is written, `last` being the last edge: a span of 63 distances or fewer whose ends have different buckets begins below it.
__host__ __device__ inline int bias_table_end(int last) { return kNear < last + 64 ? kNear : last + 64; }

struct BiasSpec {
    const float* bias;  // [H, buckets]
    int buckets;
    int32_t edges[kMaxBuckets - 1];
};

// The buckets of one head in a wave.
struct BiasLanes {
    int edge;    // of lane u: the first distance of bucket u + 1
    float bias;  // of lane u: that of bucket u, in the base-2 domain

    __device__ __forceinline__ void set_edges(const BiasSpec& a, int lane)
    {
        edge = lane < a.buckets - 1 ? a.edges[lane] : INT32_MAX;
    }
    __device__ __forceinline__ void set_head(const BiasSpec& a, int h, int lane)
    {
        const float x = lane < a.buckets ? a.bias[(size_t)h * a.buckets + lane] : 0.f;
        bias = x < kBiasNone ? -INFINITY : x * kLog2e;
    }
    // the bucket of a distance that is the same in every lane
    __device__ __forceinline__ int bucket(int n) const { return __popcll(__ballot(edge <= n)); }
    // u: the same in every lane
    __device__ __forceinline__ float of(int u) const { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(bias), u)); }
    __device__ __forceinline__ int first(int u) const { return __builtin_amdgcn_readlane(edge, u - 1); }
    // 64 distances from n0 on, the lane's n0 + lane: f(its bucket, that bucket's bias)
    template <typename Fn> __device__ __forceinline__ void each(int n0, int lane, Fn f) const
    {
        const int lo = bucket(n0), hi = bucket(n0 + 63);
        int u = lo;
        float x = of(lo);
        for (int w = lo + 1; w <= hi; ++w) {
            const bool in = n0 + lane >= first(w);
            u = in ? w : u;
            x = in ? of(w) : x;
        }
        f(u, x);
    }
    // The table of the near distances, as far as two of a tile's can have different buckets: each wave of the workgroup writes some of it.
    __device__ __forceinline__ void table(const BiasSpec& a, float* near, int wave, int waves, int lane) const
    {
        const int last = a.buckets > 1 ? a.edges[a.buckets - 2] : 0;
        if (wave == 0) near[lane] = of(0);
        for (int c = wave; 64 * c < bias_table_end(last); c += waves)
            each(64 * c, lane, [&](int, float x) { near[kPad + 64 * c + lane] = x; });
    }
};

// The scores s of 32 keys (rows) from index i0 on and 16 QT queries (columns) from index qi on, of S^T = K Q^T: where all pairs share a bucket they stay as they are,
// the score in the base-2 domain being s sx + bu; elsewhere they take their biases and go there, from the table where it holds them, or by a selection at each edge.
template <int QT>
__device__ __forceinline__ void bias_scores(floatx4 (&s)[QT][2], float& sx, float& bu, const BiasLanes& lanes, const float* near, float sc, int qi,
                                            int i0, int far, int g, int r)
{
    const BiasSpan span = bias_span(qi, 16 * QT, i0, far);
    const int ulo = lanes.bucket(span.lo), uhi = lanes.bucket(span.hi);
    bu = lanes.of(ulo);
    if (ulo == uhi) return;
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        float bv[8];
        const int n = qi + 16 * qt + r - i0 - 4 * g;  // of the lane's first key
        if (bias_near(span, i0)) {
            const float* from = near + kPad + n + (i0 < 0 ? far : 0);
#pragma unroll
            for (int e = 0; e < 8; ++e) bv[e] = from[-16 * (e >> 2) - (e & 3)];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) bv[e] = bu;
            for (int w = ulo + 1; w <= uhi; ++w) {
                const int edge = lanes.first(w);
                const float x = lanes.of(w);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int m = n - 16 * (e >> 2) - (e & 3), j = i0 + 4 * g + 16 * (e >> 2) + (e & 3);
                    bv[e] = m + (j < 0 ? far : 0) >= edge ? x : bv[e];
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) s[qt][e >> 2][e & 3] = __builtin_fmaf(s[qt][e >> 2][e & 3], sc, bv[e]);
    }
    sx = 1.f, bu = 0.f;
}

}  // namespace bla
