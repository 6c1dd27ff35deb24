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
        for (int c = wave; 64 * c < min(kNear, last + 64); c += waves)
            each(64 * c, lane, [&](int, float x) { near[kPad + 64 * c + lane] = x; });
    }
};

}  // namespace bla
