// Attention over a cache of bounded size that gives up its tokens of least weight: kernel arguments.
#pragma once

#include "bla_window_step.h"

namespace bla {

// The weight that each token gets from the queries of a call.
struct EvictSumArgs {
    const void *q, *k, *ck;    // [B, H, L, D], [B, Hkv, L, D], [B, Hkv, slots, D] or null
    const float* lse;          // [B, H, L]
    const int32_t* lengths;
    const int64_t* pos;
    int64_t t0;
    int B, H, Hkv, L, slots;
    float scale;
    int ncb, nkb;              // key blocks of the cache, of cache and call together
    long long units, per;
    float* part;               // [B, H, slots + L]
    const float* score_in;     // [B, Hkv, slots] or null
    float* score_out;          // [B, Hkv, slots + L]
};

struct EvictSelectArgs {
    const void *k, *v, *ck, *cv;
    const float* score;        // [B, Hkv, slots + L]
    const int64_t* at_in;      // [B, Hkv, slots] or null
    const int32_t* lengths;
    const int64_t* pos;
    int64_t t0;
    int B, Hkv, L, slots, recent;
    int slices, pieces;        // workgroups of a key head, pieces of 16 bytes of a key
    void *ck_out, *cv_out;
    float* score_out;
    int64_t* at_out;
};

hipError_t launch_evict_sum(int bf16_io, int D, const EvictSumArgs& a, hipStream_t s);
hipError_t launch_evict_select(const EvictSelectArgs& a, hipStream_t s);
hipError_t launch_evict_step(int bf16_io, int D, const EvictStepArgs& a, int waves, hipStream_t s);
// Bytes of scores that a workgroup of the step keeps in LDS: four such workgroups fill a compute unit's registers at d = 64.  The tiles of eight waves take 133 KiB of
// the 160 in float32 at d = 128.
constexpr int score_lds(int waves, bool bf16_io, int D) { return waves == 8 && !bf16_io && D == 128 ? 16 * 1024 : 32 * 1024; }
constexpr int kEvictKeys = 128;    // keys of a workgroup of the sums
constexpr int kSliceSlots = 4096;  // most slots of a slice of the selection

}  // namespace bla
