// Window attention: kernel arguments and what its kernels share.
//
// A query at position p sees the keys at positions j <= p with p - j < window, and those with j < sinks.
// The past of a row lies in a ring of sinks + window slots: position j in slot j while j < sinks, else in
// slot sinks + (j - sinks) mod window.
#pragma once

#include "bla_seq.h"

namespace bla {

constexpr int64_t kMaxPos = int64_t(1) << 62;  // positions past it (and negative ones) mark a row without tokens
constexpr float kNoMax = -1e30f;               // the running maximum before the first visible key
constexpr int kWinKeys = 64;                   // keys per tile

struct WindowArgs {
    const void *q, *k, *v;          // [B, H, L, D], [B, Hkv, L, D]
    const void *ck, *cv;            // rings before the call [B, Hkv, sinks + window, D], or null
    void* o;
    float* lse;                     // [B, H, L] or null
    void *ck_out, *cv_out;          // rings after the call, or null
    const int32_t* lengths;         // [B] or null
    const int64_t* pos;             // [B] or null
    int64_t t0;
    int B, H, Hkv, L, W, S;
    float scale;                    // softmax scale
    int nqb, nsplit;                // query blocks of a sequence, parts of a block's keys
    long long units, per;           // workgroups with work, per XCD
    float *part_o, *part_ml;        // parts: [nsplit][B H L][D] unnormalised outputs, [nsplit][B H L][2] maximum and sum
};

struct WindowStepArgs {
    const void *q, *k, *v;          // [B, H, D], [B, Hkv, D]
    void *ck, *cv, *o;
    const int64_t* pos;
    int64_t t0;
    int B, H, Hkv, W, S;
    float scale;
    int ngrp, nsplit;               // groups of 16 query heads of a key head, parts of the ring
    float *part_o, *part_ml;        // [nsplit][B H][D], [nsplit][B H][2]
};

struct WindowBwdArgs {
    const void *q, *k, *v, *o, *dO; // o: the forward's outputs
    const float* lse;
    void *dq, *dk, *dv;
    const int32_t* lengths;
    int B, H, Hkv, L, W, S;
    float scale;
    float* delta;                   // [B, H, L]: sum of dO o
    int nqb, nkb;                   // query and key blocks of a sequence
    int ns, ssplit;                 // sinks of a sequence, parts of the queries that see them from beyond their windows
    float *near, *part;             // float32 dk and dv of the sinks: [B Hkv][ns][2][D], [ssplit][B Hkv][ns][2][D]
    long long q_units, q_per, k_units, k_per;
    unsigned s_units;               // workgroups of the sinks' far queries
};

// Tokens of row b in this call, and the position of its first.
__device__ __forceinline__ int row_tokens(const int32_t* lengths, const int64_t* pos, int64_t t0, int b, int L, int64_t& p)
{
    p = pos ? pos[b] : t0;
    if (p < 0 || p > kMaxPos) return 0;
    return lengths ? min(max(lengths[b], 0), L) : L;
}

hipError_t launch_window_forward(int bf16_io, int D, int waves, const WindowArgs& a, hipStream_t s);
hipError_t launch_window_step(int bf16_io, int D, const WindowStepArgs& a, hipStream_t s);
hipError_t launch_window_backward(int bf16_io, int D, const WindowBwdArgs& a, hipStream_t s);
int window_bwd_block(int D);  // queries (keys) per block of the query (key) pass

// Join of nsplit (at most 64) parts of a softmax: o = sum_s e^{m_s - m} O_s / sum_s e^{m_s - m} l_s (m in the base-2 domain).
struct JoinArgs {
    const float *part_o, *part_ml;
    void* o;
    float* lse;       // or null
    long long rows;
    int nsplit;
};
hipError_t launch_window_join(int bf16_io, int D, const JoinArgs& a, hipStream_t s);

}  // namespace bla
