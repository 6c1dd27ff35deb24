// Window attention: argument checks and work split, for its own calls and for those that add to them.
#pragma once

#include "bla_window.h"

namespace bla {

// Workgroups that fill the device twice over (256 compute units).  With fewer, a block's keys are split into parts.
constexpr long long kFill = 512;
constexpr int kMaxParts = 64;

inline bla_status check(const bla_window_params* p, bool step)
{
    if (!p) return BLA_ERR_INVALID_ARG;
    if (p->B < 0 || p->H < 0 || p->H_kv < 0 || (!step && p->L < 0) || p->d <= 0) return BLA_ERR_INVALID_ARG;
    if (p->window < 1 || p->sinks < 0 || p->t0 < 0 || p->t0 > kMaxPos) return BLA_ERR_INVALID_ARG;
    if (p->io_dtype != BLA_F32 && p->io_dtype != BLA_BF16) return BLA_ERR_INVALID_ARG;
    if (!isfinite(p->scale)) return BLA_ERR_INVALID_ARG;
    if (p->H > 0 && (p->H_kv < 1 || p->H % p->H_kv != 0)) return BLA_ERR_INVALID_ARG;
    if (p->d != 32 && p->d != 64 && p->d != 128) return BLA_ERR_UNSUPPORTED;
    // the kernels keep the running maximum in units of the raw products and place keys by 32-bit indices
    if (p->scale != 0.f && (fabsf(p->scale) < 1e-6f || fabsf(p->scale) > 1e6f)) return BLA_ERR_UNSUPPORTED;
    if ((long long)p->window + p->sinks > (1ll << 30) || (!step && p->L > (1 << 30))) return BLA_ERR_UNSUPPORTED;
    const long long L = step ? 1 : p->L, slots = (long long)p->window + p->sinks;
    if ((double)p->B * p->H * ((L + 63) / 64) > kMaxUnits) return BLA_ERR_UNSUPPORTED;
    if ((double)p->B * p->H_kv * slots * p->d > 256.0 * (1 << 30)) return BLA_ERR_UNSUPPORTED;
    return BLA_OK;
}

inline float scale_of(const bla_window_params* p) { return p->scale == 0.f ? 1.f / sqrtf((float)p->d) : p->scale; }

// A call without rows or query heads: done, unless key heads have outputs that nothing would write.
inline bla_status empty(const bla_window_params* p, bool outputs)
{
    return outputs && p->B > 0 && p->H_kv > 0 ? BLA_ERR_UNSUPPORTED : BLA_OK;
}

// Forward: 128 queries to a workgroup (fewer reads of keys), 64 where that fills the device better;
// the keys of a block, `front` tokens that every query sees among them, in parts of at least two tiles where the blocks alone do not fill it.
struct ForwardPlan {
    int waves, nqb, nsplit;
    long long units;
    size_t total;
};
inline ForwardPlan forward_plan(const bla_window_params* p, bool cached, int front = 0)
{
    ForwardPlan f;
    const long long bh = (long long)p->B * p->H;
    f.waves = bh * ((p->L + 127) / 128) >= kFill ? 8 : 4;
    f.nqb = (p->L + 16 * f.waves - 1) / (16 * f.waves);
    const long long blocks = bh * f.nqb;
    long long keys = (long long)p->window - 1 + 16 * f.waves + p->sinks;
    if (!cached && keys > p->L) keys = p->L;
    const long long tiles = (keys + kWinKeys - 1) / kWinKeys + (front + kWinKeys - 1) / kWinKeys;
    long long n = 1;
    if (blocks > 0 && blocks < kFill) n = (kFill + blocks - 1) / blocks;
    if (n > tiles / 2) n = tiles / 2;
    f.nsplit = (int)(n < 1 ? 1 : n > kMaxParts ? kMaxParts : n);
    f.units = blocks * f.nsplit;
    f.total = f.nsplit > 1 ? seq_align((size_t)f.nsplit * bh * p->L * (p->d + 2) * 4) : 0;
    return f;
}

// whether the forward kernel's launch is one, with the workgroups that write the rings after the call
inline bool fits(const bla_window_params* p, const ForwardPlan& f, bool rings)
{
    const double pieces = (double)p->B * p->H_kv * ((double)p->window + p->sinks) * (p->d * elem_bytes(p->io_dtype) / 16);
    return launchable(8.0 * ((f.units + 7) / 8) + (rings ? ceil(pieces / (64 * f.waves)) : 0.0), 64 * f.waves);
}

// Step: a key head's ring in parts of at least 128 slots where the key heads of all rows alone do not fill the device.
struct StepPlan {
    int ngrp, nsplit;
    size_t total;
};
inline StepPlan step_plan(const bla_window_params* p)
{
    StepPlan s;
    const int grp = p->H_kv > 0 ? p->H / p->H_kv : 1;
    s.ngrp = (grp + 15) / 16;
    const long long units = (long long)p->B * p->H_kv * s.ngrp, blocks = ((long long)p->window + p->sinks + 127) / 128;
    long long n = units > 0 && units < kFill ? (kFill + units - 1) / units : 1;
    if (n > blocks) n = blocks;
    s.nsplit = (int)(n < 1 ? 1 : n > kMaxParts ? kMaxParts : n);
    s.total = s.nsplit > 1 ? seq_align((size_t)s.nsplit * p->B * p->H * (p->d + 2) * 4) : 0;
    return s;
}
// The step of the calls that add to window attention: a short ring's blocks of 32 slots go to the eight waves of one workgroup for each key head, in one launch, rather
// than in parts that a second launch joins.  With a bias and 4 key heads, one launch against parts: 1 row, d = 64 bf16, 256 slots 7.8 against 9.7 us in a graph, 9.9
// against 13.8 called; 1024 slots 10.4 against 9.8 and 10.9 against 14.4; 1536 slots 12.0 against 9.9 and 12.1 against 14.2.  d = 128 float32, 224 slots 14.5 against
// 15.2 and 14.1 against 15.5; 512 slots 24.8 against 15.2 and 24.4 against 15.5.  Key heads that need two parts to fill the device keep it busy by themselves: 36 rows,
// d = 64 bf16, 2048 slots 17.6 against 22.4 us; d = 128 float32, 1024 slots 43.3 against 57.9, but 2048 slots over an evicting cache 81.6 against 72.8.
inline bool short_ring(const bla_window_params* p, long long slots, bool many)
{
    return slots <= (many ? 2048 : 1024) && slots * p->d * elem_bytes(p->io_dtype) <= (many ? 512 : 120) * 1024;
}
struct ShortStepPlan : StepPlan {
    int waves;
};
inline ShortStepPlan short_step_plan(const bla_window_params* p)
{
    ShortStepPlan s;
    static_cast<StepPlan&>(s) = step_plan(p);
    s.waves = 4;
    const bool many = 2ll * p->B * p->H_kv * s.ngrp > kFill;
    if (s.nsplit > 1 && short_ring(p, (long long)p->window + p->sinks, many)) s.nsplit = 1, s.total = 0, s.waves = 8;
    return s;
}
inline bool fits(const bla_window_params* p, const StepPlan& s) { return launchable((double)p->B * p->H_kv * s.ngrp * s.nsplit, 256); }
inline bool fits(const bla_window_params* p, const ShortStepPlan& s) { return launchable((double)p->B * p->H_kv * s.ngrp * s.nsplit, 64 * s.waves); }

// Backward: the sinks' queries beyond their windows in as many parts as fill the device with waves, a block of 32 queries or more to each.
struct BackwardPlan {
    int nqb, nkb, ns, ssplit;
    long long q_units, k_units, s_units;
    size_t off_near, off_part, total;
};
inline BackwardPlan backward_plan(const bla_window_params* p)
{
    BackwardPlan b;
    const long long bh = (long long)p->B * p->H, bk = (long long)p->B * p->H_kv;
    const int nk = window_bwd_block(p->d);
    b.nqb = (p->L + nk - 1) / nk;
    b.nkb = (p->L + nk - 1) / nk;
    b.ns = p->sinks < p->L ? p->sinks : p->L;
    const long long wgs = bk * ((b.ns + 15) / 16), items = p->H_kv > 0 ? (long long)(p->H / p->H_kv) * ((p->L + 31) / 32) : 1;
    long long n = wgs > 0 ? (2 * kFill + wgs - 1) / wgs : 1;
    if (n > items / 4) n = items / 4;
    b.ssplit = (int)(n < 1 ? 1 : n > kMaxParts ? kMaxParts : n);
    b.q_units = bh * b.nqb;
    b.k_units = bk * b.nkb;
    b.s_units = bk * ((b.ns + 15) / 16) * b.ssplit;
    const size_t one = seq_align((size_t)bk * b.ns * 2 * p->d * 4);
    b.off_near = seq_align((size_t)bh * p->L * 4);
    b.off_part = b.off_near + one;
    b.total = b.off_part + seq_align((size_t)b.ssplit * bk * b.ns * 2 * p->d * 4);
    return b;
}

inline bool fits(const bla_window_params* p, const BackwardPlan& b)
{
    return launchable(8.0 * ((b.q_units + 7) / 8), 256) && launchable(8.0 * ((b.k_units + 7) / 8) + b.s_units, 256) &&
           launchable((double)p->B * p->H_kv * b.ns * (2 * p->d / 4) / 256 + 1, 256);
}

inline bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }


// The forward call's pointers, checked and laid down (extra: inputs of a call that adds to window attention).
template <int N>
bla_status forward_args(WindowArgs& a, const bla_window_params* p, const ForwardPlan& f, const void* q, const void* k, const void* v,
                        const int32_t* lengths, const int64_t* pos, const void* cache_k_in, const void* cache_v_in, void* o, float* lse,
                        void* cache_k_out, void* cache_v_out, const Span (&extra)[N], void* workspace, size_t workspace_bytes)
{
    const int e = elem_bytes(p->io_dtype);
    const size_t nq = (size_t)p->B * p->H * p->L * p->d * e, nk = (size_t)p->B * p->H_kv * p->L * p->d * e;
    const size_t nc = (size_t)p->B * p->H_kv * ((size_t)p->window + p->sinks) * p->d * e;
    if (p->L > 0 && (!q || !k || !v || !o)) return BLA_ERR_INVALID_ARG;
    if (!cache_k_in != !cache_v_in || !cache_k_out != !cache_v_out) return BLA_ERR_INVALID_ARG;
    const void* ptr[] = {q, k, v, o, cache_k_in, cache_v_in, cache_k_out, cache_v_out};
    for (const void* x : ptr)
        if (x && !is_aligned16(x)) return BLA_ERR_INVALID_ARG;
    if (!aligned(lengths, 4) || !aligned(pos, 8) || !aligned(lse, 4)) return BLA_ERR_INVALID_ARG;
    const size_t nl = (size_t)p->B * p->H * p->L * 4, nb = (size_t)p->B;
    const Span in[] = {{q, nq}, {k, nk}, {v, nk}, {cache_k_in, nc}, {cache_v_in, nc}, {lengths, 4 * nb}, {pos, 8 * nb}};
    const Span out[] = {{o, nq}, {lse, nl}, {cache_k_out, nc}, {cache_v_out, nc}};
    if (clash(in, out) || clash(extra, out)) return BLA_ERR_INVALID_ARG;
    if (f.total > 0 && (!workspace || workspace_bytes < f.total || !is_aligned16(workspace))) return BLA_ERR_WORKSPACE;
    if (f.total > 0 && !tables_overwritten(workspace, f.total)) return BLA_ERR_HIP;

    a.q = q, a.k = k, a.v = v, a.ck = cache_k_in, a.cv = cache_v_in, a.o = o, a.lse = lse;
    a.ck_out = cache_k_out, a.cv_out = cache_v_out, a.lengths = lengths, a.pos = pos, a.t0 = p->t0;
    a.B = p->B, a.H = p->H, a.Hkv = p->H_kv, a.L = p->L, a.W = p->window, a.S = p->sinks, a.scale = scale_of(p);
    a.nqb = f.nqb, a.nsplit = f.nsplit, a.units = f.units, a.per = (f.units + 7) / 8;
    a.part_o = (float*)workspace;
    a.part_ml = f.nsplit > 1 ? a.part_o + (size_t)f.nsplit * p->B * p->H * p->L * p->d : nullptr;
    return BLA_OK;
}

// The step's.  total: the call's workspace, in which part_o and part_ml stand first where it has parts of the rings alone.
template <int N>
bla_status step_args(WindowStepArgs& a, const bla_window_params* p, const StepPlan& sp, const void* q, const void* k, const void* v,
                     const int64_t* pos, void* cache_k, void* cache_v, void* o, const Span (&extra)[N], void* workspace, size_t total,
                     size_t workspace_bytes)
{
    const int e = elem_bytes(p->io_dtype);
    const size_t nq = (size_t)p->B * p->H * p->d * e, nk = (size_t)p->B * p->H_kv * p->d * e;
    const size_t nc = (size_t)p->B * p->H_kv * ((size_t)p->window + p->sinks) * p->d * e;
    const void* ptr[] = {q, k, v, cache_k, cache_v, o};
    for (const void* x : ptr)
        if (!x || !is_aligned16(x)) return BLA_ERR_INVALID_ARG;
    if (!aligned(pos, 8)) return BLA_ERR_INVALID_ARG;
    const Span in[] = {{q, nq}, {k, nk}, {v, nk}, {pos, 8 * (size_t)p->B}};
    const Span out[] = {{o, nq}, {cache_k, nc}, {cache_v, nc}};
    if (clash(in, out) || clash(extra, out)) return BLA_ERR_INVALID_ARG;
    if (total > 0 && (!workspace || workspace_bytes < total || !is_aligned16(workspace))) return BLA_ERR_WORKSPACE;
    if (total > 0 && !tables_overwritten(workspace, total)) return BLA_ERR_HIP;

    a.q = q, a.k = k, a.v = v, a.ck = cache_k, a.cv = cache_v, a.o = o, a.pos = pos, a.t0 = p->t0;
    a.B = p->B, a.H = p->H, a.Hkv = p->H_kv, a.W = p->window, a.S = p->sinks, a.scale = scale_of(p);
    a.ngrp = sp.ngrp, a.nsplit = sp.nsplit;
    a.part_o = (float*)workspace;
    a.part_ml = sp.nsplit > 1 ? a.part_o + (size_t)sp.nsplit * p->B * p->H * p->d : nullptr;
    return BLA_OK;
}

// The backward call's.
template <int I, int O>
bla_status backward_args(WindowBwdArgs& a, const bla_window_params* p, const BackwardPlan& b, const void* q, const void* k, const void* v,
                         const void* o, const float* lse, const void* dO, const int32_t* lengths, void* dq, void* dk, void* dv,
                         const Span (&more_in)[I], const Span (&more_out)[O], void* workspace, size_t total, size_t workspace_bytes)
{
    const int e = elem_bytes(p->io_dtype);
    const size_t nq = (size_t)p->B * p->H * p->L * p->d * e, nk = (size_t)p->B * p->H_kv * p->L * p->d * e;
    const void* ptr[] = {q, k, v, o, dO, dq, dk, dv};
    for (const void* x : ptr)
        if (!x || !is_aligned16(x)) return BLA_ERR_INVALID_ARG;
    if (!lse || !aligned(lse, 4) || !aligned(lengths, 4)) return BLA_ERR_INVALID_ARG;
    const Span in[] = {{q, nq}, {k, nk}, {v, nk}, {o, nq}, {dO, nq}, {lse, (size_t)p->B * p->H * p->L * 4}, {lengths, 4 * (size_t)p->B}};
    const Span out[] = {{dq, nq}, {dk, nk}, {dv, nk}};
    if (clash(in, out) || clash(more_in, out) || clash(in, more_out) || clash(more_in, more_out) || clash(more_out, out)) return BLA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < total || !is_aligned16(workspace)) return BLA_ERR_WORKSPACE;
    if (!tables_overwritten(workspace, total)) return BLA_ERR_HIP;

    a.q = q, a.k = k, a.v = v, a.o = o, a.dO = dO, a.lse = lse, a.dq = dq, a.dk = dk, a.dv = dv, a.lengths = lengths;
    a.B = p->B, a.H = p->H, a.Hkv = p->H_kv, a.L = p->L, a.W = p->window, a.S = p->sinks, a.scale = scale_of(p);
    a.delta = (float*)workspace, a.near = (float*)((char*)workspace + b.off_near);
    a.part = (float*)((char*)workspace + b.off_part);
    a.nqb = b.nqb, a.nkb = b.nkb, a.ns = b.ns, a.ssplit = b.ssplit;
    a.q_units = b.q_units, a.q_per = (b.q_units + 7) / 8, a.k_units = b.k_units, a.k_per = (b.k_units + 7) / 8;
    a.s_units = (unsigned)b.s_units;
    return BLA_OK;
}

// Joins the parts of L tokens of every row, where there are several.
inline bla_status join_parts(const bla_window_params* p, int L, int nsplit, float* part_o, float* part_ml, void* o, float* lse, hipStream_t s)
{
    if (L == 0 || nsplit <= 1) return BLA_OK;
    const JoinArgs j = {part_o, part_ml, o, lse, (long long)p->B * p->H * L, nsplit};
    return launch_window_join(p->io_dtype == BLA_BF16, p->d, j, s) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

constexpr Span kNone[] = {{nullptr, 0}};

}  // namespace bla
