// Window attention: argument checks, work split and entry points.
#include "bla_window.h"

using namespace bla;

namespace {

// Workgroups that fill the device twice over (256 compute units).  With fewer, a block's keys are split into parts.
constexpr long long kFill = 512;
constexpr int kMaxParts = 64;

bla_status check(const bla_window_params* p, bool step)
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

float scale_of(const bla_window_params* p) { return p->scale == 0.f ? 1.f / sqrtf((float)p->d) : p->scale; }

// A call without rows or query heads: done, unless key heads have outputs that nothing would write.
bla_status empty(const bla_window_params* p, bool outputs)
{
    return outputs && p->B > 0 && p->H_kv > 0 ? BLA_ERR_UNSUPPORTED : BLA_OK;
}

// Forward: 128 queries to a workgroup (fewer reads of keys), 64 where that fills the device better;
// the keys of a block in parts of at least two tiles where the blocks alone do not fill it.
struct ForwardPlan {
    int waves, nqb, nsplit;
    long long units;
    size_t total;
};
ForwardPlan forward_plan(const bla_window_params* p, bool cached)
{
    ForwardPlan f;
    const long long bh = (long long)p->B * p->H;
    f.waves = bh * ((p->L + 127) / 128) >= kFill ? 8 : 4;
    f.nqb = (p->L + 16 * f.waves - 1) / (16 * f.waves);
    const long long blocks = bh * f.nqb;
    long long keys = (long long)p->window - 1 + 16 * f.waves + p->sinks;
    if (!cached && keys > p->L) keys = p->L;
    const long long tiles = (keys + kWinKeys - 1) / kWinKeys;
    long long n = 1;
    if (blocks > 0 && blocks < kFill) n = (kFill + blocks - 1) / blocks;
    if (n > tiles / 2) n = tiles / 2;
    f.nsplit = (int)(n < 1 ? 1 : n > kMaxParts ? kMaxParts : n);
    f.units = blocks * f.nsplit;
    f.total = f.nsplit > 1 ? seq_align((size_t)f.nsplit * bh * p->L * (p->d + 2) * 4) : 0;
    return f;
}

// whether the forward kernel's launch is one, with the workgroups that write the rings after the call
bool fits(const bla_window_params* p, const ForwardPlan& f, bool rings)
{
    const double pieces = (double)p->B * p->H_kv * ((double)p->window + p->sinks) * (p->d * elem_bytes(p->io_dtype) / 16);
    return launchable(8.0 * ((f.units + 7) / 8) + (rings ? ceil(pieces / (64 * f.waves)) : 0.0), 64 * f.waves);
}

// Step: a key head's ring in parts of at least 128 slots where the key heads of all rows alone do not fill the device.
struct StepPlan {
    int ngrp, nsplit;
    size_t total;
};
StepPlan step_plan(const bla_window_params* p)
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
bool fits(const bla_window_params* p, const StepPlan& s) { return launchable((double)p->B * p->H_kv * s.ngrp * s.nsplit, 256); }

// Backward: the sinks' queries beyond their windows in as many parts as fill the device with waves, a block of 32 queries or more to each.
struct BackwardPlan {
    int nqb, nkb, ns, ssplit;
    long long q_units, k_units, s_units;
    size_t off_near, off_part, total;
};
BackwardPlan backward_plan(const bla_window_params* p)
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

bool fits(const bla_window_params* p, const BackwardPlan& b)
{
    return launchable(8.0 * ((b.q_units + 7) / 8), 256) && launchable(8.0 * ((b.k_units + 7) / 8) + b.s_units, 256) &&
           launchable((double)p->B * p->H_kv * b.ns * (2 * p->d / 4) / 256 + 1, 256);
}

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

}  // namespace

extern "C" {

size_t bla_window_workspace_size(const bla_window_params* p)
{
    return bla_window_supported(p) == BLA_OK ? forward_plan(p, true).total : 0;
}

bla_status bla_window_supported(const bla_window_params* p)
{
    const bla_status st = check(p, false);
    return st == BLA_OK && !fits(p, forward_plan(p, true), false) ? BLA_ERR_UNSUPPORTED : st;
}

bla_status bla_window_forward(const bla_window_params* p, const void* q, const void* k, const void* v, const int32_t* lengths,
                              const int64_t* pos, const void* cache_k_in, const void* cache_v_in, void* o, float* lse,
                              void* cache_k_out, void* cache_v_out, void* workspace, size_t workspace_bytes, void* stream)
{
    const bla_status st = check(p, false);
    if (st != BLA_OK) return st;
    if (p->B == 0 || p->H == 0) return empty(p, cache_k_out || cache_v_out);
    const ForwardPlan f = forward_plan(p, cache_k_in != nullptr);
    if (!fits(p, f, cache_k_out != nullptr)) return BLA_ERR_UNSUPPORTED;
    const int e = elem_bytes(p->io_dtype), bf16 = p->io_dtype == BLA_BF16;
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
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    if (f.total > 0 && (!workspace || workspace_bytes < f.total || !is_aligned16(workspace))) return BLA_ERR_WORKSPACE;
    if (f.total > 0 && !tables_overwritten(workspace, f.total)) return BLA_ERR_HIP;

    WindowArgs a = {};
    a.q = q, a.k = k, a.v = v, a.ck = cache_k_in, a.cv = cache_v_in, a.o = o, a.lse = lse;
    a.ck_out = cache_k_out, a.cv_out = cache_v_out, a.lengths = lengths, a.pos = pos, a.t0 = p->t0;
    a.B = p->B, a.H = p->H, a.Hkv = p->H_kv, a.L = p->L, a.W = p->window, a.S = p->sinks, a.scale = scale_of(p);
    a.nqb = f.nqb, a.nsplit = f.nsplit, a.units = f.units, a.per = (f.units + 7) / 8;
    const size_t rows = (size_t)p->B * p->H * p->L;
    a.part_o = (float*)workspace;
    a.part_ml = f.nsplit > 1 ? a.part_o + (size_t)f.nsplit * rows * p->d : nullptr;
    hipStream_t s = (hipStream_t)stream;
    if ((p->L > 0 || cache_k_out) && launch_window_forward(bf16, p->d, f.waves, a, s) != hipSuccess) return BLA_ERR_HIP;
    if (p->L > 0 && f.nsplit > 1) {
        const JoinArgs j = {a.part_o, a.part_ml, o, lse, (long long)rows, f.nsplit};
        if (launch_window_join(bf16, p->d, j, s) != hipSuccess) return BLA_ERR_HIP;
    }
    return BLA_OK;
}

size_t bla_window_step_workspace_size(const bla_window_params* p)
{
    if (check(p, true) != BLA_OK) return 0;
    const StepPlan s = step_plan(p);
    return fits(p, s) ? s.total : 0;
}

bla_status bla_window_step(const bla_window_params* p, const void* q, const void* k, const void* v, const int64_t* pos,
                           void* cache_k, void* cache_v, void* o, void* workspace, size_t workspace_bytes, void* stream)
{
    const bla_status st = check(p, true);
    if (st != BLA_OK) return st;
    if (p->B == 0 || p->H == 0) return empty(p, true);
    const StepPlan sp = step_plan(p);
    if (!fits(p, sp)) return BLA_ERR_UNSUPPORTED;
    const int e = elem_bytes(p->io_dtype), bf16 = p->io_dtype == BLA_BF16;
    const size_t nq = (size_t)p->B * p->H * p->d * e, nk = (size_t)p->B * p->H_kv * p->d * e;
    const size_t nc = (size_t)p->B * p->H_kv * ((size_t)p->window + p->sinks) * p->d * e;
    const void* ptr[] = {q, k, v, cache_k, cache_v, o};
    for (const void* x : ptr)
        if (!x || !is_aligned16(x)) return BLA_ERR_INVALID_ARG;
    if (!aligned(pos, 8)) return BLA_ERR_INVALID_ARG;
    const Span in[] = {{q, nq}, {k, nk}, {v, nk}, {pos, 8 * (size_t)p->B}};
    const Span out[] = {{o, nq}, {cache_k, nc}, {cache_v, nc}};
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    if (sp.total > 0 && (!workspace || workspace_bytes < sp.total || !is_aligned16(workspace))) return BLA_ERR_WORKSPACE;
    if (sp.total > 0 && !tables_overwritten(workspace, sp.total)) return BLA_ERR_HIP;

    WindowStepArgs a = {};
    a.q = q, a.k = k, a.v = v, a.ck = cache_k, a.cv = cache_v, a.o = o, a.pos = pos, a.t0 = p->t0;
    a.B = p->B, a.H = p->H, a.Hkv = p->H_kv, a.W = p->window, a.S = p->sinks, a.scale = scale_of(p);
    a.ngrp = sp.ngrp, a.nsplit = sp.nsplit;
    const size_t rows = (size_t)p->B * p->H;
    a.part_o = (float*)workspace;
    a.part_ml = sp.nsplit > 1 ? a.part_o + (size_t)sp.nsplit * rows * p->d : nullptr;
    hipStream_t s = (hipStream_t)stream;
    if (launch_window_step(bf16, p->d, a, s) != hipSuccess) return BLA_ERR_HIP;
    if (sp.nsplit > 1) {
        const JoinArgs j = {a.part_o, a.part_ml, o, nullptr, (long long)rows, sp.nsplit};
        if (launch_window_join(bf16, p->d, j, s) != hipSuccess) return BLA_ERR_HIP;
    }
    return BLA_OK;
}

size_t bla_window_backward_workspace_size(const bla_window_params* p)
{
    if (check(p, false) != BLA_OK) return 0;
    const BackwardPlan b = backward_plan(p);
    return fits(p, b) ? b.total : 0;
}

bla_status bla_window_backward(const bla_window_params* p, const void* q, const void* k, const void* v, const void* o,
                               const float* lse, const void* dO, const int32_t* lengths, void* dq, void* dk, void* dv,
                               void* workspace, size_t workspace_bytes, void* stream)
{
    const bla_status st = check(p, false);
    if (st != BLA_OK) return st;
    if (p->t0 != 0) return BLA_ERR_UNSUPPORTED;
    if (p->B == 0 || p->H == 0 || p->L == 0) return empty(p, p->L > 0);
    const BackwardPlan b = backward_plan(p);
    if (!fits(p, b)) return BLA_ERR_UNSUPPORTED;
    const int e = elem_bytes(p->io_dtype), bf16 = p->io_dtype == BLA_BF16;
    const size_t nq = (size_t)p->B * p->H * p->L * p->d * e, nk = (size_t)p->B * p->H_kv * p->L * p->d * e;
    const void* ptr[] = {q, k, v, o, dO, dq, dk, dv};
    for (const void* x : ptr)
        if (!x || !is_aligned16(x)) return BLA_ERR_INVALID_ARG;
    if (!lse || !aligned(lse, 4) || !aligned(lengths, 4)) return BLA_ERR_INVALID_ARG;
    const Span in[] = {{q, nq}, {k, nk}, {v, nk}, {o, nq}, {dO, nq}, {lse, (size_t)p->B * p->H * p->L * 4}, {lengths, 4 * (size_t)p->B}};
    const Span out[] = {{dq, nq}, {dk, nk}, {dv, nk}};
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < b.total || !is_aligned16(workspace)) return BLA_ERR_WORKSPACE;
    if (!tables_overwritten(workspace, b.total)) return BLA_ERR_HIP;

    WindowBwdArgs a = {};
    a.q = q, a.k = k, a.v = v, a.o = o, a.dO = dO, a.lse = lse, a.dq = dq, a.dk = dk, a.dv = dv, a.lengths = lengths;
    a.B = p->B, a.H = p->H, a.Hkv = p->H_kv, a.L = p->L, a.W = p->window, a.S = p->sinks, a.scale = scale_of(p);
    a.delta = (float*)workspace, a.near = (float*)((char*)workspace + b.off_near);
    a.part = (float*)((char*)workspace + b.off_part);
    a.nqb = b.nqb, a.nkb = b.nkb, a.ns = b.ns, a.ssplit = b.ssplit;
    a.q_units = b.q_units, a.q_per = (b.q_units + 7) / 8, a.k_units = b.k_units, a.k_per = (b.k_units + 7) / 8;
    a.s_units = (unsigned)b.s_units;
    return launch_window_backward(bf16, p->d, a, (hipStream_t)stream) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

}  // extern "C"
