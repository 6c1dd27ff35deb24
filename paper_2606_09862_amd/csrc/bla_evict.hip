// Attention over a cache of bounded size: entry points.
#include "bla_evict.h"
#include "bla_window_plan.h"

namespace bla {
hipError_t launch_prefix_forward(int bf16_io, int D, int waves, const PrefixArgs& a, hipStream_t s);
}  // namespace bla

using namespace bla;

namespace {

constexpr int kMaxSlots = 1 << 24;

// The call as attention over a window without end.
bla_window_params window_of(const bla_evict_params* p, int window)
{
    return {p->B, p->H, p->H_kv, p->L, p->d, window, 0, p->io_dtype, p->t0, p->scale};
}

bla_status check_evict(const bla_evict_params* p, bool step)
{
    if (!p) return BLA_ERR_INVALID_ARG;
    if (p->slots < 1 || p->recent < 0 || p->recent >= p->slots) return BLA_ERR_INVALID_ARG;
    const bla_window_params w = window_of(p, p->slots);
    const bla_status st = check(&w, step);
    if (st != BLA_OK) return st;
    if (p->slots > kMaxSlots) return BLA_ERR_UNSUPPORTED;
    const double entries = (double)p->slots + (step ? 0 : p->L);
    return launchable((double)p->B * p->H * entries / 256 + 1, 256) ? BLA_OK : BLA_ERR_UNSUPPORTED;
}

// Forward: attention with the cache in the place of a prefix, then the sums: a workgroup to 128 keys of a query head.
struct EvictPlan : ForwardPlan {
    int ncb, nkb;
    long long sum_units;
    size_t off_lse, off_part;
};
EvictPlan evict_plan(const bla_evict_params* p, bool cached)
{
    EvictPlan e;
    const bla_window_params w = window_of(p, p->L > 0 ? p->L : 1);
    static_cast<ForwardPlan&>(e) = forward_plan(&w, false, cached ? p->slots : 0);
    e.ncb = cached ? (p->slots + kEvictKeys - 1) / kEvictKeys : 0;
    e.nkb = e.ncb + (p->L + kEvictKeys - 1) / kEvictKeys;
    const size_t bh = (size_t)p->B * p->H;
    e.sum_units = (long long)bh * e.nkb;
    e.off_lse = e.total;
    e.off_part = e.off_lse + seq_align(bh * p->L * 4);
    e.total = e.off_part + seq_align(bh * ((size_t)p->slots + p->L) * 4);
    return e;
}
bool fits(const bla_evict_params* p, const EvictPlan& e)
{
    const bla_window_params w = window_of(p, p->L > 0 ? p->L : 1);
    return fits(&w, e, false) && launchable(8.0 * ((e.sum_units + 7) / 8), 256);
}

// Step: window attention's split; the sums are formed by the same workgroups where each has all slots and heads of its key head.
struct EvictStepPlan : ShortStepPlan {
    bool fused, in_lds;
    int pitch;
    size_t off_z, off_mine;
};
EvictStepPlan evict_step_plan(const bla_evict_params* p)
{
    EvictStepPlan s;
    const bla_window_params w = window_of(p, p->slots);
    static_cast<ShortStepPlan&>(s) = short_step_plan(&w);
    s.fused = s.nsplit == 1 && s.ngrp == 1;
    s.pitch = (p->slots + 31) & ~31;
    const size_t rows = (size_t)p->B * p->H;
    s.off_z = s.fused ? 0 : seq_align(s.nsplit * rows * (p->d + 2) * 4);
    s.in_lds = s.fused && p->H_kv > 0 && (long long)(p->H / p->H_kv) * s.pitch * 4 <= score_lds(s.waves, p->io_dtype == BLA_BF16, p->d);
    s.off_mine = s.off_z + (s.in_lds ? 0 : seq_align(rows * s.pitch * 4));
    s.total = s.off_mine + seq_align((size_t)p->B * p->H_kv * 4);
    return s;
}
bool fits(const bla_evict_params* p, const EvictStepPlan& s)
{
    return launchable((double)p->B * p->H_kv * s.ngrp * s.nsplit, 64 * s.waves) &&
           launchable((double)p->B * p->H_kv * ((p->slots + 255) / 256) + (double)p->B * p->H / 4 + 1, 256);
}

// Select: a workgroup to a key head's slice of the slots, as many slices as fill the device (each finds what stays by itself).
int select_slices(const bla_evict_params* p)
{
    const long long bh = (long long)p->B * p->H_kv, least = (p->slots + kSliceSlots - 1) / kSliceSlots;
    long long n = bh > 0 ? 256 / bh : 1;
    const long long most = (p->slots + 63) / 64;
    if (n > most) n = most;
    return (int)(n < least ? least : n < 1 ? 1 : n);
}
bool select_fits(const bla_evict_params* p) { return launchable((double)p->B * p->H_kv * select_slices(p), 1024); }

bool enough(const void* workspace, size_t bytes, size_t total) { return total == 0 || (workspace && bytes >= total && is_aligned16(workspace)); }

}  // namespace

extern "C" {

bla_status bla_evict_supported(const bla_evict_params* p)
{
    const bla_status st = check_evict(p, false);
    return st == BLA_OK && !fits(p, evict_plan(p, true)) ? BLA_ERR_UNSUPPORTED : st;
}

size_t bla_evict_workspace_size(const bla_evict_params* p) { return bla_evict_supported(p) == BLA_OK ? evict_plan(p, true).total : 0; }

bla_status bla_evict_forward(const bla_evict_params* p, const void* q, const void* k, const void* v, const int32_t* lengths,
                             const int64_t* pos, const void* cache_k, const void* cache_v, const float* score_in, void* o, float* lse,
                             float* score_out, void* workspace, size_t workspace_bytes, void* stream)
{
    bla_status st = check_evict(p, false);
    if (st != BLA_OK) return st;
    const bla_window_params w = window_of(p, p->L > 0 ? p->L : 1);
    if (p->B == 0 || p->H == 0) return empty(&w, true);
    const bool cached = cache_k != nullptr;
    const EvictPlan e = evict_plan(p, cached);
    if (!fits(p, e)) return BLA_ERR_UNSUPPORTED;
    if (!cache_k != !cache_v || !cache_k != !score_in) return BLA_ERR_INVALID_ARG;
    if (!score_out || !aligned(score_out, 4) || !aligned(score_in, 4)) return BLA_ERR_INVALID_ARG;
    if (cached && (!is_aligned16(cache_k) || !is_aligned16(cache_v))) return BLA_ERR_INVALID_ARG;
    const size_t nc = (size_t)p->B * p->H_kv * p->slots * p->d * elem_bytes(p->io_dtype), nb = (size_t)p->B;
    const size_t entries = (size_t)p->B * p->H_kv * ((size_t)p->slots + p->L), nq = (size_t)p->B * p->H * p->L * p->d * elem_bytes(p->io_dtype);
    const size_t nk = (size_t)p->B * p->H_kv * p->L * p->d * elem_bytes(p->io_dtype);
    const Span extra[] = {{cache_k, nc}, {cache_v, nc}, {score_in, (size_t)p->B * p->H_kv * p->slots * 4}, {score_out, entries * 4}};
    const Span in[] = {{q, nq}, {k, nk}, {v, nk}, {cache_k, nc}, {cache_v, nc}, {score_in, (size_t)p->B * p->H_kv * p->slots * 4},
                       {lengths, 4 * nb}, {pos, 8 * nb}};
    const Span out[] = {{score_out, entries * 4}};
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    if (!enough(workspace, workspace_bytes, e.total)) return BLA_ERR_WORKSPACE;
    PrefixArgs a = {};
    if ((st = forward_args(a, &w, e, q, k, v, lengths, pos, nullptr, nullptr, o, lse, nullptr, nullptr, extra, workspace, workspace_bytes)) != BLA_OK)
        return st;
    if (!a.lse) a.lse = (float*)((char*)workspace + e.off_lse);
    a.pk = cache_k, a.pv = cache_v, a.P = cached ? p->slots : 0, a.G = p->B, a.by_pos = true;
    hipStream_t s = (hipStream_t)stream;
    const int bf16 = p->io_dtype == BLA_BF16;
    if (p->L > 0) {
        if (launch_prefix_forward(bf16, p->d, e.waves, a, s) != hipSuccess) return BLA_ERR_HIP;
        if ((st = join_parts(&w, p->L, e.nsplit, a.part_o, a.part_ml, o, a.lse, s)) != BLA_OK) return st;
    }
    EvictSumArgs m = {};
    m.q = q, m.k = k, m.ck = cache_k, m.lse = a.lse, m.lengths = lengths, m.pos = pos, m.t0 = p->t0;
    m.B = p->B, m.H = p->H, m.Hkv = p->H_kv, m.L = p->L, m.slots = p->slots, m.scale = scale_of(&w);
    m.ncb = e.ncb, m.nkb = e.nkb, m.units = e.sum_units, m.per = (e.sum_units + 7) / 8;
    m.part = (float*)((char*)workspace + e.off_part), m.score_in = score_in, m.score_out = score_out;
    return launch_evict_sum(bf16, p->d, m, s) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

bla_status bla_evict_select(const bla_evict_params* p, const void* k, const void* v, const float* score, const int32_t* lengths,
                            const int64_t* pos, const void* cache_k_in, const void* cache_v_in, const int64_t* at_in, void* cache_k_out,
                            void* cache_v_out, float* score_out, int64_t* at_out, void* stream)
{
    if (!p) return BLA_ERR_INVALID_ARG;
    bla_evict_params own = *p;  // query heads and the scale are no part of this call, whatever they hold
    own.H = 0, own.scale = 0.f;
    const bla_status st = check_evict(&own, false);
    if (st != BLA_OK) return st;
    if (!select_fits(p)) return BLA_ERR_UNSUPPORTED;
    if (p->B == 0 || p->H_kv == 0) return BLA_OK;
    if (p->L > 0 && (!k || !v)) return BLA_ERR_INVALID_ARG;
    if (!score || !cache_k_out || !cache_v_out || !score_out || !at_out) return BLA_ERR_INVALID_ARG;
    if (!cache_k_in != !cache_v_in || !cache_k_in != !at_in) return BLA_ERR_INVALID_ARG;
    const void* ptr[] = {k, v, cache_k_in, cache_v_in, cache_k_out, cache_v_out};
    for (const void* x : ptr)
        if (x && !is_aligned16(x)) return BLA_ERR_INVALID_ARG;
    if (!aligned(score, 4) || !aligned(score_out, 4) || !aligned(at_in, 8) || !aligned(at_out, 8) || !aligned(lengths, 4) || !aligned(pos, 8))
        return BLA_ERR_INVALID_ARG;
    const size_t bh = (size_t)p->B * p->H_kv, row = (size_t)p->d * elem_bytes(p->io_dtype), n = bh * p->slots;
    const Span in[] = {{k, bh * p->L * row}, {v, bh * p->L * row}, {score, bh * ((size_t)p->slots + p->L) * 4}, {lengths, 4 * (size_t)p->B},
                       {pos, 8 * (size_t)p->B}, {cache_k_in, n * row}, {cache_v_in, n * row}, {at_in, n * 8}};
    const Span out[] = {{cache_k_out, n * row}, {cache_v_out, n * row}, {score_out, n * 4}, {at_out, n * 8}};
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    EvictSelectArgs a = {};
    a.k = k, a.v = v, a.ck = cache_k_in, a.cv = cache_v_in, a.score = score, a.at_in = at_in, a.lengths = lengths, a.pos = pos, a.t0 = p->t0;
    a.B = p->B, a.Hkv = p->H_kv, a.L = p->L, a.slots = p->slots, a.recent = p->recent, a.slices = select_slices(p);
    a.pieces = (int)(row / 16);
    a.ck_out = cache_k_out, a.cv_out = cache_v_out, a.score_out = score_out, a.at_out = at_out;
    return launch_evict_select(a, (hipStream_t)stream) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

size_t bla_evict_step_workspace_size(const bla_evict_params* p)
{
    if (check_evict(p, true) != BLA_OK) return 0;
    const EvictStepPlan s = evict_step_plan(p);
    return fits(p, s) ? s.total : 0;
}

bla_status bla_evict_step(const bla_evict_params* p, const void* q, const void* k, const void* v, const int64_t* pos, void* cache_k,
                          void* cache_v, const float* score_in, const int64_t* at_in, void* o, float* score_out, int64_t* at_out,
                          void* workspace, size_t workspace_bytes, void* stream)
{
    bla_status st = check_evict(p, true);
    if (st != BLA_OK) return st;
    const bla_window_params w = window_of(p, p->slots);
    if (p->B == 0 || p->H == 0) return empty(&w, true);
    const EvictStepPlan sp = evict_step_plan(p);
    if (!fits(p, sp)) return BLA_ERR_UNSUPPORTED;
    if (!score_in || !at_in || !score_out || !at_out) return BLA_ERR_INVALID_ARG;
    if (!aligned(score_in, 4) || !aligned(score_out, 4) || !aligned(at_in, 8) || !aligned(at_out, 8)) return BLA_ERR_INVALID_ARG;
    const size_t n = (size_t)p->B * p->H_kv * p->slots, nq = (size_t)p->B * p->H * p->d * elem_bytes(p->io_dtype);
    const size_t nk = (size_t)p->B * p->H_kv * p->d * elem_bytes(p->io_dtype);
    // each of score_out and at_out may be its input, and nothing else
    const Span in[] = {{q, nq}, {k, nk}, {v, nk}, {pos, 8 * (size_t)p->B}, {score_out == score_in ? nullptr : (const void*)score_in, n * 4},
                       {at_out == at_in ? nullptr : (const void*)at_in, n * 8}};
    const Span out[] = {{score_out, n * 4}, {at_out, n * 8}};
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    const Span extra[] = {{score_in, n * 4}, {at_in, n * 8}, {score_out, n * 4}, {at_out, n * 8}};
    EvictStepArgs a = {};
    if ((st = step_args(a, &w, sp, q, k, v, pos, cache_k, cache_v, o, extra, workspace, sp.total, workspace_bytes)) != BLA_OK) return st;
    const size_t rows = (size_t)p->B * p->H;
    a.part_ml = a.part_o + (size_t)sp.nsplit * rows * p->d;
    a.score_in = score_in, a.score_out = score_out, a.at_in = at_in, a.at_out = at_out, a.recent = p->recent;
    a.z = (float*)((char*)workspace + sp.off_z), a.pitch = sp.pitch, a.mine = (int*)((char*)workspace + sp.off_mine), a.fused = sp.fused, a.in_lds = sp.in_lds;
    hipStream_t s = (hipStream_t)stream;
    const int bf16 = p->io_dtype == BLA_BF16;
    return launch_evict_step(bf16, p->d, a, sp.waves, s) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

}  // extern "C"
