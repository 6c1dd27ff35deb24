// Window attention behind a prefix that rows share: entry points.
#include "bla_window_plan.h"
#include "bla_window_step.h"

namespace bla {
hipError_t launch_prefix_forward(int bf16_io, int D, int waves, const PrefixArgs& a, hipStream_t s);
hipError_t launch_prefix_step(int bf16_io, int D, const PrefixStepArgs& a, PrefixForm form, hipStream_t s);
}  // namespace bla

using namespace bla;

namespace {

bla_status check_prefix(const bla_prefix_params* p, bool step)
{
    if (!p) return BLA_ERR_INVALID_ARG;
    const bla_window_params* w = &p->w;
    const bla_status st = check(w, step);
    if (st != BLA_OK) return st;
    if (p->P < 0 || p->G < 0 || (w->B > 0 && (p->G < 1 || w->B % p->G != 0))) return BLA_ERR_INVALID_ARG;
    if (p->P > (1 << 30) || (double)p->G * w->H_kv * p->P * w->d > 256.0 * (1 << 30)) return BLA_ERR_UNSUPPORTED;
    return BLA_OK;
}

// The step's: the prefix in parts that fill the device with the blocks of its queries, of at least a tile for each group of waves, beside the rings' parts.  Few
// queries go in blocks of 16, whose four waves take 32 tokens each: against tiles, bf16 at d = 64 with 4 key heads, 16 queries behind each of 16 prefixes of 8192 tokens
// 30.2 against 41.6 us, 32 queries 35.4 against 45.6, 64 queries 60.8 against 54.4; 32 queries behind one of 2048 7.4 against 9.0.  With a prefix and rings that are
// short together they need no parts at all: 16 queries behind 512 tokens, rings of 128, 6.1 us in a graph against 6.9 with parts, 10.0 against 13.5 called; behind
// 1024, rings of 512, 10.1 against 7.0 and 10.8 against 14.4.
constexpr int kFewQueries = 32, kMaxPrefixParts = 192;
struct PrefixStepPlan : StepPlan {
    bool few, both;  // both: no parts
    int npart, nqb, threads;
    long long units;
};
PrefixStepPlan prefix_step_plan(const bla_prefix_params* p)
{
    PrefixStepPlan s;
    static_cast<StepPlan&>(s) = step_plan(&p->w);
    const bla_window_params* w = &p->w;
    if (s.nsplit > kMaxParts / 4) s.nsplit = kMaxParts / 4;
    const long long rows = w->H_kv > 0 && p->G > 0 ? (long long)(w->B / p->G) * (w->H / w->H_kv) : 0;
    const PrefixShape shape = prefix_shape(w->io_dtype == BLA_BF16, w->d);
    s.few = rows <= kFewQueries;
    s.both = s.few && short_ring(w, (long long)p->P + w->window + w->sinks, false);
    if (s.both) {
        s.npart = s.nqb = 0, s.nsplit = 1, s.units = 0, s.threads = 512, s.total = 0;
        return s;
    }
    s.threads = s.few ? 256 : shape.threads;
    const int block = s.few ? 16 : shape.block, least = s.few ? 128 : kWinKeys * shape.groups;
    s.nqb = (int)((rows + block - 1) / block);
    const long long blocks = (long long)p->G * w->H_kv * s.nqb, fill = s.few ? 2 * kFill : shape.fill;
    long long n = blocks > 0 ? (fill + blocks - 1) / blocks : 1, most = (p->P + least - 1) / least;
    if (n > most) n = most;
    s.npart = (int)(n > kMaxPrefixParts ? kMaxPrefixParts : n);  // none where P = 0
    s.units = blocks * s.npart;
    s.total = seq_align((size_t)(s.npart + s.nsplit) * w->B * w->H * (w->d + 2) * 4);
    return s;
}
bool fits(const bla_prefix_params* p, const PrefixStepPlan& s)
{
    return launchable(8.0 * ((s.units + 7) / 8) + (double)p->w.B * p->w.H_kv * s.ngrp * s.nsplit, s.threads);
}

bla_status check_pointers(const bla_prefix_params* p, const void* prefix_k, const void* prefix_v, const int32_t* prefix_lengths)
{
    if (p->P > 0 && (!prefix_k || !prefix_v || !is_aligned16(prefix_k) || !is_aligned16(prefix_v))) return BLA_ERR_INVALID_ARG;
    return aligned(prefix_lengths, 4) ? BLA_OK : BLA_ERR_INVALID_ARG;
}

size_t prefix_bytes(const bla_prefix_params* p) { return (size_t)p->G * p->w.H_kv * p->P * p->w.d * elem_bytes(p->w.io_dtype); }

}  // namespace

extern "C" {

bla_status bla_prefix_supported(const bla_prefix_params* p)
{
    const bla_status st = check_prefix(p, false);
    return st == BLA_OK && !fits(&p->w, forward_plan(&p->w, true, p->P), false) ? BLA_ERR_UNSUPPORTED : st;
}

size_t bla_prefix_workspace_size(const bla_prefix_params* p)
{
    return bla_prefix_supported(p) == BLA_OK ? forward_plan(&p->w, true, p->P).total : 0;
}

bla_status bla_prefix_forward(const bla_prefix_params* p, const void* q, const void* k, const void* v, const void* prefix_k,
                              const void* prefix_v, const int32_t* prefix_lengths, const int32_t* lengths, const int64_t* pos,
                              const void* cache_k_in, const void* cache_v_in, void* o, float* lse, void* cache_k_out, void* cache_v_out,
                              void* workspace, size_t workspace_bytes, void* stream)
{
    bla_status st = check_prefix(p, false);
    if (st != BLA_OK) return st;
    const bla_window_params* w = &p->w;
    if (w->B == 0 || w->H == 0) return empty(w, cache_k_out || cache_v_out);
    const ForwardPlan f = forward_plan(w, cache_k_in != nullptr, p->P);
    if (!fits(w, f, cache_k_out != nullptr)) return BLA_ERR_UNSUPPORTED;
    if (w->L > 0 && (st = check_pointers(p, prefix_k, prefix_v, prefix_lengths)) != BLA_OK) return st;
    PrefixArgs a = {};
    const Span extra[] = {{prefix_k, prefix_bytes(p)}, {prefix_v, prefix_bytes(p)}, {prefix_lengths, 4 * (size_t)p->G}};
    if ((st = forward_args(a, w, f, q, k, v, lengths, pos, cache_k_in, cache_v_in, o, lse, cache_k_out, cache_v_out, extra, workspace,
                           workspace_bytes)) != BLA_OK)
        return st;
    a.pk = prefix_k, a.pv = prefix_v, a.plen = prefix_lengths, a.P = p->P, a.G = p->G, a.by_pos = false;
    hipStream_t s = (hipStream_t)stream;
    if ((w->L > 0 || cache_k_out) && launch_prefix_forward(w->io_dtype == BLA_BF16, w->d, f.waves, a, s) != hipSuccess) return BLA_ERR_HIP;
    return join_parts(w, w->L, f.nsplit, a.part_o, a.part_ml, o, lse, s);
}

size_t bla_prefix_step_workspace_size(const bla_prefix_params* p)
{
    if (check_prefix(p, true) != BLA_OK) return 0;
    const PrefixStepPlan s = prefix_step_plan(p);
    return fits(p, s) ? s.total : 0;
}

bla_status bla_prefix_step(const bla_prefix_params* p, const void* q, const void* k, const void* v, const void* prefix_k,
                           const void* prefix_v, const int32_t* prefix_lengths, const int64_t* pos, void* cache_k, void* cache_v, void* o,
                           void* workspace, size_t workspace_bytes, void* stream)
{
    bla_status st = check_prefix(p, true);
    if (st != BLA_OK) return st;
    const bla_window_params* w = &p->w;
    if (w->B == 0 || w->H == 0) return empty(w, true);
    const PrefixStepPlan sp = prefix_step_plan(p);
    if (!fits(p, sp)) return BLA_ERR_UNSUPPORTED;
    if ((st = check_pointers(p, prefix_k, prefix_v, prefix_lengths)) != BLA_OK) return st;
    PrefixStepArgs a = {};
    const Span extra[] = {{prefix_k, prefix_bytes(p)}, {prefix_v, prefix_bytes(p)}, {prefix_lengths, 4 * (size_t)p->G}};
    if ((st = step_args(a, w, sp, q, k, v, pos, cache_k, cache_v, o, extra, workspace, sp.total, workspace_bytes)) != BLA_OK) return st;
    a.pk = prefix_k, a.pv = prefix_v, a.plen = prefix_lengths, a.P = p->P, a.G = p->G;
    a.npart = sp.npart, a.nqb = sp.nqb, a.units = sp.units, a.per = (sp.units + 7) / 8;
    hipStream_t s = (hipStream_t)stream;
    if (sp.both) return launch_prefix_step(w->io_dtype == BLA_BF16, w->d, a, kFormBoth, s) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
    const size_t rows = (size_t)w->B * w->H;
    const int parts = sp.npart + sp.nsplit;
    a.pre_o = (float*)workspace, a.pre_ml = a.pre_o + (size_t)parts * rows * w->d;
    a.part_o = a.pre_o + (size_t)sp.npart * rows * w->d, a.part_ml = a.pre_ml + (size_t)sp.npart * rows * 2;
    if (launch_prefix_step(w->io_dtype == BLA_BF16, w->d, a, sp.few ? kFormFew : kFormTiles, s) != hipSuccess) return BLA_ERR_HIP;
    const JoinArgs j = {a.pre_o, a.pre_ml, o, nullptr, (long long)rows, parts};
    return launch_window_join(w->io_dtype == BLA_BF16, w->d, j, s) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

}  // extern "C"
