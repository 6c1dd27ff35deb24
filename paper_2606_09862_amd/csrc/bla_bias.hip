// Window attention with a learned bias: entry points.
#include "bla_window_bwd.h"
#include "bla_window_plan.h"
#include "bla_window_step.h"

namespace bla {
hipError_t launch_bias_forward(int bf16_io, int D, int waves, const BiasArgs& a, hipStream_t s);
hipError_t launch_bias_step(int bf16_io, int D, const BiasStepArgs& a, int waves, hipStream_t s);
hipError_t launch_bias_backward(int bf16_io, int D, const BiasBwdArgs& a, hipStream_t s);
}  // namespace bla

using namespace bla;

namespace {

constexpr int kMaxEdge = 1 << 29;

// The buckets of a call; edges is a host array.
bla_status check_buckets(int buckets, const int32_t* edges)
{
    if (buckets < 1) return BLA_ERR_INVALID_ARG;
    if (buckets > kMaxBuckets) return BLA_ERR_UNSUPPORTED;
    if (buckets > 1 && !edges) return BLA_ERR_INVALID_ARG;
    for (int i = 0; i + 1 < buckets; ++i) {
        if (edges[i] < (i ? edges[i - 1] : 0)) return BLA_ERR_INVALID_ARG;
        if (edges[i] > kMaxEdge) return BLA_ERR_UNSUPPORTED;
    }
    return BLA_OK;
}

void set_spec(BiasSpec& s, const float* bias, int buckets, const int32_t* edges)
{
    s.bias = bias, s.buckets = buckets;
    for (int i = 0; i + 1 < buckets; ++i) s.edges[i] = edges[i];
}

// The backward pass's plan is window attention's, with the sums of dS behind its workspace.
struct BiasBackwardPlan : BackwardPlan {
    size_t off_db;
};
BiasBackwardPlan bias_backward_plan(const bla_window_params* p, int buckets)
{
    BiasBackwardPlan b;
    static_cast<BackwardPlan&>(b) = backward_plan(p);
    b.off_db = b.total;
    b.total += seq_align((size_t)(b.k_units + b.s_units) * 4 * (p->H_kv > 0 ? p->H / p->H_kv : 0) * buckets * 4);
    return b;
}

}  // namespace

extern "C" {

bla_status bla_bias_forward(const bla_window_params* p, int32_t buckets, const int32_t* edges, const void* q, const void* k, const void* v,
                            const float* bias, const int32_t* lengths, const int64_t* pos, const void* cache_k_in, const void* cache_v_in,
                            void* o, float* lse, void* cache_k_out, void* cache_v_out, void* workspace, size_t workspace_bytes, void* stream)
{
    bla_status st = check(p, false);
    if (st == BLA_OK) st = check_buckets(buckets, edges);
    if (st != BLA_OK) return st;
    if (p->B == 0 || p->H == 0) return empty(p, cache_k_out || cache_v_out);
    const ForwardPlan f = forward_plan(p, cache_k_in != nullptr);
    if (!fits(p, f, cache_k_out != nullptr)) return BLA_ERR_UNSUPPORTED;
    if (p->L > 0 && (!bias || !aligned(bias, 4))) return BLA_ERR_INVALID_ARG;
    BiasArgs a = {};
    const Span extra[] = {{bias, (size_t)p->H * buckets * 4}};
    if ((st = forward_args(a, p, f, q, k, v, lengths, pos, cache_k_in, cache_v_in, o, lse, cache_k_out, cache_v_out, extra, workspace,
                           workspace_bytes)) != BLA_OK)
        return st;
    set_spec(a.spec, bias, buckets, edges);
    hipStream_t s = (hipStream_t)stream;
    const int bf16 = p->io_dtype == BLA_BF16;
    if ((p->L > 0 || cache_k_out) && launch_bias_forward(bf16, p->d, f.waves, a, s) != hipSuccess) return BLA_ERR_HIP;
    return join_parts(p, p->L, f.nsplit, a.part_o, a.part_ml, o, lse, s);
}

size_t bla_bias_step_workspace_size(const bla_window_params* p)
{
    if (check(p, true) != BLA_OK) return 0;
    const ShortStepPlan s = short_step_plan(p);
    return fits(p, s) ? s.total : 0;
}

bla_status bla_bias_step(const bla_window_params* p, int32_t buckets, const int32_t* edges, const void* q, const void* k, const void* v,
                         const float* bias, const int64_t* pos, void* cache_k, void* cache_v, void* o, void* workspace,
                         size_t workspace_bytes, void* stream)
{
    bla_status st = check(p, true);
    if (st == BLA_OK) st = check_buckets(buckets, edges);
    if (st != BLA_OK) return st;
    if (p->B == 0 || p->H == 0) return empty(p, true);
    const ShortStepPlan sp = short_step_plan(p);
    if (!fits(p, sp)) return BLA_ERR_UNSUPPORTED;
    if (!bias || !aligned(bias, 4)) return BLA_ERR_INVALID_ARG;
    BiasStepArgs a = {};
    const Span extra[] = {{bias, (size_t)p->H * buckets * 4}};
    if ((st = step_args(a, p, sp, q, k, v, pos, cache_k, cache_v, o, extra, workspace, sp.total, workspace_bytes)) != BLA_OK) return st;
    set_spec(a.spec, bias, buckets, edges);
    hipStream_t s = (hipStream_t)stream;
    if (launch_bias_step(p->io_dtype == BLA_BF16, p->d, a, sp.waves, s) != hipSuccess) return BLA_ERR_HIP;
    return join_parts(p, 1, sp.nsplit, a.part_o, a.part_ml, o, nullptr, s);
}

size_t bla_bias_backward_workspace_size(const bla_window_params* p, int32_t buckets)
{
    if (check(p, false) != BLA_OK || buckets < 1 || buckets > kMaxBuckets) return 0;
    const BiasBackwardPlan b = bias_backward_plan(p, buckets);
    return fits(p, b) ? b.total : 0;
}

bla_status bla_bias_backward(const bla_window_params* p, int32_t buckets, const int32_t* edges, const void* q, const void* k, const void* v,
                             const float* bias, const void* o, const float* lse, const void* dO, const int32_t* lengths, void* dq, void* dk,
                             void* dv, float* dbias, void* workspace, size_t workspace_bytes, void* stream)
{
    bla_status st = check(p, false);
    if (st == BLA_OK) st = check_buckets(buckets, edges);
    if (st != BLA_OK) return st;
    if (p->t0 != 0) return BLA_ERR_UNSUPPORTED;
    if (p->H == 0) return empty(p, p->L > 0);
    if (p->B == 0 || p->L == 0) return BLA_ERR_UNSUPPORTED;
    const BiasBackwardPlan b = bias_backward_plan(p, buckets);
    if (!fits(p, b)) return BLA_ERR_UNSUPPORTED;
    if (!bias || !dbias || !aligned(bias, 4) || !aligned(dbias, 4)) return BLA_ERR_INVALID_ARG;
    BiasBwdArgs a = {};
    const Span more_in[] = {{bias, (size_t)p->H * buckets * 4}}, more_out[] = {{dbias, (size_t)p->H * buckets * 4}};
    if ((st = backward_args(a, p, b, q, k, v, o, lse, dO, lengths, dq, dk, dv, more_in, more_out, workspace, b.total, workspace_bytes)) != BLA_OK)
        return st;
    set_spec(a.spec, bias, buckets, edges);
    a.db_part = (float*)((char*)workspace + b.off_db), a.dbias = dbias;
    return launch_bias_backward(p->io_dtype == BLA_BF16, p->d, a, (hipStream_t)stream) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

}  // extern "C"
