// Window attention: entry points.
#include "bla_window_plan.h"

using namespace bla;

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
    bla_status st = check(p, false);
    if (st != BLA_OK) return st;
    if (p->B == 0 || p->H == 0) return empty(p, cache_k_out || cache_v_out);
    const ForwardPlan f = forward_plan(p, cache_k_in != nullptr);
    if (!fits(p, f, cache_k_out != nullptr)) return BLA_ERR_UNSUPPORTED;
    WindowArgs a = {};
    if ((st = forward_args(a, p, f, q, k, v, lengths, pos, cache_k_in, cache_v_in, o, lse, cache_k_out, cache_v_out, kNone, workspace,
                           workspace_bytes)) != BLA_OK)
        return st;
    hipStream_t s = (hipStream_t)stream;
    if ((p->L > 0 || cache_k_out) && launch_window_forward(p->io_dtype == BLA_BF16, p->d, f.waves, a, s) != hipSuccess) return BLA_ERR_HIP;
    return join_parts(p, p->L, f.nsplit, a.part_o, a.part_ml, o, lse, s);
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
    bla_status st = check(p, true);
    if (st != BLA_OK) return st;
    if (p->B == 0 || p->H == 0) return empty(p, true);
    const StepPlan sp = step_plan(p);
    if (!fits(p, sp)) return BLA_ERR_UNSUPPORTED;
    WindowStepArgs a = {};
    if ((st = step_args(a, p, sp, q, k, v, pos, cache_k, cache_v, o, kNone, workspace, sp.total, workspace_bytes)) != BLA_OK) return st;
    hipStream_t s = (hipStream_t)stream;
    if (launch_window_step(p->io_dtype == BLA_BF16, p->d, a, s) != hipSuccess) return BLA_ERR_HIP;
    return join_parts(p, 1, sp.nsplit, a.part_o, a.part_ml, o, nullptr, s);
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
    bla_status st = check(p, false);
    if (st != BLA_OK) return st;
    if (p->t0 != 0) return BLA_ERR_UNSUPPORTED;
    if (p->B == 0 || p->H == 0 || p->L == 0) return empty(p, p->L > 0);
    const BackwardPlan b = backward_plan(p);
    if (!fits(p, b)) return BLA_ERR_UNSUPPORTED;
    WindowBwdArgs a = {};
    if ((st = backward_args(a, p, b, q, k, v, o, lse, dO, lengths, dq, dk, dv, kNone, kNone, workspace, b.total, workspace_bytes)) != BLA_OK)
        return st;
    return launch_window_backward(p->io_dtype == BLA_BF16, p->d, a, (hipStream_t)stream) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

}  // extern "C"
