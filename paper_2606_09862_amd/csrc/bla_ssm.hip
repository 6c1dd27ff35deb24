// The selective state space scan: argument checks, work split and entry points.
#include "bla_ssm.h"

using namespace bla;

namespace {

constexpr long long kFill = 512;  // workgroups that fill the device twice over (256 compute units)
constexpr int kMaxSegments = 64;

bla_status check(const bla_ssm_params* p, bool step)
{
    if (!p) return BLA_ERR_INVALID_ARG;
    if (p->B < 0 || p->H < 0 || p->G < 0 || (!step && p->L < 0) || p->d <= 0 || p->N <= 0) return BLA_ERR_INVALID_ARG;
    if (p->io_dtype != BLA_F32 && p->io_dtype != BLA_BF16) return BLA_ERR_INVALID_ARG;
    if (p->H > 0 && (p->G < 1 || p->H % p->G != 0)) return BLA_ERR_INVALID_ARG;
    if (p->d != 32 && p->d != 64 && p->d != 128) return BLA_ERR_UNSUPPORTED;
    if (p->N > 128 || p->N % 8 != 0) return BLA_ERR_UNSUPPORTED;
    if (!step && p->L > (1 << 30)) return BLA_ERR_UNSUPPORTED;
    const long long nch = step ? 1 : (p->L + kSsmChunk - 1) / kSsmChunk;
    if ((double)p->B * p->H * (nch > 0 ? nch : 1) * (p->d / 32) > kMaxUnits) return BLA_ERR_UNSUPPORTED;
    return BLA_OK;
}

// Segments of a sequence: enough for the workgroups to fill the device, each of at least four chunks (a segment costs the reading and
// writing of a state besides; 8 x 16 heads x 4096 tokens, d = 64, N = 128, bf16: 134 us, with half and twice as many workgroups 151 and 145; 16 heads x 16411
// tokens, d = N = 64, float32: 126, 142 and 145).  All but the last segment have a summary, so where the segments are few the summaries leave a half
// to a quarter of the compute units idle, and are taken in two parts.  With more segments the scan over twice the parts costs more than that (4096 tokens, 16
// heads, d = 64, N = 128, bf16, in one part and in two: 16 rows in two segments 234 and 221 us, 8 rows in four 131 and 124, 6 rows in six 124 and 130, 4 rows in
// eight 78 and 83; float32 likewise, N = 64 in bf16 alike from six on).
struct ForwardPlan {
    int nch, cps, nseg, sub;
    size_t off_decay, total;
};
ForwardPlan forward_plan(const bla_ssm_params* p)
{
    ForwardPlan f;
    f.nch = (p->L + kSsmChunk - 1) / kSsmChunk;
    const long long bh = (long long)p->B * p->H;
    long long n = bh > 0 ? (kFill + bh - 1) / bh : 1;
    if (n > f.nch / 4) n = f.nch / 4;
    n = n < 1 ? 1 : n > kMaxSegments ? kMaxSegments : n;
    f.cps = f.nch > 0 ? (int)((f.nch + n - 1) / n) : 1;
    f.nseg = f.nch > 0 ? (f.nch + f.cps - 1) / f.cps : 1;
    f.sub = f.nseg <= 4 ? 2 : 1;
    const size_t states = (size_t)f.sub * (f.nseg - 1) * bh;
    f.off_decay = seq_align(states * p->N * p->d * 4);
    f.total = f.nseg > 1 ? f.off_decay + seq_align(states * 4) : 0;
    return f;
}

bool fits(const bla_ssm_params* p, const ForwardPlan& f)
{
    const double bh = (double)p->B * p->H;
    return launchable(8.0 * ceil(bh * f.nseg / 8), 256) && launchable(8.0 * ceil(bh * f.sub * (f.nseg - 1) / 8), 256);
}

struct BackwardPlan {
    int nch, hsplit;
    size_t off_leave, off_head, off_bc, total;
};
BackwardPlan backward_plan(const bla_ssm_params* p)
{
    BackwardPlan b;
    b.nch = (p->L + kSsmChunk - 1) / kSsmChunk;
    const size_t bhc = (size_t)p->B * p->H * b.nch, states = seq_align(bhc * p->N * p->d * 4);
    const long long units = (long long)p->B * p->G * b.nch;
    const int rep = p->G > 0 ? p->H / p->G : 1;
    long long n = units > 0 ? (kFill + units - 1) / units : 1;
    if (n > rep) n = rep;
    if (n < 1) n = 1;
    b.hsplit = rep > 0 ? (int)((rep + (rep + n - 1) / n - 1) / ((rep + n - 1) / n)) : 1;  // parts of equal size, none empty
    b.off_leave = states;
    b.off_head = 2 * states;
    b.off_bc = b.off_head + seq_align(bhc * 2 * 8);
    b.total = b.off_bc + (b.hsplit > 1 ? seq_align((size_t)b.hsplit * units * 2 * 64 * p->N * 4) : 0);
    return b;
}

bool fits(const bla_ssm_params* p, const BackwardPlan& b)
{
    return launchable(16.0 * ceil((double)p->B * p->H * (p->d / 32) / 8), 256) && launchable(8.0 * ceil((double)p->B * p->G * b.nch * b.hsplit / 8), 256) &&
           launchable(p->H, 256);
}

struct Sizes {
    size_t x, bc, dt, head, state;
};
Sizes sizes(const bla_ssm_params* p, size_t L)
{
    const size_t e = elem_bytes(p->io_dtype), bh = (size_t)p->B * p->H;
    return {bh * L * p->d * e, (size_t)p->B * p->G * L * p->N * e, bh * L * 4, (size_t)p->H * 4, bh * p->N * p->d * 4};
}

bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

}  // namespace

extern "C" {

bla_status bla_ssm_supported(const bla_ssm_params* p)
{
    const bla_status st = check(p, false);
    return st == BLA_OK && !fits(p, forward_plan(p)) ? BLA_ERR_UNSUPPORTED : st;
}

size_t bla_ssm_workspace_size(const bla_ssm_params* p) { return bla_ssm_supported(p) == BLA_OK ? forward_plan(p).total : 0; }

bla_status bla_ssm_forward(const bla_ssm_params* p, const void* x, const float* dt, const float* A, const void* Bm,
                           const void* Cm, const float* D, const int32_t* lengths, const float* state_in, void* y,
                           float* state_out, void* workspace, size_t workspace_bytes, void* stream)
{
    const bla_status st = check(p, false);
    if (st != BLA_OK) return st;
    if (p->B == 0 || p->H == 0) return BLA_OK;
    const ForwardPlan f = forward_plan(p);
    if (!fits(p, f)) return BLA_ERR_UNSUPPORTED;
    const Sizes z = sizes(p, p->L);
    if (!A || (p->L > 0 && (!x || !dt || !Bm || !Cm || !y))) return BLA_ERR_INVALID_ARG;
    const void* ptr[] = {x, Bm, Cm, state_in, y, state_out};
    for (const void* q : ptr)
        if (q && !is_aligned16(q)) return BLA_ERR_INVALID_ARG;
    if (!aligned4(dt) || !aligned4(A) || !aligned4(D) || !aligned4(lengths)) return BLA_ERR_INVALID_ARG;
    const Span in[] = {{x, z.x}, {Bm, z.bc}, {Cm, z.bc}, {dt, z.dt}, {A, z.head}, {D, z.head}, {state_in, z.state}, {lengths, 4 * (size_t)p->B}};
    const Span out[] = {{y, z.x}, {state_out, z.state}};
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    if (f.total > 0 && (!workspace || workspace_bytes < f.total || !is_aligned16(workspace))) return BLA_ERR_WORKSPACE;
    if (f.total > 0 && !tables_overwritten(workspace, f.total)) return BLA_ERR_HIP;
    SsmArgs a = {};
    a.x = x, a.Bm = Bm, a.Cm = Cm, a.dt = dt, a.A = A, a.Dm = D, a.state_in = state_in, a.lengths = lengths, a.y = y;
    a.state_out = state_out, a.seg_state = (float*)workspace;
    a.seg_decay = f.nseg > 1 ? (float*)((char*)workspace + f.off_decay) : nullptr;
    a.B = p->B, a.H = p->H, a.G = p->G, a.L = p->L, a.N = p->N, a.nch = f.nch, a.cps = f.cps, a.nseg = f.nseg, a.sub = f.sub;
    a.units = (long long)p->B * p->H * f.nseg, a.per = (a.units + 7) / 8;
    return launch_ssm_forward(p->io_dtype == BLA_BF16, p->d, a, (hipStream_t)stream) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

bla_status bla_ssm_step(const bla_ssm_params* p, const void* x, const float* dt, const float* A, const void* Bm,
                        const void* Cm, const float* D, const float* state_in, void* y, float* state_out, void* stream)
{
    const bla_status st = check(p, true);
    if (st != BLA_OK) return st;
    if (p->B == 0 || p->H == 0) return BLA_OK;
    if (!launchable((double)p->B * p->H, 256)) return BLA_ERR_UNSUPPORTED;
    const Sizes z = sizes(p, 1);
    const void* ptr[] = {x, Bm, Cm, state_in, y, state_out};
    for (const void* q : ptr)
        if (!q || !is_aligned16(q)) return BLA_ERR_INVALID_ARG;
    if (!A || !dt || !aligned4(dt) || !aligned4(A) || !aligned4(D)) return BLA_ERR_INVALID_ARG;
    const Span in[] = {{x, z.x}, {Bm, z.bc}, {Cm, z.bc}, {dt, z.dt}, {A, z.head}, {D, z.head}, {state_in == state_out ? nullptr : state_in, z.state}};
    const Span out[] = {{y, z.x}, {state_out, z.state}};
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    const SsmStepArgs a = {x, Bm, Cm, dt, A, D, state_in, y, state_out, p->B, p->H, p->G, p->N};
    return launch_ssm_step(p->io_dtype == BLA_BF16, p->d, a, (hipStream_t)stream) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

size_t bla_ssm_backward_workspace_size(const bla_ssm_params* p)
{
    if (check(p, false) != BLA_OK) return 0;
    const BackwardPlan b = backward_plan(p);
    return fits(p, b) ? b.total : 0;
}

bla_status bla_ssm_backward(const bla_ssm_params* p, const void* x, const float* dt, const float* A, const void* Bm,
                            const void* Cm, const float* D, const void* dy, const int32_t* lengths, const float* state_in,
                            const float* dstate_out, void* dx, float* ddt, float* dA, void* dB, void* dC, float* dD,
                            float* dstate_in, void* workspace, size_t workspace_bytes, void* stream)
{
    const bla_status st = check(p, false);
    if (st != BLA_OK) return st;
    if (p->H == 0 && (p->G == 0 || p->B == 0 || p->L == 0)) return BLA_OK;
    if (p->H == 0 || p->B == 0 || p->L == 0) return BLA_ERR_UNSUPPORTED;
    const BackwardPlan b = backward_plan(p);
    if (!fits(p, b)) return BLA_ERR_UNSUPPORTED;
    const Sizes z = sizes(p, p->L);
    const Span in[] = {{x, z.x}, {Bm, z.bc}, {Cm, z.bc}, {dy, z.x}, {state_in, z.state}, {dstate_out, z.state}, {dt, z.dt}, {A, z.head},
                       {D, z.head}, {lengths, 4 * (size_t)p->B}};
    const Span out[] = {{dx, z.x}, {dB, z.bc}, {dC, z.bc}, {dstate_in, z.state}, {ddt, z.dt}, {dA, z.head}, {dD, z.head}};
    if (!x || !dt || !A || !Bm || !Cm || !dy || !dx || !ddt || !dA || !dB || !dC) return BLA_ERR_INVALID_ARG;
    const void* wide[] = {x, Bm, Cm, dy, state_in, dstate_out, dx, dB, dC, dstate_in};
    for (const void* q : wide)
        if (!is_aligned16(q)) return BLA_ERR_INVALID_ARG;
    const void* narrow[] = {dt, A, D, lengths, ddt, dA, dD};
    for (const void* q : narrow)
        if (!aligned4(q)) return BLA_ERR_INVALID_ARG;
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < b.total || !is_aligned16(workspace)) return BLA_ERR_WORKSPACE;
    if (!tables_overwritten(workspace, b.total)) return BLA_ERR_HIP;
    char* ws = (char*)workspace;
    SsmBwdArgs a = {};
    a.x = x, a.Bm = Bm, a.Cm = Cm, a.dy = dy, a.dt = dt, a.A = A, a.Dm = D, a.state_in = state_in, a.dstate_out = dstate_out;
    a.lengths = lengths, a.dx = dx, a.dBm = dB, a.dCm = dC, a.ddt = ddt, a.dA = dA, a.dD = dD, a.dstate_in = dstate_in;
    a.enter = (float*)ws, a.leave = (float*)(ws + b.off_leave), a.part_head = (double*)(ws + b.off_head);
    a.part_bc = (float*)(ws + b.off_bc);
    a.B = p->B, a.H = p->H, a.G = p->G, a.L = p->L, a.N = p->N, a.nch = b.nch, a.hsplit = b.hsplit;
    a.walk_units = (long long)p->B * p->H * (p->d / 32), a.walk_per = (a.walk_units + 7) / 8;
    a.units = (long long)p->B * p->G * b.nch * b.hsplit, a.per = (a.units + 7) / 8;
    return launch_ssm_backward(p->io_dtype == BLA_BF16, p->d, a, (hipStream_t)stream) == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

}  // extern "C"
