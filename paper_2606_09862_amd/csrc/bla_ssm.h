// The selective state space scan: kernel arguments and what its kernels share.
//
//   h_t = exp(dt_t A) h_{t-1} + dt_t B_t x_t^T   (h: N x d),   y_t = h_t^T C_t + D x_t
// per row and head; the heads of a group share B and C.  In chunks of 64 tokens, with s_t the sum of dt A over the chunk's tokens
// up to t and s_c its whole sum:
//   y_t   = sum_{u <= t} e^{s_t - s_u} dt_u (C_t . B_u) x_u + e^{s_t} h_in^T C_t + D x_t
//   h_out = e^{s_c} h_in + sum_u e^{s_c - s_u} dt_u B_u x_u^T
// Only differences s_t - s_u of a chunk are exponentiated, so nothing overflows where A <= 0.  The sums s run in float64 and are
// kept as two float32 each, so that a difference is as good behind a token that decays by far more than its neighbours (with the upper halves
// alone y was off by nine times its bound in bf16 behind a token of dt A = -1e6).
#pragma once

#include "bla_seq.h"

namespace bla {

constexpr int kSsmChunk = 64;

struct SsmArgs {
    const void *x, *Bm, *Cm;        // [B, H, L, D], [B, G, L, N]
    const float *dt, *A, *Dm;       // [B, H, L], [H], [H] or null
    const float* state_in;          // [B, H, N, D] or null
    const int32_t* lengths;
    void* y;
    float* state_out;               // or null
    float* seg_state;               // [sub (nseg - 1)][B H][N][D]: summaries of the segments' parts, the last part's then the state entering the next segment
    float* seg_decay;               // [sub (nseg - 1)][B H]
    int B, H, G, L, N;
    int nch, cps, nseg, sub;        // chunks, chunks of a segment, segments, parts of a segment's summary
    long long units, per;
};

struct SsmStepArgs {
    const void *x, *Bm, *Cm;        // [B, H, D], [B, G, N]
    const float *dt, *A, *Dm;       // [B, H], [H], [H] or null
    const float* state_in;
    void* y;
    float* state_out;
    int B, H, G, N;
};

struct SsmBwdArgs {
    const void *x, *Bm, *Cm, *dy;
    const float *dt, *A, *Dm, *state_in, *dstate_out;
    const int32_t* lengths;
    void *dx, *dBm, *dCm;
    float *ddt, *dA, *dD, *dstate_in;  // dD, dstate_in: or null
    float* enter;                   // [B H][nch][N][D]: the states entering the chunks
    float* leave;                   // [B H][nch][N][D]: the gradients of the states leaving them
    double* part_head;              // [B H][nch][2]: a chunk's parts of dA and dD
    float* part_bc;                 // hsplit > 1: [hsplit][B][G][nch][2][64][N]
    int B, H, G, L, N, nch, hsplit;
    long long walk_units, walk_per, units, per;
};

// Eight products of a float32 weight and an operand value, as an operand of a contraction whose float32 results keep float32's
// precision: in bf16 as a sum of three roundings (2^-26 relative at most; two would leave 2^-17, which the results of a long sum show), in
// float32 as it is.
template <typename T> struct Split;
template <> struct Split<bf16> {
    bf16x8 hi, mid, lo;
    __device__ __forceinline__ void set(floatx8 v)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            hi[e] = (bf16)v[e];
            const float x = v[e] - (float)hi[e];
            mid[e] = (bf16)x;
            lo[e] = (bf16)(x - (float)mid[e]);
        }
    }
};
template <> struct Split<float> {
    floatx8 hi;
    __device__ __forceinline__ void set(floatx8 v) { hi = v; }
};
// c[i] += a[i] b for N tiles, term by term: consecutive products belong to different tiles and do not wait for each other.
template <int N> __device__ __forceinline__ void mma_split(const bf16x8 (&a)[N], const Split<bf16>& b, floatx4 (&c)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = mma(a[i], b.lo, c[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = mma(a[i], b.mid, c[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = mma(a[i], b.hi, c[i]);
}
template <int N> __device__ __forceinline__ void mma_split(const floatx8 (&a)[N], const Split<float>& b, floatx4 (&c)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = mma(a[i], b.hi, c[i]);
}
__device__ __forceinline__ floatx8 to_f8(bf16x8 x)
{
    floatx8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (float)x[e];
    return r;
}
__device__ __forceinline__ floatx8 to_f8(floatx8 x) { return x; }

// Fragments in the accumulator order of rows of N real columns in memory (zeros past them): the halves lie 16 columns apart.
template <typename T> __device__ __forceinline__ typename Frag<T>::type ld_acc_row(const T* row, int kb, int g, int N)
{
    const int k = 32 * kb + 4 * g;
    return join(k < N ? ld4<T>(row + k) : zero_half<T>(), k + 16 < N ? ld4<T>(row + k + 16) : zero_half<T>());
}
// The same of an LDS tile (row x0 + r, x0 a multiple of 16).
__device__ __forceinline__ bf16x8 ld_acc(const bf16* M, int ld, int x0, int kb, int g, int r)
{
    return ld_frag_2x8(M + (x0 + r) * ld, kb, g);
}
__device__ __forceinline__ floatx8 ld_acc(const float* M, int ld, int x0, int kb, int g, int r)
{
    return ld_frag<float>(M + (x0 + r) * ld, 32 * kb, g);
}

constexpr double kLog2e64 = 1.4426950408889634;

// The exponent (in units of 2) of a token's decay, from the head's rate A log2 e.  Below -2^14 the decay is zero in any type, whatever the exponent, so it
// counts as -2^14 there: a sum of exponents keeps its precision behind such a token, and stays finite where dt A does not.
__device__ __forceinline__ double ssm_rate(float A) { return (double)(A < -__FLT_MAX__ ? -__FLT_MAX__ : A) * kLog2e64; }
__device__ __forceinline__ double ssm_exponent(float dt, double rate)
{
    const double y = (double)dt * rate;
    return y < -16384.0 ? -16384.0 : y;  // a NaN stays
}

// 2^y of a float64 exponent to float32 precision: the part of y that float32 cannot hold goes in as a factor 1 + y_lo ln 2.
__device__ __forceinline__ float exp2_f64(double y)
{
    const float hi = (float)y;
    const float e = exp2_fast(hi);
    return __builtin_fmaf(e, (float)(y - (double)hi) * kLn2, e);
}

// x of the lane that a data-parallel primitive names, zero where there is none.
template <int CTRL, int ROWS> __device__ __forceinline__ double dpp_f64(double x)
{
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, ROWS, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, ROWS, 0xf, false);
    return __hiloint2double(hi, lo);
}

// Inclusive sum over the wave's lanes (lane = token): within rows of 16 lanes, then the last lanes of rows 0 and 2 into rows 1 and 3, then
// lane 31 into the upper half.  In registers; through LDS (six exchanges) it took 900 cycles.
__device__ __forceinline__ double wave_scan(double x)
{
    x += dpp_f64<0x111, 0xf>(x);  // lane - 1
    x += dpp_f64<0x112, 0xf>(x);
    x += dpp_f64<0x114, 0xf>(x);
    x += dpp_f64<0x118, 0xf>(x);
    x += dpp_f64<0x142, 0xa>(x);  // lane 15 of the row before, into rows 1 and 3
    x += dpp_f64<0x143, 0xc>(x);  // lane 31, into rows 2 and 3
    return x;
}
// rows_sum (over the four row groups of a column) of float64 values
__device__ __forceinline__ double rows_sum_f64(double x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
// The last lane's value in every lane.
__device__ __forceinline__ double wave_last(double x)
{
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), 63), __builtin_amdgcn_readlane(__double2loint(x), 63));
}

__device__ __forceinline__ int ssm_length(const int32_t* lengths, int b, int L) { return lengths ? min(max(lengths[b], 0), L) : L; }

hipError_t launch_ssm_forward(int bf16_io, int D, const SsmArgs& a, hipStream_t s);
hipError_t launch_ssm_step(int bf16_io, int D, const SsmStepArgs& a, hipStream_t s);
hipError_t launch_ssm_backward(int bf16_io, int D, const SsmBwdArgs& a, hipStream_t s);

// State rows of a kernel: N padded to 64 or 128 (rows past N are zero and not stored).
inline int ssm_rows(int N) { return N <= 64 ? 64 : 128; }

}  // namespace bla
