// Building blocks shared by the window, convolution and selective-scan operators.
#pragma once

#include <math.h>

#include "bla_device.h"
#include "bla_plan.h"

namespace bla {

// Operand fragment of a row whose reduction index is contiguous, in the natural order k(e) = 32kb + 8g + e
// (both operands of a contraction use it): one 16-byte read in bf16, two in float32.
__device__ __forceinline__ bf16x8 ld_nat(const bf16* row, int kb, int g)
{
    return *reinterpret_cast<const bf16x8*>(row + 32 * kb + 8 * g);
}
__device__ __forceinline__ floatx8 ld_nat(const float* row, int kb, int g)
{
    const float* p = row + 32 * kb + 8 * g;
    return join(*reinterpret_cast<const floatx4*>(p), *reinterpret_cast<const floatx4*>(p + 4));
}

// Operand fragment of an LDS tile M[k][x] stored reduction-major, in the accumulator order
// k(e) = 32kb + 16(e/4) + 4g + e%4: the transposing read in bf16, eight reads of a dword in float32 (whose
// products take sixteen times the cycles of bf16's, so the reads hide behind them).
__device__ __forceinline__ bf16x8 ld_red(const bf16* M, int ld, int x0, int kb, int g, int r)
{
    return ld_frag_tr(M, ld, x0, kb, g, r);
}
__device__ __forceinline__ floatx8 ld_red(const float* M, int ld, int x0, int kb, int g, int r)
{
    const float* p = M + (size_t)(32 * kb + 4 * g) * ld + x0 + r;
    floatx8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = p[(16 * (e >> 2) + (e & 3)) * ld];
    return f;
}

// Row strides (elements) of LDS tiles of D columns.  A tile read by rows (ld_nat) is padded by 16 bytes: the sixteen
// rows of a fragment start on different banks.  A tile read transposed is padded to 8 x odd dwords in bf16
// (no conflicts in the transposing reads) and by four dwords in float32 (the four row groups of a
// fragment read 16 banks apart).  A tile read both ways takes the row reads' padding, which leaves the transposing reads of bf16 one overlap in eight
// rows (the 8 x odd dwords that avoid it need a swizzle for the row reads and a sixth more LDS, which costs a workgroup per compute unit).
template <typename T> __host__ __device__ constexpr int nat_ld(int D) { return D + 16 / (int)sizeof(T); }
template <typename T> __host__ __device__ constexpr int red_ld(int D) { return sizeof(T) == 2 ? D + 16 : D + 4; }

// The largest of three, a NaN if one of them is (v_maximum3_f32; fmaxf would first quiet each operand, an instruction apiece).
__device__ __forceinline__ float max3(float a, float b, float c)
{
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Work index of a workgroup: workgroups are dealt to the eight XCDs by index mod 8, so index w works on
// unit (w mod 8) * per + w / 8 and each XCD walks `per` consecutive units, whose shared rows stay in its L2.
__device__ __forceinline__ long long xcd_unit(unsigned w, long long per) { return (long long)(w & 7) * per + (w >> 3); }

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

inline bool is_aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline size_t seq_align(size_t x) { return (x + 255) / 256 * 256; }
inline int elem_bytes(int io_dtype) { return io_dtype == BLA_BF16 ? 2 : 4; }
// whether [a, a + n) and [b, b + m) share a byte
inline bool overlap(const void* a, size_t n, const void* b, size_t m)
{
    return a && b && (uintptr_t)a < (uintptr_t)b + m && (uintptr_t)b < (uintptr_t)a + n;
}
// A tensor of a call (null: not given).
struct Span {
    const void* p;
    size_t n;  // bytes
};
// whether an output shares a byte with an input or with another output
template <int I, int O> bool clash(const Span (&in)[I], const Span (&out)[O])
{
    for (int i = 0; i < O; ++i) {
        for (const Span& x : in)
            if (overlap(out[i].p, out[i].n, x.p, x.n)) return true;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return true;
    }
    return false;
}

// A launch holds fewer than 2^32 threads.
inline bool launchable(double workgroups, int threads) { return workgroups * threads < 4294967296.0; }
constexpr double kMaxUnits = 1 << 24;  // units of work that a plan is made for (its arithmetic stays in 64 bits)

}  // namespace bla
