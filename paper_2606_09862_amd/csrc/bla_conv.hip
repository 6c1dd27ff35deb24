// The short causal convolution of each channel in front of a sequence operator, with its backward pass and its single-token
// form (bla_conv_forward, bla_conv_backward, bla_conv_step).
//
//   z_t = b + sum_{j < K} w_j x_{t-K+1+j},   y_t = z_t or z_t sigmoid(z_t)
// and, with dz_t = dy_t y'(z_t):   dx_n = sum_j w_j dz_{n+K-1-j},   dw_j = sum_t dz_t x_{t-K+1+j},   db = sum_t dz_t.
// The tokens before the call are the K - 1 rows of the state.  All sums are float32.  Bound: the bytes of x and y (and dy, dx).
#include "bla_seq.h"

using namespace bla;

namespace {

constexpr int kMaxTaps = 8;

struct ConvArgs {
    const void* x;
    const float *w, *bias, *state;  // bias, state: or null
    const int32_t* lengths;
    void* y;
    float* state_out;               // or null
    int B, H, L, d, seg, nseg, silu;
    unsigned threads;
};

struct ConvBwdArgs {
    const void *x, *dy;
    const float *w, *bias, *state, *dstate_out;
    const int32_t* lengths;
    void* dx;
    float *dw, *dbias, *dstate_in;  // dbias, dstate_in: or null
    float* part;                    // [parts][H][d][K + 1]
    int B, H, L, d, seg, nchunk, cw, ncb, silu;
    int parts;                      // B * nchunk
};

// PE consecutive elements
template <typename T, int PE> struct Piece { float v[PE]; };
template <typename T, int PE> __device__ __forceinline__ Piece<T, PE> ld_piece(const T* p)
{
    typedef T V __attribute__((ext_vector_type(PE)));
    const V x = *(const V*)p;
    Piece<T, PE> r;
#pragma unroll
    for (int e = 0; e < PE; ++e) r.v[e] = (float)x[e];
    return r;
}
template <typename T, int PE> __device__ __forceinline__ void st_piece(T* p, const float (&v)[PE])
{
    typedef T V __attribute__((ext_vector_type(PE)));
    V x;
#pragma unroll
    for (int e = 0; e < PE; ++e) x[e] = (T)v[e];
    *(V*)p = x;
}
template <int PE> __device__ __forceinline__ void ld_floats(const float* p, float (&v)[PE])
{
#pragma unroll
    for (int e = 0; e < PE; e += 4) {
        const floatx4 x = ld4f(p + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[e + i] = x[i];
    }
}
template <int PE> __device__ __forceinline__ void st_floats(float* p, const float (&v)[PE])
{
#pragma unroll
    for (int e = 0; e < PE; e += 4) st4f(p + e, floatx4{v[e], v[e + 1], v[e + 2], v[e + 3]});
}

__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + exp2_fast(-z * kLog2e)); }

// The taps and bias of PE channels: w[j][e]
template <int K, int PE>
__device__ __forceinline__ void ld_taps(const float* w, const float* bias, size_t c0, float (&t)[K][PE], float (&b)[PE])
{
    float flat[K * PE];
    ld_floats<K * PE>(w + c0 * K, flat);
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
        for (int e = 0; e < PE; ++e) t[j][e] = flat[e * K + j];
#pragma unroll
    for (int e = 0; e < PE; ++e) b[e] = 0.f;
    if (bias) ld_floats<PE>(bias + c0, b);
}

// Token n of the sequence (n < 0: the state's rows, or zero).
template <typename T, int K, int PE>
__device__ __forceinline__ void ld_token(const T* x, const float* state, int n, int d, float (&v)[PE])
{
    if (n >= 0) {
        const Piece<T, PE> p = ld_piece<T, PE>(x + (size_t)n * d);
#pragma unroll
        for (int e = 0; e < PE; ++e) v[e] = p.v[e];
    } else if (state) {
        ld_floats<PE>(state + (size_t)(n + K - 1) * d, v);
    } else {
#pragma unroll
        for (int e = 0; e < PE; ++e) v[e] = 0.f;
    }
}

// A thread takes PE channels and a segment of tokens, with the last K - 1 tokens in registers and eight rows loaded at a time.
template <typename T, int K, int PE> __global__ void __launch_bounds__(256) conv_forward_kernel(ConvArgs a)
{
    constexpr int U = 8;
    typedef T V __attribute__((ext_vector_type(PE)));
    unsigned id = blockIdx.x * 256u + threadIdx.x;
    if (id >= a.threads) return;
    const unsigned nch = (unsigned)a.d / PE;
    const int ch = (int)(id % nch);
    id /= nch;
    const int sg = (int)(id % (unsigned)a.nseg);
    const unsigned bh = id / (unsigned)a.nseg;
    const int b = (int)(bh / (unsigned)a.H), h = (int)(bh % (unsigned)a.H);
    const int len = a.lengths ? min(max(a.lengths[b], 0), a.L) : a.L;
    const T* x = (const T*)a.x + (size_t)bh * a.L * a.d + ch * PE;
    T* y = (T*)a.y + (size_t)bh * a.L * a.d + ch * PE;
    const float* state = a.state ? a.state + (size_t)bh * (K - 1) * a.d + ch * PE : nullptr;

    if (sg == 0 && a.state_out) {
#pragma unroll
        for (int i = 0; i < K - 1; ++i) {
            float v[PE];
            ld_token<T, K, PE>(x, state, len - (K - 1) + i, a.d, v);
            st_floats<PE>(a.state_out + ((size_t)bh * (K - 1) + i) * a.d + ch * PE, v);
        }
    }
    const int t0 = sg * a.seg, t1 = min(a.L, t0 + a.seg), last = min(t1, len);
    int t = t0;
    if (t0 < last) {
        float w[K][PE], bias[PE], past[K][PE];  // past[j]: token t - K + 1 + j (past[K - 1] is set with each token)
        ld_taps<K, PE>(a.w, a.bias, (size_t)h * a.d + ch * PE, w, bias);
#pragma unroll
        for (int j = 0; j < K - 1; ++j) ld_token<T, K, PE>(x, state, t0 - (K - 1) + j, a.d, past[j]);
        auto token = [&](V in, T* to) {
            float z[PE];
#pragma unroll
            for (int e = 0; e < PE; ++e) {
                past[K - 1][e] = (float)in[e];
                z[e] = bias[e];
            }
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int e = 0; e < PE; ++e) z[e] = __builtin_fmaf(w[j][e], past[j][e], z[e]);
            if (a.silu)
#pragma unroll
                for (int e = 0; e < PE; ++e) z[e] *= sigmoid(z[e]);
            st_piece<T, PE>(to, z);
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
#pragma unroll
                for (int e = 0; e < PE; ++e) past[j][e] = past[j + 1][e];
        };
        const T* px = x + (size_t)t0 * a.d;
        T* py = y + (size_t)t0 * a.d;
        for (; t + U <= last; t += U, px += (size_t)U * a.d, py += (size_t)U * a.d) {
            V in[U];
#pragma unroll
            for (int i = 0; i < U; ++i) in[i] = *(const V*)(px + (size_t)i * a.d);
#pragma unroll
            for (int i = 0; i < U; ++i) token(in[i], py + (size_t)i * a.d);
        }
        for (; t < last; ++t, px += a.d, py += a.d) token(*(const V*)px, py);
    }
    const float none[PE] = {};
    for (; t < t1; ++t) st_piece<T, PE>(y + (size_t)t * a.d, none);
}

template <typename T, int K> __global__ void __launch_bounds__(256) conv_step_kernel(ConvArgs a)
{
    constexpr int PE = 4;
    unsigned id = blockIdx.x * 256u + threadIdx.x;
    if (id >= a.threads) return;
    const unsigned nch = (unsigned)a.d / PE;
    const int ch = (int)(id % nch);
    const unsigned bh = id / nch;
    const int h = (int)(bh % (unsigned)a.H);
    const float* state = a.state + (size_t)bh * (K - 1) * a.d + ch * PE;
    float* out = a.state_out + (size_t)bh * (K - 1) * a.d + ch * PE;
    float w[K][PE], z[PE], past[K][PE];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) ld_floats<PE>(state + (size_t)j * a.d, past[j]);
    const Piece<T, PE> p = ld_piece<T, PE>((const T*)a.x + (size_t)bh * a.d + ch * PE);
    ld_taps<K, PE>(a.w, a.bias, (size_t)h * a.d + ch * PE, w, z);
#pragma unroll
    for (int e = 0; e < PE; ++e) past[K - 1][e] = p.v[e];
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
        for (int e = 0; e < PE; ++e) z[e] = __builtin_fmaf(w[j][e], past[j][e], z[e]);
    if (a.silu)
#pragma unroll
        for (int e = 0; e < PE; ++e) z[e] *= sigmoid(z[e]);
    st_piece<T, PE>((T*)a.y + (size_t)bh * a.d + ch * PE, z);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) st_floats<PE>(out + (size_t)j * a.d, past[j + 1]);
}

// A thread takes four channels and a segment of `seg` tokens and walks seg + K - 1 of them, four rows loaded at a time (eight cost a third of
// the waves: 55 us instead of 47 for 8 x 16 heads x 4096 tokens at d = 64, bf16, four taps, the same inputs in every call; 51-54 us with inputs that change from
// call to call, 201 MB, 3.9 TB/s): dz of the last K tokens in registers
// gives dx of the token K - 1 back.  A workgroup holds cw channel threads by 256 / cw segments, adds their taps'
// gradients up in LDS in order and writes one part; conv_taps_kernel adds the parts.
template <typename T, int K> __global__ void __launch_bounds__(256) conv_backward_kernel(ConvBwdArgs a)
{
    constexpr int PE = 4, U = 4;
    __shared__ float red[(K + 1) * PE * 256];
    unsigned u = blockIdx.x;
    const int cb = (int)(u % (unsigned)a.ncb);
    u /= (unsigned)a.ncb;
    const int chunk = (int)(u % (unsigned)a.nchunk);
    const unsigned bh = u / (unsigned)a.nchunk;
    const int b = (int)(bh / (unsigned)a.H), h = (int)(bh % (unsigned)a.H);
    const int rows = 256 / a.cw, col = threadIdx.x % a.cw, row = threadIdx.x / a.cw;
    const int c0 = (cb * a.cw + col) * PE;
    const bool live = c0 < a.d;
    const int len = a.lengths ? min(max(a.lengths[b], 0), a.L) : a.L;

    float dw[K + 1][PE];
#pragma unroll
    for (int j = 0; j <= K; ++j)
#pragma unroll
        for (int e = 0; e < PE; ++e) dw[j][e] = 0.f;

    const int t0 = (chunk * rows + row) * a.seg;
    if (live && (t0 < a.L || t0 == 0)) {
        const T* x = (const T*)a.x + (size_t)bh * a.L * a.d + c0;
        const T* dy = (const T*)a.dy + (size_t)bh * a.L * a.d + c0;
        T* dx = (T*)a.dx + (size_t)bh * a.L * a.d + c0;
        const float* state = a.state ? a.state + (size_t)bh * (K - 1) * a.d + c0 : nullptr;
        const float* dso = a.dstate_out ? a.dstate_out + (size_t)bh * (K - 1) * a.d + c0 : nullptr;
        float* dsi = a.dstate_in ? a.dstate_in + (size_t)bh * (K - 1) * a.d + c0 : nullptr;
        typedef T V __attribute__((ext_vector_type(PE)));
        const int t1 = min(a.L, t0 + a.seg), end = t1 + K - 1;
        float w[K][PE], bias[PE], past[K][PE], dz[K][PE];  // dz[j]: of token t - j
        ld_taps<K, PE>(a.w, a.bias, (size_t)h * a.d + c0, w, bias);
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            if (t0 < len)
                ld_token<T, K, PE>(x, state, t0 - (K - 1) + j, a.d, past[j]);
            else
#pragma unroll
                for (int e = 0; e < PE; ++e) past[j][e] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int e = 0; e < PE; ++e) dz[j][e] = 0.f;
        // dz of a token; the taps' gradients count it in the segment that owns it
        auto token = [&](V xv, V dv, bool own) {
#pragma unroll
            for (int j = K - 1; j > 0; --j)
#pragma unroll
                for (int e = 0; e < PE; ++e) dz[j][e] = dz[j - 1][e];
#pragma unroll
            for (int e = 0; e < PE; ++e) {
                past[K - 1][e] = (float)xv[e];
                float z = bias[e];
#pragma unroll
                for (int j = 0; j < K; ++j) z = __builtin_fmaf(w[j][e], past[j][e], z);
                float g = (float)dv[e];
                if (a.silu) {
                    const float s = sigmoid(z);
                    g *= s * __builtin_fmaf(z, 1.f - s, 1.f);
                }
                dz[0][e] = g;
                g = own ? g : 0.f;
#pragma unroll
                for (int j = 0; j < K; ++j) dw[j][e] = __builtin_fmaf(g, past[j][e], dw[j][e]);
                dw[K][e] += g;
#pragma unroll
                for (int j = 0; j < K - 1; ++j) past[j][e] = past[j + 1][e];
            }
        };
        auto grad = [&](float (&g)[PE]) {  // of the token K - 1 back
#pragma unroll
            for (int e = 0; e < PE; ++e) {
                g[e] = 0.f;
#pragma unroll
                for (int j = 0; j < K; ++j) g[e] = __builtin_fmaf(w[j][e], dz[j][e], g[e]);
            }
        };
        int t = t0;
        auto one = [&]() {  // a token with every case
            if (t < len) {
                token(*(const V*)(x + (size_t)t * a.d), *(const V*)(dy + (size_t)t * a.d), t < t1);
            } else {
#pragma unroll
                for (int j = K - 1; j > 0; --j)
#pragma unroll
                    for (int e = 0; e < PE; ++e) dz[j][e] = dz[j - 1][e];
#pragma unroll
                for (int e = 0; e < PE; ++e) dz[0][e] = 0.f;
            }
            const int n = t - (K - 1);
            ++t;
            if (n < t0 && !(t0 == 0 && n < 0)) return;
            float g[PE];
            grad(g);
            if (dso && n < len && n >= len - (K - 1)) {
                float s[PE];
                ld_floats<PE>(dso + (size_t)(n - len + K - 1) * a.d, s);
#pragma unroll
                for (int e = 0; e < PE; ++e) g[e] += s[e];
            }
            if (n < 0) {
                if (dsi) st_floats<PE>(dsi + (size_t)(n + K - 1) * a.d, g);
            } else {
                if (n >= len)
#pragma unroll
                    for (int e = 0; e < PE; ++e) g[e] = 0.f;
                st_piece<T, PE>(dx + (size_t)n * a.d, g);
            }
        };
        while (t < min(end, t0 + K - 1)) one();
        // groups of tokens whose every gradient is plain: owned, and clear of the state after the last token
        const int clear = min(t1, dso ? len - (K - 1) : len);
        for (; t + U <= clear; t += U) {
            V xi[U], di[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                xi[i] = *(const V*)(x + (size_t)(t + i) * a.d);
                di[i] = *(const V*)(dy + (size_t)(t + i) * a.d);
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                token(xi[i], di[i], true);
                float g[PE];
                grad(g);
                st_piece<T, PE>(dx + (size_t)(t + i - (K - 1)) * a.d, g);
            }
        }
        while (t < end) one();
    }
#pragma unroll
    for (int j = 0; j <= K; ++j)
#pragma unroll
        for (int e = 0; e < PE; ++e) red[(e * (K + 1) + j) * 256 + threadIdx.x] = dw[j][e];
    __syncthreads();
    float* part = a.part + ((size_t)(b * a.nchunk + chunk) * a.H + h) * a.d * (K + 1);
    for (int i = threadIdx.x; i < a.cw * PE * (K + 1); i += 256) {
        const int q = i % (PE * (K + 1)), cl = i / (PE * (K + 1));
        const int c = (cb * a.cw + cl) * PE;
        if (c >= a.d) continue;
        float s = 0.f;
        for (int r = 0; r < rows; ++r) s += red[q * 256 + r * a.cw + cl];
        part[(size_t)c * (K + 1) + q] = s;
    }
}

// dw and db: a workgroup adds the parts of 32 of their elements, eight threads to an element, in a fixed order.
__global__ void __launch_bounds__(256) conv_taps_kernel(ConvBwdArgs a, int K)
{
    __shared__ float red[8][32];
    const size_t n = (size_t)a.H * a.d * (K + 1);
    const int col = threadIdx.x & 31, lane = threadIdx.x >> 5;
    const size_t i = (size_t)blockIdx.x * 32 + col;
    float s = 0.f;
    if (i < n)
        for (int p = lane; p < a.parts; p += 8) s += a.part[(size_t)p * n + i];
    red[lane][col] = s;
    __syncthreads();
    if (lane != 0 || i >= n) return;
#pragma unroll
    for (int r = 1; r < 8; ++r) s += red[r][col];
    const size_t c = i / (K + 1);
    const int j = (int)(i % (K + 1));
    if (j < K)
        a.dw[c * K + j] = s;
    else if (a.dbias)
        a.dbias[c] = s;
}

#define BLA_TAPS(CALL)                                              \
    switch (p->taps) {                                              \
        case 1: CALL(1); break;                                     \
        case 2: CALL(2); break;                                     \
        case 3: CALL(3); break;                                     \
        case 4: CALL(4); break;                                     \
        case 5: CALL(5); break;                                     \
        case 6: CALL(6); break;                                     \
        case 7: CALL(7); break;                                     \
        default: CALL(8); break;                                    \
    }

// Tokens of a thread of the forward kernel: 32, so that the tokens before a segment and the taps are a small part of its loads, or
// eight where that gives the device too few threads.
constexpr int kLongSegment = 32, kShortSegment = 8;
// Channels of a thread there: with four the registers leave room for seven waves on a SIMD (8 x 16 heads x 4096 tokens at d = 64, bf16, four taps: 30 us
// with four channels, 33 with eight; 134 MB, 4.5 TB/s).
constexpr int kForwardChannels = 4;

struct ConvPlan {
    int seg, nseg;
    unsigned long long threads;
    // backward
    int cw, ncb, bseg, nchunk;
    unsigned long long blocks;
    size_t total;
};

bla_status conv_plan(const bla_conv_params* p, bool step, ConvPlan* c)
{
    if (!p) return BLA_ERR_INVALID_ARG;
    if (p->B < 0 || p->H < 0 || (!step && p->L < 0) || p->d <= 0 || p->taps < 1) return BLA_ERR_INVALID_ARG;
    if (p->silu != 0 && p->silu != 1) return BLA_ERR_INVALID_ARG;
    if (p->io_dtype != BLA_F32 && p->io_dtype != BLA_BF16) return BLA_ERR_INVALID_ARG;
    if (p->taps > kMaxTaps || p->d % 8 != 0 || p->d > (1 << 24)) return BLA_ERR_UNSUPPORTED;
    const unsigned long long bh = (unsigned long long)p->B * p->H;
    if (bh > (1ull << 31) || (!step && p->L > (1 << 30))) return BLA_ERR_UNSUPPORTED;
    const int L = step ? 1 : p->L, pe = step ? 4 : kForwardChannels;
    auto threads = [&](int seg) { return bh * (L > seg ? (L + seg - 1) / seg : 1) * (p->d / pe); };
    if ((double)bh * ((L + kLongSegment - 1) / kLongSegment) * (p->d / pe) > 1ull << 31) return BLA_ERR_UNSUPPORTED;  // the sums below stay in 64 bits
    c->seg = threads(kLongSegment) >= (1u << 16) ? kLongSegment : kShortSegment;
    c->nseg = L > c->seg ? (L + c->seg - 1) / c->seg : 1;
    c->threads = threads(c->seg);
    if (c->threads >= (1ull << 31)) return BLA_ERR_UNSUPPORTED;
    // backward: the channel threads of a workgroup are a power of two, at most a wave
    c->cw = 1;
    while (c->cw < 64 && c->cw * 4 < p->d) c->cw *= 2;
    c->ncb = (p->d / 4 + c->cw - 1) / c->cw;
    const int rows = 256 / c->cw;
    auto blocks = [&](int seg) {
        const long long per = (long long)rows * seg;
        return bh * (unsigned long long)(L > per ? (L + per - 1) / per : 1) * c->ncb;
    };
    c->bseg = blocks(kLongSegment) >= 512 ? kLongSegment : kShortSegment;
    const long long per = (long long)rows * c->bseg;
    c->nchunk = (int)(L > per ? (L + per - 1) / per : 1);
    c->blocks = blocks(c->bseg);
    c->total = seq_align((size_t)p->B * c->nchunk * p->H * p->d * (p->taps + 1) * 4);
    return BLA_OK;
}

// whether the backward pass's launches are ones
bool backward_fits(const bla_conv_params* p, const ConvPlan& c)
{
    return launchable((double)c.blocks, 256) && launchable(ceil((double)p->H * p->d * (p->taps + 1) / 32), 256);
}

}  // namespace

extern "C" {

bla_status bla_conv_supported(const bla_conv_params* p)
{
    ConvPlan c;
    return conv_plan(p, false, &c);
}

bla_status bla_conv_forward(const bla_conv_params* p, const void* x, const float* w, const float* bias,
                            const int32_t* lengths, const float* state_in, void* y, float* state_out, void* stream)
{
    ConvPlan c;
    const bla_status st = conv_plan(p, false, &c);
    if (st != BLA_OK) return st;
    if (p->B == 0 || p->H == 0) return BLA_OK;
    const size_t n = (size_t)p->B * p->H * p->L * p->d * elem_bytes(p->io_dtype);
    const size_t ns = (size_t)p->B * p->H * (p->taps - 1) * p->d * 4, nw = (size_t)p->H * p->d * p->taps * 4;
    if (!w || (p->L > 0 && (!x || !y))) return BLA_ERR_INVALID_ARG;
    const void* ptr[] = {x, w, bias, state_in, y, state_out};
    for (const void* q : ptr)
        if (q && !is_aligned16(q)) return BLA_ERR_INVALID_ARG;
    if ((uintptr_t)lengths & 3) return BLA_ERR_INVALID_ARG;
    const Span in[] = {{x, n}, {w, nw}, {bias, (size_t)p->H * p->d * 4}, {state_in, ns}, {lengths, 4 * (size_t)p->B}};
    const Span out[] = {{y, n}, {state_out, ns}};
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    const ConvArgs a = {x, w, bias, state_in, lengths, y, state_out, p->B, p->H, p->L, p->d, c.seg, c.nseg, p->silu,
                        (unsigned)c.threads};
    const dim3 grid((unsigned)((c.threads + 255) / 256));
    hipStream_t s = (hipStream_t)stream;
#define BLA_CALL(K)                                                                                    \
    if (p->io_dtype == BLA_BF16)                                                                       \
        hipLaunchKernelGGL((conv_forward_kernel<bf16, K, kForwardChannels>), grid, dim3(256), 0, s, a);                  \
    else                                                                                               \
        hipLaunchKernelGGL((conv_forward_kernel<float, K, kForwardChannels>), grid, dim3(256), 0, s, a)
    BLA_TAPS(BLA_CALL)
#undef BLA_CALL
    return hipGetLastError() == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

bla_status bla_conv_step(const bla_conv_params* p, const void* x, const float* w, const float* bias, const float* state_in,
                         void* y, float* state_out, void* stream)
{
    ConvPlan c;
    const bla_status st = conv_plan(p, true, &c);
    if (st != BLA_OK) return st;
    if (p->B == 0 || p->H == 0) return BLA_OK;
    const size_t n = (size_t)p->B * p->H * p->d * elem_bytes(p->io_dtype);
    const size_t ns = (size_t)p->B * p->H * (p->taps - 1) * p->d * 4, nw = (size_t)p->H * p->d * p->taps * 4;
    if (!x || !w || !y || (p->taps > 1 && (!state_in || !state_out))) return BLA_ERR_INVALID_ARG;
    const void* ptr[] = {x, w, bias, state_in, y, state_out};
    for (const void* q : ptr)
        if (q && !is_aligned16(q)) return BLA_ERR_INVALID_ARG;
    const Span in[] = {{x, n}, {w, nw}, {bias, (size_t)p->H * p->d * 4}, {state_in == state_out ? nullptr : state_in, ns}};
    const Span out[] = {{y, n}, {state_out, ns}};
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    const ConvArgs a = {x, w, bias, state_in, nullptr, y, state_out, p->B, p->H, 1, p->d, 1, 1, p->silu, (unsigned)c.threads};
    const dim3 grid((unsigned)((c.threads + 255) / 256));
    hipStream_t s = (hipStream_t)stream;
#define BLA_CALL(K)                                                                                    \
    if (p->io_dtype == BLA_BF16)                                                                       \
        hipLaunchKernelGGL((conv_step_kernel<bf16, K>), grid, dim3(256), 0, s, a);                     \
    else                                                                                               \
        hipLaunchKernelGGL((conv_step_kernel<float, K>), grid, dim3(256), 0, s, a)
    BLA_TAPS(BLA_CALL)
#undef BLA_CALL
    return hipGetLastError() == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

size_t bla_conv_backward_workspace_size(const bla_conv_params* p)
{
    ConvPlan c;
    return conv_plan(p, false, &c) == BLA_OK && backward_fits(p, c) ? c.total : 0;
}

bla_status bla_conv_backward(const bla_conv_params* p, const void* x, const float* w, const float* bias, const void* dy,
                             const int32_t* lengths, const float* state_in, const float* dstate_out, void* dx, float* dw,
                             float* dbias, float* dstate_in, void* workspace, size_t workspace_bytes, void* stream)
{
    ConvPlan c;
    const bla_status st = conv_plan(p, false, &c);
    if (st != BLA_OK) return st;
    if (p->B == 0 || p->H == 0) return p->H == 0 ? BLA_OK : BLA_ERR_UNSUPPORTED;
    if (!backward_fits(p, c)) return BLA_ERR_UNSUPPORTED;
    const size_t n = (size_t)p->B * p->H * p->L * p->d * elem_bytes(p->io_dtype);
    const size_t ns = (size_t)p->B * p->H * (p->taps - 1) * p->d * 4, nc = (size_t)p->H * p->d * 4, nw = nc * p->taps;
    if (!w || !dw || (p->L > 0 && (!x || !dy || !dx))) return BLA_ERR_INVALID_ARG;
    const void* ptr[] = {x, w, bias, dy, state_in, dstate_out, dx, dw, dbias, dstate_in};
    for (const void* q : ptr)
        if (q && !is_aligned16(q)) return BLA_ERR_INVALID_ARG;
    if ((uintptr_t)lengths & 3) return BLA_ERR_INVALID_ARG;
    const Span in[] = {{x, n}, {w, nw}, {bias, nc}, {dy, n}, {state_in, ns}, {dstate_out, ns}, {lengths, 4 * (size_t)p->B}};
    const Span out[] = {{dx, n}, {dw, nw}, {dbias, nc}, {dstate_in, ns}};
    if (clash(in, out)) return BLA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < c.total || !is_aligned16(workspace)) return BLA_ERR_WORKSPACE;
    if (!tables_overwritten(workspace, c.total)) return BLA_ERR_HIP;
    const ConvBwdArgs a = {x, dy, w, bias, state_in, dstate_out, lengths, dx, dw, dbias, dstate_in, (float*)workspace,
                           p->B, p->H, p->L, p->d, c.bseg, c.nchunk, c.cw, c.ncb, p->silu, p->B * c.nchunk};
    const dim3 grid((unsigned)c.blocks);
    hipStream_t s = (hipStream_t)stream;
#define BLA_CALL(K)                                                                                    \
    if (p->io_dtype == BLA_BF16)                                                                       \
        hipLaunchKernelGGL((conv_backward_kernel<bf16, K>), grid, dim3(256), 0, s, a);                 \
    else                                                                                               \
        hipLaunchKernelGGL((conv_backward_kernel<float, K>), grid, dim3(256), 0, s, a)
    BLA_TAPS(BLA_CALL)
#undef BLA_CALL
    const size_t taps = (size_t)p->H * p->d * (p->taps + 1);
    hipLaunchKernelGGL(conv_taps_kernel, dim3((unsigned)((taps + 31) / 32)), dim3(256), 0, s, a, p->taps);
    return hipGetLastError() == hipSuccess ? BLA_OK : BLA_ERR_HIP;
}

}  // extern "C"
