// What the 8-bit operators (aqsgd_quant8, aqsgd_matmul8, aqsgd_ffn8) share: the arguments of their
// kernels, elements of any of the three types, the activations.
#pragma once

#include "aqsgd_kernels.h"

namespace aqsgd {

constexpr int kCodePad = 64;                     // vectors of codes start at multiples of this many bytes
constexpr float kCodeHalf = 127.0f;              // largest signed code
constexpr float kLevelHalf = 127.5f;             // half the top level of an 8-bit message
constexpr int64_t kMaxSumLength = 131072;        // 131072 * 127 * 128 < 2^31

inline int64_t code_stride(int64_t length) { return (length + kCodePad - 1) / kCodePad * kCodePad; }

// Four consecutive elements at any element's address.
typedef uint16_t u16x4_any_t __attribute__((ext_vector_type(4), aligned(2)));

template <int DT>
__device__ __forceinline__ f32x4_t load4(const void* base, int64_t idx) {
    if constexpr (DT == AQSGD_F32) {
        return *reinterpret_cast<const f32x4_any_t*>(static_cast<const float*>(base) + idx);
    } else {
        const u16x4_any_t r = *reinterpret_cast<const u16x4_any_t*>(static_cast<const uint16_t*>(base) + idx);
        f32x4_t v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = DT == AQSGD_F16 ? static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(r[e]))) : bf16_bits_to_f32(r[e]);
        return v;
    }
}

typedef uint32_t u32x2_any_t __attribute__((ext_vector_type(2), aligned(2)));

// STREAM: past the caches, for results of which there are many.
template <int DT, bool STREAM>
__device__ __forceinline__ void store4(void* base, int64_t idx, const f32x4_t& v) {
    if constexpr (DT == AQSGD_F32) {
        f32x4_any_t* to = reinterpret_cast<f32x4_any_t*>(static_cast<float*>(base) + idx);
        if constexpr (STREAM) __builtin_nontemporal_store(v, to);
        else *to = v;
    } else {
        u32x2_any_t w;
        if constexpr (DT == AQSGD_F16) {
            typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
            half4_t h;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = static_cast<_Float16>(v[e]);
            w = __builtin_bit_cast(u32x2_any_t, h);
        } else {
            w[0] = f32x2_to_bf16x2(v[0], v[1]);
            w[1] = f32x2_to_bf16x2(v[2], v[3]);
        }
        u32x2_any_t* to = reinterpret_cast<u32x2_any_t*>(static_cast<uint16_t*>(base) + idx);
        if constexpr (STREAM) __builtin_nontemporal_store(w, to);
        else *to = w;
    }
}

// A whole number as an integer by the instruction itself, which takes a NaN to 0 (a conversion from C++ would leave that
// open).
__device__ __forceinline__ int32_t integer_of(float x) {
    int32_t k;
    asm("v_cvt_i32_f32 %0, %1" : "=v"(k) : "v"(x));
    return k;
}

// ---- activations ---------------------------------------------------------------------------
constexpr float kDensity = 0.39894228040143268f;           // 1 / sqrt(2 pi)
constexpr float kTanhSlope = 1.5957691216057308f;          // 2 sqrt(2 / pi)

// exp(x) of an x that is not above 0, a NaN included, for results of type DT.  The hardware's exponential is good to an ulp
// and ends at 2^-126; x log2(e) rounded in front of it puts the result off by |x| half steps of binary32.  float32 results are to
// be right to an ulp, subnormal ones too: the exponential takes only the fraction of x log2(e), formed of two parts of log2(e).
// bfloat16 has 2^-126 and what is below it as well, but |x| half steps of binary32 (88 at most) are nothing next to one of
// its own: the square of exp(x / 2).  What float16 can hold ends long before either.  ffn8 4096 x 6400 x 1600 gated,
// float16 with silu, 101.6 us, with the float32 form 106.2; ffn8_grad of that size not gated, bfloat16, 28.7 and 29.9.
template <int DT>
__device__ __forceinline__ float exp_below(float x) {
    if constexpr (DT == AQSGD_F32) {
        x = x < -150.0f ? -150.0f : x;        // 0 from there on; a NaN stays
        const float whole = rintf(x * 1.44269502f), part = fmaf(x, 1.92596299e-8f, fmaf(x, 1.44269502f, -whole));
        return ldexpf(__builtin_amdgcn_exp2f(part), integer_of(whole));
    } else if constexpr (DT == AQSGD_BF16) {
        const float half = __builtin_amdgcn_exp2f(x * 0.72134752044448170f);
        return half * half;
    } else {
        return __builtin_amdgcn_exp2f(x * 1.44269504088896341f);
    }
}

// p = 1 / (1 + exp(-x)) and q = 1 - p, both without a difference of nearly equal numbers and without an exponential that
// overflows: the exponential, a sum, the hardware's reciprocal and a product, 10 half steps of p and q (float32).
template <int DT>
__device__ __forceinline__ void sigmoids(float x, float& p, float& q) {
    const float e = exp_below<DT>(-fabsf(x)), r = __builtin_amdgcn_rcpf(1.0f + e), er = e * r;
    p = x >= 0.0f ? r : er;
    q = x >= 0.0f ? er : r;                   // a NaN gives e, r and er NaN
}

// (1 + tanh(y / 2)) / 2 is the sigmoid of y; y's own roundings (five half steps) put its tail off by 5 |y| half steps.
__device__ __forceinline__ float tanh_argument(float x) { return kTanhSlope * (x + 0.044715f * x * x * x); }

// The normal distribution's density but for its factor, bell = exp(-x^2 / 2), and its tail beyond |x|, right relative to
// themselves: 1 + erf(x / sqrt(2)) of a negative x is a difference of nearly equal numbers, off by 4 % at -5 and 0 at -6.
// tail / bell falls smoothly from 1/2 to 1 / (|x| sqrt(2 pi)); with t = 1 / (1 + 0.345 |x|) it is t times a polynomial of
// degree 8 in t, least squares on the interval to |x| = 14.5, reweighted until the relative error was level (2.3e-8;
// 5e-8 with rounded coefficients).  float32: x^2 in two parts, 20 half steps of the tail in all.  With erff
// instead, which is not right there: ffn8 4096 x 6400 x 1600 gated float16 119 us, so 109; its ffn8_grad 46.9 and 44.3.
template <int DT>
__device__ __forceinline__ void normal_tail(float x, float& tail, float& bell) {
    const float z = fminf(fabsf(x), 64.0f), square = z * z;            // both are 0 long before; x^2 may be infinite
    bell = exp_below<DT>(-0.5f * square);
    if constexpr (DT == AQSGD_F32) bell = fmaf(-0.5f * fmaf(z, z, -square), bell, bell);
    const float t = __builtin_amdgcn_rcpf(fmaf(z, 0.345f, 1.0f));
    float v = fmaf(t, -0.028151786f, 0.144233525f);
    v = fmaf(t, v, -0.269153446f);
    v = fmaf(t, v, 0.185054511f);
    v = fmaf(t, v, -0.0362378471f);
    v = fmaf(t, v, 0.111267686f);
    v = fmaf(t, v, 0.117362f);
    v = fmaf(t, v, 0.138005242f);
    v = fmaf(t, v, 0.137620106f);
    tail = bell * (t * v);
}

// The normal distribution's function at x.  float32: 1/2 and a series in odd powers up to |x| = 1 (fitted as the tail, 7e-10;
// 3.5e-8 with rounded coefficients), where most of what a layer computes lies and the tail's roundings would be seen: the
// slope's 2-norm error on normal numbers is 4.0e-8 with it, 5.8e-8 without, for 48.7 us of 4096 x 6400 not gated either way.
template <int DT>
__device__ __forceinline__ float normal_below(float x, float tail) {
    const float far = x < 0.0f ? tail : 1.0f - tail;
    if constexpr (DT == AQSGD_F32) {
        const float w = x * x;
        float v = fmaf(w, -7.65400637e-06f, 0.000113485825f);
        v = fmaf(w, v, -0.00118632941f);
        v = fmaf(w, v, 0.00997332297f);
        v = fmaf(w, v, -0.0664903596f);
        v = fmaf(w, v, 0.398942292f);
        return fabsf(x) < 1.0f ? fmaf(x, v, 0.5f) : far;
    }
    return far;
}

template <int DT>
__device__ __forceinline__ float activation(int act, float x) {
    if (act == AQSGD_ACT_GELU) {
        float tail, bell;
        normal_tail<DT>(x, tail, bell);
        return x * normal_below<DT>(x, tail);
    }
    float p, q;
    sigmoids<DT>(act == AQSGD_ACT_SILU ? x : tanh_argument(x), p, q);
    return x * p;
}

// The activation's value and slope.
template <int DT>
__device__ __forceinline__ void activation_slope(int act, float x, float& value, float& slope) {
    if (act == AQSGD_ACT_GELU) {
        float tail, bell;
        normal_tail<DT>(x, tail, bell);
        const float below = normal_below<DT>(x, tail);
        value = x * below;
        slope = below + x * (kDensity * bell);
        return;
    }
    float p, q;
    sigmoids<DT>(act == AQSGD_ACT_SILU ? x : tanh_argument(x), p, q);
    value = x * p;
    if (act == AQSGD_ACT_SILU) {
        slope = p + value * q;
    } else {
        const float near0 = fminf(fmaxf(x, -64.0f), 64.0f);      // beyond, p q is 0 and x^2 may be infinite
        slope = p + near0 * (p * q) * (kTanhSlope * (1.0f + 0.134145f * near0 * near0));
    }
}

// ---- the product's arguments -----------------------------------------------------------------
enum ProductKind {
    kPlain = 0,        // out = product (+ bias) (+ add)
    kMessage,          // the same, a is a message's levels
    kActivation,       // out = act(product + bias), pre = product + bias
    kGated             // out = act(first half) * second half, pre = both
};

struct ProductArgs {
    const uint8_t* a;
    const int8_t* b;
    const float* a_scales;
    const float* b_scales;
    const void* bias;
    const void* add;
    void* out;
    void* pre;
    int64_t lda, ldb;          // bytes
    int32_t m, n, k;           // n: rows of b
    int32_t dtype, act;
    bool stream;               // rows of results are whole sectors of memory
};

struct ProductShape { int32_t m, n, k; };
int64_t product_workspace_bytes(ProductKind kind, const ProductShape& p);
hipError_t launch_product(ProductKind kind, const ProductArgs& p, void* workspace, hipStream_t stream);

// ---- the quantiser's -------------------------------------------------------------------------
struct Quant8Args {
    const void* x;
    int8_t* row_codes;
    float* row_scales;
    int8_t* col_codes;
    float* col_scales;
    float* col_sums;
    void* workspace;
    int64_t ld, row_stride, col_stride;      // elements, bytes, bytes
    int64_t rows, cols;
    uint64_t seed;
};

int64_t quant8_workspace_bytes(int64_t rows, int64_t cols);
hipError_t launch_quant8_empty(float* scales, float* sums, int64_t count, hipStream_t stream);
hipError_t launch_quant8(int dtype, int rounding, const Quant8Args& a, hipStream_t stream);

struct Ffn8GradArgs {
    const void* dh;
    const void* pre;
    void* dpre;
    int64_t m, f;
    int32_t dtype, act, gated;
};
hipError_t launch_ffn8_grad(const Ffn8GradArgs& a, hipStream_t stream);

}  // namespace aqsgd
