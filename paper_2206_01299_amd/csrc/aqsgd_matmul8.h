// Kernels of aqsgd_matmul8 and aqsgd_ffn8: products of 8-bit codes on the matrix units, exact in 32-bit
// integers, with the scales, the bias and the activation applied to the sums before they are stored.
#pragma once

#include "aqsgd_products8.h"

namespace aqsgd {

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));

// A row of b for column c of a tile's columns that start at c0.  In the gated product the columns
// alternate in sixteens between the gate's rows and those it is multiplied with, so that one lane
// ends up with both sums of an element.
template <int KIND>
__device__ __forceinline__ int32_t row_of_b(int32_t c0, int32_t c, int32_t n) {
    if constexpr (KIND == kGated) {
        const int32_t half = n >> 1;
        const int32_t f = min((c0 >> 1) + ((c >> 5) << 4) + (c & 15), half - 1);
        return f + ((c & 16) ? half : 0);
    } else {
        return min(c0 + c, n - 1);
    }
}

// Scales, bias and the rest for four consecutive columns of one row, in binary32.
__device__ __forceinline__ f32x4_t scaled4(const ProductArgs& p, const f32x4_t& sum, float a_step, int32_t n0, int32_t left) {
    f32x4_t v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int32_t c = n0 + (e < left ? e : 0);
        v[e] = sum[e] * a_step * (p.b_scales[c] / kCodeHalf);
        if (p.bias) v[e] += load1(p.dtype, p.bias, c);
    }
    return v;
}

__device__ __forceinline__ void put4(int dtype, void* base, int64_t idx, const f32x4_t& v, int32_t left) {
    if (left >= 4) {
        store4(dtype, base, idx, v);
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < left) store1(dtype, base, idx + e, v[e]);
    }
}

// A tile of 64 x 64 sums by four waves, one 64-byte step of k at a time.
template <int KIND>
__global__ __launch_bounds__(256) void product64_kernel(const ProductArgs p) {
    constexpr int kRow = 80;                                   // bytes of a row in LDS: 64 and a pad
    __shared__ __attribute__((aligned(16))) uint8_t sa[64 * kRow], sb[64 * kRow];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int32_t tiles_n = (p.n + 63) / 64;
    const int32_t m0 = static_cast<int32_t>(blockIdx.x / tiles_n) * 64, n0 = static_cast<int32_t>(blockIdx.x % tiles_n) * 64;
    const int32_t row = t >> 2, piece = (t & 3) * 16;
    const uint8_t* ga = p.a + static_cast<int64_t>(min(m0 + row, p.m - 1)) * p.lda;
    const int8_t* gb = p.b + static_cast<int64_t>(row_of_b<KIND>(n0, row, p.n)) * p.ldb;
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    i32x4_t acc[2][2] = {};
    int32_t ones[2] = {0, 0};
    const int32_t last = KIND == kMessage ? p.k - 16 : 0x7fffffff;     // a message's rows have no padding
    for (int32_t k = 0; k < p.k; k += 64) {
        const i32x4_t va = *reinterpret_cast<const i32x4_t*>(ga + min(k + piece, last));
        const i32x4_t vb = *reinterpret_cast<const i32x4_t*>(gb + k + piece);
        __syncthreads();
        *reinterpret_cast<i32x4_t*>(sa + row * kRow + piece) = va;
        *reinterpret_cast<i32x4_t*>(sb + row * kRow + piece) = vb;
        __syncthreads();
        i32x4_t fa[2], fb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            fa[i] = *reinterpret_cast<const i32x4_t*>(sa + (wm + 16 * i + (lane & 15)) * kRow + (lane >> 4) * 16);
            fb[i] = *reinterpret_cast<const i32x4_t*>(sb + (wn + 16 * i + (lane & 15)) * kRow + (lane >> 4) * 16);
            if constexpr (KIND == kMessage) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    fa[i][e] ^= static_cast<int32_t>(0x80808080u);                      // level - 128
                    ones[i] = __builtin_amdgcn_sdot4(fb[i][e], 0x01010101, ones[i], false);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
    if constexpr (KIND == kMessage) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            ones[j] += __shfl_xor(ones[j], 16, kWave);
            ones[j] += __shfl_xor(ones[j], 32, kWave);
        }
    }
    const int cn = (lane >> 4) * 4;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int32_t m = m0 + wm + 16 * i + (lane & 15);
        const float a_step = p.a_scales[min(m, p.m - 1)] / (KIND == kMessage ? kLevelHalf : kCodeHalf);
        f32x4_t sum[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum[j][e] = static_cast<float>(acc[i][j][e]);
                if constexpr (KIND == kMessage)
                    sum[j][e] += 0.5f * static_cast<float>(__shfl(ones[j], cn + e, kWave));   // levels - 127.5
            }
        }
        if (m >= p.m) continue;
        if constexpr (KIND == kGated) {
            const int32_t half = p.n >> 1, f = ((n0 + wn) >> 1) + cn, left = half - f;
            if (left <= 0) continue;
            const f32x4_t g = scaled4(p, sum[0], a_step, f, left), u = scaled4(p, sum[1], a_step, half + f, left);
            f32x4_t h;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = activation(p.act, g[e]) * u[e];
            put4(p.dtype, p.out, static_cast<int64_t>(m) * half + f, h, left);
            if (p.pre) {
                put4(p.dtype, p.pre, static_cast<int64_t>(m) * p.n + f, g, left);
                put4(p.dtype, p.pre, static_cast<int64_t>(m) * p.n + half + f, u, left);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int32_t n = n0 + wn + 16 * j + cn, left = p.n - n;
                if (left <= 0) continue;
                f32x4_t v = scaled4(p, sum[j], a_step, n, left);
                const int64_t at = static_cast<int64_t>(m) * p.n + n;
                if constexpr (KIND == kActivation) {
                    if (p.pre) put4(p.dtype, p.pre, at, v, left);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = activation(p.act, v[e]);
                } else if (p.add) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < left) v[e] += load1(p.dtype, p.add, at + e);
                }
                put4(p.dtype, p.out, at, v, left);
            }
        }
    }
}

}  // namespace aqsgd
