// Kernels of aqsgd_quant8: signed 8-bit codes with a scale for each row, for each column, or both.
#pragma once

#include "aqsgd_products8.h"

namespace aqsgd {

// Max-abs on bit patterns: infinities and NaN order above every finite value, so they are not lost.
__device__ __forceinline__ uint32_t magnitude_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

struct CodeScale {
    float scale;       // stored: max-abs, 0 below 2^-120, NaN where it is not finite
    float inv;         // 127 / scale, or 0: every code is then 0
};

__device__ __forceinline__ CodeScale code_scale(uint32_t bits) {
    const float s = __uint_as_float(bits);
    const bool finite = bits < 0x7f800000u, live = finite && !(s < 0x1p-120f);
    CodeScale c;
    c.scale = live ? s : finite ? 0.0f : __uint_as_float(0x7fc00000u);
    c.inv = live ? kCodeHalf / (live ? s : 1.0f) : 0.0f;
    return c;
}

// Code of one value; a NaN or an infinity meets inv = 0 and must give 0, which the clamps see to
// (fmaxf and fminf return the number among a number and a NaN).
__device__ __forceinline__ int32_t code_of(float x, float inv, float r) {
    const float t = x * inv;
    return static_cast<int32_t>(fminf(fmaxf(floorf(inv == 0.0f ? r : t + r), -kCodeHalf), kCodeHalf));
}

// Uniform draw of element (row, col); which = 1 for row codes, 2 for column codes.
__device__ __forceinline__ float code_draw(uint64_t seed, int64_t row, int64_t col, uint32_t which) {
    uint32_t w[4];
    philox4x32_10(static_cast<uint32_t>(col >> 2) | (which << 30), static_cast<uint32_t>(row), static_cast<uint32_t>(seed),
                  static_cast<uint32_t>(seed >> 32), w);
    const int k = static_cast<int>(col & 3);
    return uniform_from_word(k == 0 ? w[0] : k == 1 ? w[1] : k == 2 ? w[2] : w[3]);
}

template <int ROUND>
__device__ __forceinline__ float code_offset(uint64_t seed, int64_t row, int64_t col, uint32_t which) {
    if constexpr (ROUND == AQSGD_ROUND_STOCHASTIC) return code_draw(seed, row, col, which);
    else return 0.5f;
}

// A workgroup per row.
template <int DT, int ROUND>
__global__ __launch_bounds__(256) void quant8_rows_kernel(const Quant8Args a) {
    __shared__ uint32_t part[4];
    const int64_t row = blockIdx.x, base = row * a.ld;
    uint32_t top = 0;
    for (int64_t c = threadIdx.x; c < a.cols; c += 256) top = max(top, magnitude_bits(load_elem<DT>(a.x, base + c)));
    top = __float_as_uint(team_max<64>(__uint_as_float(top)));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
    __syncthreads();
    const CodeScale s = code_scale(max(max(part[0], part[1]), max(part[2], part[3])));
    if (threadIdx.x == 0) a.row_scales[row] = s.scale;
    int8_t* out = a.row_codes + row * a.row_stride;
    for (int64_t c = threadIdx.x; c < a.row_stride; c += 256)
        out[c] = c < a.cols ? static_cast<int8_t>(code_of(load_elem<DT>(a.x, base + c), s.inv,
                                                          code_offset<ROUND>(a.seed, row, c, 1))) : 0;
}

// Columns, first pass: max-abs (and sum) of each column over a block of rows, one lane a column.
constexpr int64_t kColBlocks = 64;               // blocks of rows at most
inline int64_t col_block_rows(int64_t rows) { return rows <= 64 * kColBlocks ? 64 : (rows + kColBlocks - 1) / kColBlocks; }
inline int64_t col_blocks(int64_t rows) { return (rows + col_block_rows(rows) - 1) / col_block_rows(rows); }

template <int DT>
__global__ __launch_bounds__(64) void quant8_colmax_kernel(const Quant8Args a, int64_t block_rows, bool sums) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x;
    const int64_t r0 = blockIdx.y * block_rows, r1 = min(r0 + block_rows, a.rows);
    if (c >= a.cols) return;
    uint32_t top = 0;
    float sum = 0.0f;
    for (int64_t r = r0; r < r1; ++r) {
        const float x = load_elem<DT>(a.x, r * a.ld + c);
        top = max(top, magnitude_bits(x));
        sum += x;
    }
    uint32_t* tops = static_cast<uint32_t*>(a.workspace);
    tops[blockIdx.y * a.cols + c] = top;
    if (sums) reinterpret_cast<float*>(tops + gridDim.y * a.cols)[blockIdx.y * a.cols + c] = sum;
}

// Second pass: a tile of 64 columns x 64 rows goes through LDS to come out transposed.
template <int DT, int ROUND>
__global__ __launch_bounds__(256) void quant8_cols_kernel(const Quant8Args a, int64_t blocks) {
    __shared__ int8_t tile[64][68];
    __shared__ float inv[64];
    const int64_t c0 = static_cast<int64_t>(blockIdx.x) * 64, r0 = static_cast<int64_t>(blockIdx.y) * 64;
    const uint32_t* tops = static_cast<const uint32_t*>(a.workspace);
    if (threadIdx.x < 64 && c0 + threadIdx.x < a.cols) {
        const int64_t c = c0 + threadIdx.x;
        uint32_t top = 0;
        float sum = 0.0f;
        for (int64_t b = 0; b < blocks; ++b) {
            top = max(top, tops[b * a.cols + c]);
            if (a.col_sums && blockIdx.y == 0) sum += reinterpret_cast<const float*>(tops + blocks * a.cols)[b * a.cols + c];
        }
        const CodeScale s = code_scale(top);
        inv[threadIdx.x] = s.inv;
        if (blockIdx.y == 0) {
            if (a.col_scales) a.col_scales[c] = s.scale;
            if (a.col_sums) a.col_sums[c] = sum;
        }
    }
    __syncthreads();
    if (!a.col_codes) return;
    const int cx = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < 64; r += 4) {
        const int64_t row = r0 + r, c = c0 + cx;
        tile[cx][r] = row < a.rows && c < a.cols ? static_cast<int8_t>(code_of(load_elem<DT>(a.x, row * a.ld + c), inv[cx],
                                                                              code_offset<ROUND>(a.seed, row, c, 2))) : 0;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < 64 * 16; k += 256) {
        const int64_t c = c0 + (k >> 4);
        if (c >= a.cols) continue;
        const int8_t* t = &tile[k >> 4][(k & 15) * 4];
        *reinterpret_cast<uint32_t*>(a.col_codes + c * a.col_stride + r0 + (k & 15) * 4) =
            *reinterpret_cast<const uint32_t*>(t);
    }
}

template <int DT, int ROUND>
hipError_t launch_quant8_as(const Quant8Args& a, hipStream_t stream) {
    ProfileSpan span;
    const bool cols = a.col_codes || a.col_sums;
    hipError_t err = hipSuccess;
    if (a.row_codes) {
        if (!cols) span.last();
        err = launch_kernel(quant8_rows_kernel<DT, ROUND>, dim3(static_cast<unsigned>(a.rows)), dim3(256), stream, a);
    }
    if (cols && err == hipSuccess) {
        const int64_t blocks = col_blocks(a.rows);
        const unsigned gx = static_cast<unsigned>((a.cols + 63) / 64);
        err = launch_kernel(quant8_colmax_kernel<DT>, dim3(gx, static_cast<unsigned>(blocks)), dim3(64), stream, a,
                            col_block_rows(a.rows), a.col_sums != nullptr);
        span.last();
        if (err == hipSuccess)
            err = launch_kernel(quant8_cols_kernel<DT, ROUND>,
                                dim3(gx, a.col_codes ? static_cast<unsigned>((a.rows + 63) / 64) : 1u), dim3(256), stream, a, blocks);
    }
    return err;
}

}  // namespace aqsgd
