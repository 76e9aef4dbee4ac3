// Kernels of aqsgd_quant8: signed 8-bit codes with a scale for each row, for each column, or both.
//
// Rows alone are read once: a team of lanes holds its row in registers between the max-abs and the codes.  A
// column's max-abs needs every row, so columns take two passes: the first leaves the max-abs of blocks of rows
// (and, where rows are wanted too, of blocks of columns), the second joins them, quantises a tile both ways from
// one read and turns the column codes round in LDS.  What bounds all of it is memory.
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

// Code of one value.  x * inv is within an ulp of [-127, 127], so a nearest code needs no clamp; where inv is 0 an
// infinity or a NaN makes the product a NaN, which the conversion takes to 0 (one from C++ would leave that open;
// the conversion that rounds down by itself does not do so for every NaN).
template <int ROUND>
__device__ __forceinline__ int32_t code_of(float x, float inv, float r) {
    const float y = floorf(x * inv + r);
    int32_t k;
    asm("v_cvt_i32_f32 %0, %1" : "=v"(k) : "v"(y));
    if constexpr (ROUND == AQSGD_ROUND_STOCHASTIC) k = min(max(k, -127), 127);
    return k;
}

// The low bytes of four codes.
__device__ __forceinline__ uint32_t pack_codes(int32_t a, int32_t b, int32_t c, int32_t d) {
    const uint32_t ab = __builtin_amdgcn_perm(static_cast<uint32_t>(b), static_cast<uint32_t>(a), 0x0c0c0400u);
    const uint32_t cd = __builtin_amdgcn_perm(static_cast<uint32_t>(d), static_cast<uint32_t>(c), 0x04000c0cu);
    return ab | cd;
}

// Rounding offsets of eight consecutive columns from a multiple of 8 on; which = 1 for row codes, 2 for column codes.
template <int ROUND>
__device__ __forceinline__ void code_offsets(uint64_t seed, int64_t row, int64_t col, uint32_t which, float (&r)[kChunk]) {
    if constexpr (ROUND == AQSGD_ROUND_STOCHASTIC) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            uint32_t w[4];
            philox4x32_10((static_cast<uint32_t>(col >> 2) + b) | (which << 30), static_cast<uint32_t>(row), static_cast<uint32_t>(seed),
                          static_cast<uint32_t>(seed >> 32), w);
#pragma unroll
            for (int e = 0; e < 4; ++e) r[4 * b + e] = uniform_from_word(w[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kChunk; ++e) r[e] = 0.5f;
    }
}

// Up to eight elements from any element's address; those past the count are 0.
template <int DT>
__device__ __forceinline__ Raw<DT> load_some(const char* p, int64_t count) {
    if (count >= kChunk) {
        Raw<DT> r;
        if constexpr (DT == AQSGD_F32) {
            r.lo = *reinterpret_cast<const f32x4_any_t*>(p);
            r.hi = *reinterpret_cast<const f32x4_any_t*>(p + 16);
        } else {
            r.v = *reinterpret_cast<const u32x4_any_t*>(p);
        }
        return r;
    }
    Raw<DT> r = zero_raw<DT>();
#pragma unroll
    for (int e = 0; e < kChunk - 1; ++e) {
        if (e >= count) continue;
        if constexpr (DT == AQSGD_F32) {
            const float v = reinterpret_cast<const float*>(p)[e];
            if (e < 4) r.lo[e] = v; else r.hi[e - 4] = v;
        } else {
            r.v[e >> 1] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(p)[e]) << (16 * (e & 1));
        }
    }
    return r;
}

template <int DT>
__device__ __forceinline__ const char* element_at(const void* base, int64_t i) {
    return static_cast<const char*>(base) + i * ElemBytes<DT>::value;
}

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// ---- rows alone ---------------------------------------------------------------------------------
// TEAM lanes to a row (a wave's fraction, a wave or a workgroup of 256), CPL chunks of eight elements a lane;
// CPL = 0: a workgroup to a row of any width, which is read twice.
template <int DT, int ROUND, int TEAM, int CPL>
__global__ __launch_bounds__(256) void quant8_rows_kernel(const Quant8Args a) {
    constexpr int kRows = 256 / TEAM;
    __shared__ uint32_t part[4];
    const int lane = threadIdx.x % TEAM;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * kRows; first < a.rows; first += static_cast<int64_t>(gridDim.x) * kRows) {
        const int64_t row = first + threadIdx.x / TEAM;
        const bool here = row < a.rows;
        const int64_t base = (here ? row : 0) * a.ld;
        Raw<DT> held[CPL > 0 ? CPL : 1];
        uint32_t top = 0;
        auto see = [&](const Raw<DT>& raw) {
            float f[kChunk];
            unpack_raw<DT>(raw, f);
#pragma unroll
            for (int e = 0; e < kChunk; ++e) top = max(top, magnitude_bits(f[e]));
        };
        if constexpr (CPL > 0) {
#pragma unroll
            for (int i = 0; i < CPL; ++i) {
                const int64_t c = (static_cast<int64_t>(i) * TEAM + lane) * kChunk;
                held[i] = load_some<DT>(element_at<DT>(a.x, base + min(c, a.cols)), a.cols - c);
            }
#pragma unroll
            for (int i = 0; i < CPL; ++i) see(held[i]);
        } else {
            for (int64_t c = static_cast<int64_t>(lane) * kChunk; c < a.cols; c += TEAM * kChunk)
                see(load_some<DT>(element_at<DT>(a.x, base + c), a.cols - c));
        }
        top = __float_as_uint(team_max<(TEAM < 64 ? TEAM : 64)>(__uint_as_float(top)));
        if constexpr (TEAM > 64) {
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
            __syncthreads();
            top = max(max(part[0], part[1]), max(part[2], part[3]));
            __syncthreads();
        }
        const CodeScale s = code_scale(top);
        if (!here) break;
        if (lane == 0) a.row_scales[row] = s.scale;
        int8_t* out = a.row_codes + row * a.row_stride;
        auto send = [&](const Raw<DT>& raw, int64_t c) {
            float f[kChunk], r[kChunk];
            unpack_raw<DT>(raw, f);
            code_offsets<ROUND>(a.seed, row, c, 1, r);
            int32_t k[kChunk];
#pragma unroll
            for (int e = 0; e < kChunk; ++e) k[e] = code_of<ROUND>(f[e], s.inv, r[e]);
            *reinterpret_cast<u32x2_t*>(out + c) = u32x2_t{pack_codes(k[0], k[1], k[2], k[3]), pack_codes(k[4], k[5], k[6], k[7])};
        };
        if constexpr (CPL > 0) {
#pragma unroll
            for (int i = 0; i < CPL; ++i) {
                const int64_t c = (static_cast<int64_t>(i) * TEAM + lane) * kChunk;
                if (c < a.row_stride) send(held[i], c);
            }
        } else {
            for (int64_t c = static_cast<int64_t>(lane) * kChunk; c < a.row_stride; c += TEAM * kChunk)
                send(load_some<DT>(element_at<DT>(a.x, base + min(c, a.cols)), a.cols - c), c);
        }
    }
}

// ---- columns, with or without rows --------------------------------------------------------------
// First pass: a workgroup takes kSpan columns of a block of rows, 32 lanes of eight columns side by side, eight
// rows at a time.
constexpr int kSpan = 256;
constexpr int kTile = 128;                        // side of the second pass's tiles

struct ColumnPlan {
    int64_t blocks, block_rows;                   // of the first pass
    int64_t spans;
    int64_t tiles_c, bands, band_tiles;           // of the second: tiles across, workgroups down, tiles of each
};

// The second pass reads a block's maxima again for every tile, so there are at most 32 blocks of rows (or as many
// as give 128 workgroups where the columns are few), and a workgroup takes several tiles, one below the other,
// once there are enough of them for the chip.
inline ColumnPlan column_plan(int64_t rows, int64_t cols) {
    ColumnPlan p;
    p.spans = (cols + kSpan - 1) / kSpan;
    const int64_t most = p.spans >= 4 ? 32 : 128 / p.spans;
    const int64_t want = (rows + 63) / 64 < most ? (rows + 63) / 64 : most;
    p.block_rows = (rows + want - 1) / want;
    p.blocks = (rows + p.block_rows - 1) / p.block_rows;
    p.tiles_c = (cols + kTile - 1) / kTile;
    const int64_t tiles_r = (rows + kTile - 1) / kTile, each = p.tiles_c * tiles_r / 1024;
    p.band_tiles = each < 1 ? 1 : each > 8 ? 8 : each;
    p.bands = (tiles_r + p.band_tiles - 1) / p.band_tiles;
    return p;
}

// The workspace: maxima of columns [blocks, cols], sums of columns [blocks, cols], maxima of rows [spans, rows].
struct ColumnSpace {
    uint32_t* col_tops;
    float* col_sums;
    uint32_t* row_tops;
};
__host__ __device__ inline ColumnSpace column_space(void* workspace, const ColumnPlan& p, int64_t cols) {
    uint32_t* w = static_cast<uint32_t*>(workspace);
    return {w, reinterpret_cast<float*>(w + p.blocks * cols), w + 2 * p.blocks * cols};
}

template <int DT, bool ROWS, bool SUMS>
__global__ __launch_bounds__(256) void quant8_maxima_kernel(const Quant8Args a, const ColumnPlan p) {
    constexpr int kAhead = 4;                      // rows of a lane that are on their way at a time
    __shared__ uint32_t tops[8][kSpan + 8];
    __shared__ float sums[SUMS ? 8 : 1][SUMS ? kSpan + 8 : 1];
    const ColumnSpace w = column_space(a.workspace, p, a.cols);
    const int64_t span = blockIdx.x % p.spans, block = blockIdx.x / p.spans;
    const int lane = threadIdx.x & 31, slot = threadIdx.x >> 5;
    const int64_t c = span * kSpan + lane * kChunk, left = a.cols - c;
    const int64_t r0 = block * p.block_rows, r1 = min(r0 + p.block_rows, a.rows);
    uint32_t top[kChunk] = {};
    float sum[kChunk] = {};
    for (int64_t r = r0 + slot; r < r1; r += 8 * kAhead) {
        Raw<DT> raw[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t q = r + 8 * i;
            raw[i] = q < r1 ? load_some<DT>(element_at<DT>(a.x, q * a.ld + min(c, a.cols)), left) : zero_raw<DT>();
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            float f[kChunk];
            unpack_raw<DT>(raw[i], f);
            uint32_t row_top = 0;
#pragma unroll
            for (int e = 0; e < kChunk; ++e) {
                const uint32_t m = magnitude_bits(f[e]);
                top[e] = max(top[e], m);
                if constexpr (ROWS) row_top = max(row_top, m);
                if constexpr (SUMS) sum[e] += f[e];
            }
            if constexpr (ROWS) {
                row_top = __float_as_uint(team_max<32>(__uint_as_float(row_top)));
                if (lane == 0 && r + 8 * i < r1) w.row_tops[span * a.rows + r + 8 * i] = row_top;
            }
        }
    }
#pragma unroll
    for (int e = 0; e < kChunk; ++e) {
        tops[slot][lane * kChunk + e] = top[e];
        if constexpr (SUMS) sums[slot][lane * kChunk + e] = sum[e];
    }
    __syncthreads();
    const int64_t mine = span * kSpan + threadIdx.x;
    if (mine >= a.cols) return;
    uint32_t m = 0;
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        m = max(m, tops[k][threadIdx.x]);
        if constexpr (SUMS) s += sums[k][threadIdx.x];
    }
    w.col_tops[block * a.cols + mine] = m;
    if constexpr (SUMS) w.col_sums[block * a.cols + mine] = s;
}

// Sums alone: the blocks' sums joined in order.
static __global__ __launch_bounds__(256) void quant8_sums_kernel(const Quant8Args a, const ColumnPlan p) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (c >= a.cols) return;
    const ColumnSpace w = column_space(a.workspace, p, a.cols);
    float s = 0.0f;
    for (int64_t b = 0; b < p.blocks; ++b) s += w.col_sums[b * a.cols + c];
    a.col_sums[c] = s;
}

// Second pass.  A lane takes eight columns of four neighbouring rows, twice: its row codes are whole 8-byte pieces
// of a row, its column codes four rows of a column to a word, and those words meet in LDS.  There a column's
// 32 words lie in pieces of four, piece k of column c at place k ^ (c / 8 % 8), so that neither side crowds a bank.
template <int DT, int ROUND, bool ROWS>
__global__ __launch_bounds__(256) void quant8_tiles_kernel(const Quant8Args a, const ColumnPlan p) {
    __shared__ __attribute__((aligned(16))) uint32_t turned[kTile * 32];
    __shared__ float inv_r[kTile], inv_c[kTile];
    __shared__ uint32_t other[kTile];
    const ColumnSpace w = column_space(a.workspace, p, a.cols);
    const int64_t tc = blockIdx.x % p.tiles_c, band = blockIdx.x / p.tiles_c;
    const int64_t c0 = tc * kTile;
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int64_t c = c0 + lane * kChunk, left = a.cols - c;
    {
        // each column's maxima by two threads
        const int64_t mine = min(c0 + (threadIdx.x & 127), a.cols - 1);
        uint32_t top = 0;
#pragma unroll 8
        for (int64_t b = threadIdx.x >> 7; b < p.blocks; b += 2) top = max(top, w.col_tops[b * a.cols + mine]);
        if (threadIdx.x >= 128) other[threadIdx.x & 127] = top;
        __syncthreads();
        if (threadIdx.x < 128) {
            const CodeScale s = code_scale(max(top, other[threadIdx.x]));
            inv_c[threadIdx.x] = s.inv;
            if (band == 0 && c0 + threadIdx.x < a.cols) {
                a.col_scales[mine] = s.scale;
                if (a.col_sums) {
                    float sum = 0.0f;
                    for (int64_t b = 0; b < p.blocks; ++b) sum += w.col_sums[b * a.cols + mine];
                    a.col_sums[mine] = sum;
                }
            }
        }
    }
    const int64_t t1 = min((band + 1) * p.band_tiles * kTile, a.rows);
    for (int64_t r0 = band * p.band_tiles * kTile; r0 < t1; r0 += kTile) {
        Raw<DT> raw[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = r0 + group * 4 + (i & 3) + (i >> 2) * 64;
            raw[i] = r < a.rows ? load_some<DT>(element_at<DT>(a.x, r * a.ld + min(c, a.cols)), left) : zero_raw<DT>();
        }
        if constexpr (ROWS) {
            if (threadIdx.x < kTile) {
                const int64_t r = min(r0 + threadIdx.x, a.rows - 1);
                uint32_t top = 0;
#pragma unroll 4
                for (int64_t s = 0; s < p.spans; ++s) top = max(top, w.row_tops[s * a.rows + r]);
                const CodeScale s = code_scale(top);
                inv_r[threadIdx.x] = s.inv;
                if (tc == 0 && r0 + threadIdx.x < a.rows) a.row_scales[r] = s.scale;
            }
        }
        __syncthreads();
        float ic[kChunk];
#pragma unroll
        for (int e = 0; e < kChunk; ++e) ic[e] = inv_c[lane * kChunk + e];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t word[kChunk];                 // four rows of each column
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t r = r0 + group * 4 + i + h * 64;
                float f[kChunk], u[kChunk];
                unpack_raw<DT>(raw[4 * h + i], f);
                if constexpr (ROWS) {
                    int32_t k[kChunk];
                    const float ir = inv_r[group * 4 + i + h * 64];
                    code_offsets<ROUND>(a.seed, r, c, 1, u);
#pragma unroll
                    for (int e = 0; e < kChunk; ++e) k[e] = code_of<ROUND>(f[e], ir, u[e]);
                    if (r < a.rows && c < a.row_stride)
                        *reinterpret_cast<u32x2_t*>(a.row_codes + r * a.row_stride + c) =
                            u32x2_t{pack_codes(k[0], k[1], k[2], k[3]), pack_codes(k[4], k[5], k[6], k[7])};
                }
                code_offsets<ROUND>(a.seed, r, c, 2, u);
#pragma unroll
                for (int e = 0; e < kChunk; ++e) {
                    const uint32_t k = static_cast<uint32_t>(code_of<ROUND>(f[e], ic[e], u[e]));
                    word[e] = i == 0 ? k & 0xffu
                                     : __builtin_amdgcn_perm(k, word[e], i == 1 ? 0x0c0c0400u : i == 2 ? 0x0c040100u : 0x04020100u);
                }
            }
            const int at = ((group >> 2) + 4 * h) ^ (lane & 7);
#pragma unroll
            for (int e = 0; e < kChunk; ++e) turned[(lane * kChunk + e) * 32 + at * 4 + (group & 3)] = word[e];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = threadIdx.x + 256 * i, col = k >> 3, piece = k & 7;
            const int64_t out_c = c0 + col, out_r = r0 + piece * 16;
            if (out_c < a.cols && out_r < a.col_stride)
                *reinterpret_cast<u32x4_t*>(a.col_codes + out_c * a.col_stride + out_r) =
                    *reinterpret_cast<const u32x4_t*>(&turned[col * 32 + ((piece ^ (col >> 3 & 7)) * 4)]);
        }
        __syncthreads();
    }
}

constexpr int64_t kMostBlocks = int64_t{1} << 22;     // 2^30 lanes: a grid takes fewer than 2^32

template <int DT, int ROUND>
hipError_t launch_quant8_rows(const Quant8Args& a, hipStream_t stream) {
    const auto go = [&](void (*kernel)(const Quant8Args), int team) {
        const int64_t per = 256 / team, blocks = (a.rows + per - 1) / per;
        return launch_kernel(kernel, dim3(static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks)), dim3(256), stream, a);
    };
    if (a.cols <= 64) return go(quant8_rows_kernel<DT, ROUND, 8, 1>, 8);
    if (a.cols <= 256) return go(quant8_rows_kernel<DT, ROUND, 16, 2>, 16);
    if (a.cols <= 1024) return go(quant8_rows_kernel<DT, ROUND, 64, 2>, 64);
    if (a.cols <= 2048) return go(quant8_rows_kernel<DT, ROUND, 64, 4>, 64);
    if (a.cols <= 8192) return go(quant8_rows_kernel<DT, ROUND, 256, 4>, 256);
    if (a.cols <= 16384) return go(quant8_rows_kernel<DT, ROUND, 256, 8>, 256);
    return go(quant8_rows_kernel<DT, ROUND, 256, 0>, 256);
}

template <int DT, int ROUND>
hipError_t launch_quant8_as(const Quant8Args& a, hipStream_t stream) {
    if (!a.col_codes && !a.col_sums) return launch_quant8_rows<DT, ROUND>(a, stream);
    ProfileSpan span;
    const bool tiles = a.col_codes != nullptr, rows = a.row_codes != nullptr;
    const ColumnPlan p = column_plan(a.rows, a.cols);
    const dim3 first(static_cast<unsigned>(p.blocks * p.spans)), block(256);
    hipError_t err;
    if (rows && tiles)
        err = a.col_sums ? launch_kernel(quant8_maxima_kernel<DT, true, true>, first, block, stream, a, p)
                         : launch_kernel(quant8_maxima_kernel<DT, true, false>, first, block, stream, a, p);
    else
        err = a.col_sums ? launch_kernel(quant8_maxima_kernel<DT, false, true>, first, block, stream, a, p)
                         : launch_kernel(quant8_maxima_kernel<DT, false, false>, first, block, stream, a, p);
    if (err != hipSuccess) return err;
    if (!tiles) {                                    // sums, and perhaps rows, which then go by themselves
        if (!rows) span.last();
        err = launch_kernel(quant8_sums_kernel, dim3(static_cast<unsigned>((a.cols + 255) / 256)), block, stream, a, p);
        if (!rows || err != hipSuccess) return err;
        span.last();
        return launch_quant8_rows<DT, ROUND>(a, stream);
    }
    span.last();
    const dim3 second(static_cast<unsigned>(p.tiles_c * p.bands));
    return rows ? launch_kernel(quant8_tiles_kernel<DT, ROUND, true>, second, block, stream, a, p)
                : launch_kernel(quant8_tiles_kernel<DT, ROUND, false>, second, block, stream, a, p);
}

}  // namespace aqsgd
