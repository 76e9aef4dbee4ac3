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
// infinity or a NaN makes the product a NaN, which the conversion takes to 0 (the one that rounds down by itself does not
// do so for every NaN).
template <int ROUND>
__device__ __forceinline__ int32_t code_of(float x, float inv, float r) {
    int32_t k = integer_of(floorf(x * inv + r));
    if constexpr (ROUND == AQSGD_ROUND_STOCHASTIC) k = min(max(k, -127), 127);
    return k;
}

// The low bytes of four codes.
__device__ __forceinline__ uint32_t pack_codes(int32_t a, int32_t b, int32_t c, int32_t d) {
    const uint32_t ab = __builtin_amdgcn_perm(static_cast<uint32_t>(b), static_cast<uint32_t>(a), 0x0c0c0400u);
    const uint32_t cd = __builtin_amdgcn_perm(static_cast<uint32_t>(d), static_cast<uint32_t>(c), 0x04000c0cu);
    return ab | cd;
}

// Rounding offsets of four consecutive columns from a multiple of 4 on; which = 1 for row codes, 2 for column codes.
__device__ __forceinline__ void four_offsets(uint64_t seed, int64_t row, int64_t col, uint32_t which, float* r) {
    uint32_t w[4];
    philox4x32_10(static_cast<uint32_t>(col >> 2) | (which << 30), static_cast<uint32_t>(row), static_cast<uint32_t>(seed),
                  static_cast<uint32_t>(seed >> 32), w);
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = uniform_from_word(w[e]);
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

// A team of lanes side by side, each with eight columns: neighbouring ones, or (APART) two fours half a team's width
// apart, so that a float32 access of the team is contiguous; where codes are stored, eight of them together matter more.
template <bool APART, int LANES>
__device__ __forceinline__ int column_of(int lane, int e) {
    return APART ? (e >> 2) * (4 * LANES) + lane * 4 + (e & 3) : lane * kChunk + e;
}

// Those columns of a row.  `at`: the element in which the team's first column lies, `left`: columns that exist from there
// on (none, where negative).  Loads are not behind a condition, or those of a row's end would wait for each other: past the row's end
// they read its last elements, and mend_columns, once the values are needed, puts right what does not exist or lies
// across the end, in registers.  Rows of fewer than eight columns are left to it altogether.  FULL: all of the team's columns exist.
constexpr int kNarrow = 8;

template <int DT, bool APART, int LANES, bool FULL>
__device__ __forceinline__ Raw<DT> load_columns(const void* x, int64_t at, int lane, int64_t left, int64_t cols) {
    if (!FULL && cols < kNarrow) return zero_raw<DT>();
    Raw<DT> r;
    const auto from = [&](int c, int n) { return FULL ? static_cast<int64_t>(c) : min(static_cast<int64_t>(c), left - n); };
    if constexpr (DT == AQSGD_F32) {
        const float* p = static_cast<const float*>(x) + at;
        r.lo = *reinterpret_cast<const f32x4_any_t*>(p + from(column_of<APART, LANES>(lane, 0), 4));
        r.hi = *reinterpret_cast<const f32x4_any_t*>(p + from(column_of<APART, LANES>(lane, 4), 4));
    } else {
        const uint16_t* p = static_cast<const uint16_t*>(x) + at;
        r.v = *reinterpret_cast<const u32x4_any_t*>(p + from(lane * kChunk, kChunk));
    }
    return r;
}

template <int DT, bool APART, int LANES>
__device__ __forceinline__ void mend_columns(Raw<DT>& r, const void* x, int64_t at, int lane, int64_t left, int64_t cols) {
    if (left >= LANES * kChunk) return;
    if (cols < kNarrow) {
        float f[kChunk];
#pragma unroll
        for (int e = 0; e < kChunk; ++e) {
            const int c = column_of<APART, LANES>(lane, e);
            f[e] = c < left ? load_elem<DT>(x, at + c) : 0.0f;
        }
        r = pack_raw<DT>(f);                        // of what was widened from it: exact
        return;
    }
    // What lies across the end sits at the end of what was loaded: moved down, by as much in every lane.
    if constexpr (DT == AQSGD_F32) {
        const int down = static_cast<int>(-left & 3);
        auto four = [&](f32x4_t& v, int c) {
            f32x4_t m = v;
            if (down & 2) m = f32x4_t{m[2], m[3], 0.0f, 0.0f};
            if (down & 1) m = f32x4_t{m[1], m[2], m[3], 0.0f};
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = c >= left ? 0.0f : c + 4 > left ? m[e] : v[e];
        };
        four(r.lo, column_of<APART, LANES>(lane, 0));
        four(r.hi, column_of<APART, LANES>(lane, 4));
    } else {
        const int down = static_cast<int>(-left & 7), c = lane * kChunk;
        u32x4_t m = r.v;
        if (down & 4) m = u32x4_t{m[2], m[3], 0u, 0u};
        if (down & 2) m = u32x4_t{m[1], m[2], m[3], 0u};
        if (down & 1) m = u32x4_t{m[0] >> 16 | m[1] << 16, m[1] >> 16 | m[2] << 16, m[2] >> 16 | m[3] << 16, m[3] >> 16};
#pragma unroll
        for (int e = 0; e < 4; ++e) r.v[e] = c >= left ? 0u : c + kChunk > left ? m[e] : r.v[e];
    }
}

// Rounding offsets of eight neighbouring columns from a multiple of 4 on.
template <int ROUND>
__device__ __forceinline__ void code_offsets(uint64_t seed, int64_t row, int64_t col, uint32_t which, float (&r)[kChunk]) {
    if constexpr (ROUND == AQSGD_ROUND_STOCHASTIC) {
        four_offsets(seed, row, col, which, r);
        four_offsets(seed, row, col + 4, which, r + 4);
    } else {
#pragma unroll
        for (int e = 0; e < kChunk; ++e) r[e] = 0.5f;
    }
}

// Eight neighbouring codes of a row.  Codes go past the caches, which hold the elements for the second pass: 16384 x
// 4096 float32 both ways 127.5 us, with ordinary stores 138.9.
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void store_row_codes(int8_t* out, const int32_t (&k)[kChunk]) {
    __builtin_nontemporal_store(u32x2_t{pack_codes(k[0], k[1], k[2], k[3]), pack_codes(k[4], k[5], k[6], k[7])}, reinterpret_cast<u32x2_t*>(out));
}

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
            store_row_codes(out + c, k);
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
// First pass: a workgroup takes kSpan columns of a block of rows, 32 lanes of eight columns side by side, sixteen
// rows at a time.
constexpr int kSpan = 256;
constexpr int kTile = 128;                        // columns of the second pass's tiles; rows: 64 or 128

struct ColumnPlan {
    int64_t blocks, block_rows;                   // of the first pass
    int64_t spans;
    int64_t tiles_c, bands, band_tiles;           // of the second: tiles across, workgroups down, tiles of each
    int64_t tile_rows;
};

// The second pass reads every block's maxima again for each of its workgroups, so there are at most 32 blocks of rows
// (more where the columns are few), and a workgroup takes several tiles, one below the other, once there are enough of
// them for the chip.  Tiles of 64 rows where those of 128 would leave CUs without one.
inline ColumnPlan column_plan(int64_t rows, int64_t cols) {
    ColumnPlan p;
    p.spans = (cols + kSpan - 1) / kSpan;
    p.tiles_c = (cols + kTile - 1) / kTile;
    const int64_t tiles = p.tiles_c * ((rows + 127) / 128);
    p.tile_rows = tiles < 512 ? 64 : 128;
    p.band_tiles = tiles < 2048 ? 1 : tiles < 8192 ? tiles / 1024 : 8;
    p.bands = (rows + p.tile_rows * p.band_tiles - 1) / (p.tile_rows * p.band_tiles);
    constexpr int64_t kMost = (int64_t{1} << 23) - 1;                  // workgroups of 512 lanes: a grid takes fewer than 2^32
    const int64_t most = p.spans < 4 ? 128 / p.spans : p.spans > kMost / 32 ? kMost / p.spans : 32;
    const int64_t want = (rows + 31) / 32 < most ? (rows + 31) / 32 : most;
    p.block_rows = (rows + want - 1) / want;
    p.blocks = (rows + p.block_rows - 1) / p.block_rows;
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

constexpr int kSlots = 16;                        // rows a workgroup of the first pass takes at a time

template <int DT, bool ROWS, bool SUMS>
__global__ __launch_bounds__(32 * kSlots) void quant8_maxima_kernel(const Quant8Args a, const ColumnPlan p) {
    constexpr int kAhead = DT == AQSGD_F32 ? 4 : 8;  // rows of a lane that are on their way at a time
    __shared__ uint32_t tops[kSlots][kSpan + 8];
    __shared__ float sums[SUMS ? kSlots : 1][SUMS ? kSpan + 8 : 1];
    const ColumnSpace w = column_space(a.workspace, p, a.cols);
    const int64_t span = blockIdx.x % p.spans, block = blockIdx.x / p.spans;
    const int lane = threadIdx.x & 31, slot = threadIdx.x >> 5;
    const int64_t c0 = span * kSpan, left = a.cols - c0;
    const int64_t r0 = block * p.block_rows, r1 = min(r0 + p.block_rows, a.rows);
    uint32_t top[kChunk] = {};
    float sum[kChunk] = {};
    constexpr bool apart = DT == AQSGD_F32;
    const auto take = [&](int64_t r, auto whole, auto rows) {
        constexpr bool FULL = decltype(whole)::value;
        constexpr int kRows = decltype(rows)::value;
        Raw<DT> raw[kRows];
        const auto at = [&](int i) { return (FULL ? r + kSlots * i : min(r + kSlots * i, r1 - 1)) * a.ld + c0; };      // the last row again: no new maximum
#pragma unroll
        for (int i = 0; i < kRows; ++i) raw[i] = load_columns<DT, apart, 32, FULL>(a.x, at(i), lane, left, a.cols);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if constexpr (!FULL) {
                mend_columns<DT, apart, 32>(raw[i], a.x, at(i), lane, left, a.cols);
                if (SUMS && r + kSlots * i >= r1) raw[i] = zero_raw<DT>();
            }
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
                if (lane == 0 && (FULL || r + kSlots * i < r1)) w.row_tops[span * a.rows + r + kSlots * i] = row_top;
            }
        }
    };
    int64_t r = r0;                                // the workgroup's: what follows depends on no lane
    if (left >= kSpan)
        for (; r + kSlots * kAhead <= r1; r += kSlots * kAhead) take(r + slot, std::true_type(), std::integral_constant<int, kAhead>());
    for (; r < r1; r += kSlots * 2) take(r + slot, std::false_type(), std::integral_constant<int, 2>());
#pragma unroll
    for (int e = 0; e < kChunk; ++e) {
        tops[slot][column_of<apart, 32>(lane, e)] = top[e];
        if constexpr (SUMS) sums[slot][column_of<apart, 32>(lane, e)] = sum[e];
    }
    __syncthreads();
    const int64_t mine = c0 + threadIdx.x;
    if (threadIdx.x >= kSpan || mine >= a.cols) return;
    uint32_t m = 0;
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
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

// Second pass.  A lane takes eight columns of four neighbouring rows, HALVES times: its row codes are whole 8-byte
// pieces of a row, its column codes four rows of a column to a word, and those words meet in LDS.  There a column's
// words lie in pieces of four, moved about by the lane that writes them so that neither side crowds a bank.
template <int HALVES>
__device__ __forceinline__ int turned_at(int col, int piece) {
    return HALVES == 2 ? col * 32 + (piece ^ (col >> 3 & 7)) * 4 : col * 20 + (piece ^ (col >> 4 & 3)) * 4;
}

template <int HALVES> constexpr int kTurned = kTile * (HALVES == 2 ? 32 : 20);       // words

template <int DT, int ROUND, bool ROWS, int HALVES>
__device__ __forceinline__ void tile_codes(const Quant8Args& a, Raw<DT> (&raw)[4 * HALVES], bool full, int64_t r0, int64_t c0,
                                           const float* inv_r, const float* inv_c, uint32_t* turned) {
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int64_t c = c0 + lane * kChunk, left = a.cols - c0;
    float ic[kChunk];
#pragma unroll
    for (int e = 0; e < kChunk; ++e) ic[e] = inv_c[lane * kChunk + e];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        uint32_t word[kChunk];                 // four rows of each column
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = r0 + group * 4 + i + h * 64;
            float f[kChunk], u[kChunk];
            if (!full) {
                mend_columns<DT, false, 16>(raw[4 * h + i], a.x, min(r, a.rows - 1) * a.ld + c0, lane, left, a.cols);
                if (r >= a.rows) raw[4 * h + i] = zero_raw<DT>();
            }
            unpack_raw<DT>(raw[4 * h + i], f);
            if constexpr (ROWS) {
                int32_t k[kChunk];
                const float ir = inv_r[group * 4 + i + h * 64];
                code_offsets<ROUND>(a.seed, r, c, 1, u);
#pragma unroll
                for (int e = 0; e < kChunk; ++e) k[e] = code_of<ROUND>(f[e], ir, u[e]);
                if (r < a.rows && c < a.row_stride) store_row_codes(a.row_codes + r * a.row_stride + c, k);
            }
            code_offsets<ROUND>(a.seed, r, c, 2, u);
#pragma unroll
            for (int e = 0; e < kChunk; ++e) {
                const uint32_t k = static_cast<uint32_t>(code_of<ROUND>(f[e], ic[e], u[e]));
                word[e] = i == 0 ? k & 0xffu
                                 : __builtin_amdgcn_perm(k, word[e], i == 1 ? 0x0c0c0400u : i == 2 ? 0x0c040100u : 0x04020100u);
            }
        }
#pragma unroll
        for (int e = 0; e < kChunk; ++e)
            turned[turned_at<HALVES>(lane * kChunk + e, (group >> 2) + 4 * h) + (group & 3)] = word[e];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2 * HALVES; ++i) {
        const int k = threadIdx.x + 256 * i, col = k / (4 * HALVES), piece = k % (4 * HALVES);
        const int64_t out_c = c0 + col, out_r = r0 + piece * 16;
        if (out_c < a.cols && out_r < a.col_stride)
            __builtin_nontemporal_store(*reinterpret_cast<const u32x4_t*>(&turned[turned_at<HALVES>(col, piece)]),
                                        reinterpret_cast<u32x4_t*>(a.col_codes + out_c * a.col_stride + out_r));
    }
    __syncthreads();
}

// Small matrices of one tile a workgroup (HALVES = 1) ask for its elements before they join the maxima, all at once;
// large ones would pay for that with registers, and with them with waves (float32 16384 x 4096, both passes, 146 us
// against 134).
template <int DT, int ROUND, bool ROWS, int HALVES>
__global__ __launch_bounds__(256) void quant8_tiles_kernel(const Quant8Args a, const ColumnPlan p) {
    constexpr int kRows = 64 * HALVES;
    __shared__ __attribute__((aligned(16))) uint32_t turned[kTurned<HALVES>];
    __shared__ float inv_r[kRows], inv_c[kTile];
    __shared__ uint32_t other[kTile];
    __shared__ float other_sum[kTile];
    const ColumnSpace w = column_space(a.workspace, p, a.cols);
    const int64_t tc = blockIdx.x % p.tiles_c, band = blockIdx.x / p.tiles_c;
    const int64_t c0 = tc * kTile;
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int64_t c = c0 + lane * kChunk, left = a.cols - c0;
    Raw<DT> raw[4 * HALVES];
    uint32_t row_top = 0;
    bool full = true;                              // nothing to mend
    const auto row_of = [&](int64_t r0, int i) { return r0 + group * 4 + (i & 3) + (i >> 2) * 64; };
    auto fetch = [&](int64_t r0) {
        if constexpr (HALVES == 2) {
#pragma unroll
            for (int i = 0; i < 4 * HALVES; ++i)
                raw[i] = row_of(r0, i) < a.rows ? load_some<DT>(element_at<DT>(a.x, row_of(r0, i) * a.ld + min(c, a.cols)), left - lane * kChunk)
                                                : zero_raw<DT>();
        } else if (left >= kTile && r0 + kRows <= a.rows) {
#pragma unroll
            for (int i = 0; i < 4 * HALVES; ++i)
                raw[i] = load_columns<DT, false, 16, true>(a.x, row_of(r0, i) * a.ld + c0, lane, left, a.cols);
        } else {
            full = false;
#pragma unroll
            for (int i = 0; i < 4 * HALVES; ++i)
                raw[i] = load_columns<DT, false, 16, false>(a.x, min(row_of(r0, i), a.rows - 1) * a.ld + c0, lane, left, a.cols);
        }
        if constexpr (ROWS) {
            row_top = 0;
            if (threadIdx.x < kRows) {
                const int64_t r = min(r0 + threadIdx.x, a.rows - 1);
#pragma unroll 8
                for (int64_t s = 0; s < p.spans; ++s) row_top = max(row_top, w.row_tops[s * a.rows + r]);
            }
        }
    };
    const int64_t first = band * p.band_tiles * kRows, end = min(first + p.band_tiles * kRows, a.rows);
    if (HALVES == 1) fetch(first);
    {
        // each column's maxima (and sums) by two threads
        const bool sums = a.col_sums && band == 0;
        const int64_t mine = min(c0 + (threadIdx.x & 127), a.cols - 1);
        uint32_t top = 0;
        float sum = 0.0f;
#pragma unroll 8
        for (int64_t b = threadIdx.x >> 7; b < p.blocks; b += 2) top = max(top, w.col_tops[b * a.cols + mine]);
        if (sums) {
#pragma unroll 8
            for (int64_t b = threadIdx.x >> 7; b < p.blocks; b += 2) sum += w.col_sums[b * a.cols + mine];
        }
        if (threadIdx.x >= 128) {
            other[threadIdx.x & 127] = top;
            other_sum[threadIdx.x & 127] = sum;
        }
        __syncthreads();
        if (threadIdx.x < 128) {
            const CodeScale s = code_scale(max(top, other[threadIdx.x]));
            inv_c[threadIdx.x] = s.inv;
            if (band == 0 && c0 + threadIdx.x < a.cols) {
                a.col_scales[mine] = s.scale;
                if (sums) a.col_sums[mine] = sum + other_sum[threadIdx.x];
            }
        }
    }
    for (int64_t r0 = first; r0 < end; r0 += kRows) {
        if (HALVES == 2 || r0 > first) fetch(r0);
        if constexpr (ROWS) {
            if (threadIdx.x < kRows) {
                const CodeScale s = code_scale(row_top);
                inv_r[threadIdx.x] = s.inv;
                if (tc == 0 && r0 + threadIdx.x < a.rows) a.row_scales[r0 + threadIdx.x] = s.scale;
            }
        }
        __syncthreads();
        tile_codes<DT, ROUND, ROWS, HALVES>(a, raw, full, r0, c0, inv_r, inv_c, turned);
    }
}

// Matrices of up to 64 HALVES rows: a workgroup sees whole columns and needs no first pass; rows, where they are wanted
// too, are the business of the workgroups behind, one for each.  One launch where the two passes take two (16 x 189
// float16 both ways 7.8 us, so 4.0).
template <int DT, int ROUND, int HALVES>
__global__ __launch_bounds__(256) void quant8_short_kernel(const Quant8Args a, uint32_t tiles_c) {
    __shared__ __attribute__((aligned(16))) uint32_t turned[kTurned<HALVES>];
    __shared__ uint32_t tops[16][kTile + 4];
    __shared__ float sums[16][kTile + 4];
    __shared__ float inv_c[kTile];
    if (blockIdx.x >= tiles_c) {
        const int64_t row = blockIdx.x - tiles_c, base = row * a.ld;
        uint32_t top = 0;
        for (int64_t c = static_cast<int64_t>(threadIdx.x) * kChunk; c < a.cols; c += 256 * kChunk) {
            float f[kChunk];
            unpack_raw<DT>(load_some<DT>(element_at<DT>(a.x, base + c), a.cols - c), f);
#pragma unroll
            for (int e = 0; e < kChunk; ++e) top = max(top, magnitude_bits(f[e]));
        }
        top = __float_as_uint(team_max<64>(__uint_as_float(top)));
        if ((threadIdx.x & 63) == 0) tops[0][threadIdx.x >> 6] = top;
        __syncthreads();
        const CodeScale s = code_scale(max(max(tops[0][0], tops[0][1]), max(tops[0][2], tops[0][3])));
        if (threadIdx.x == 0) a.row_scales[row] = s.scale;
        for (int64_t c = static_cast<int64_t>(threadIdx.x) * kChunk; c < a.row_stride; c += 256 * kChunk) {
            float f[kChunk], u[kChunk];
            unpack_raw<DT>(load_some<DT>(element_at<DT>(a.x, base + min(c, a.cols)), a.cols - c), f);
            code_offsets<ROUND>(a.seed, row, c, 1, u);
            int32_t k[kChunk];
#pragma unroll
            for (int e = 0; e < kChunk; ++e) k[e] = code_of<ROUND>(f[e], s.inv, u[e]);
            store_row_codes(a.row_codes + row * a.row_stride + c, k);
        }
        return;
    }
    const int64_t c0 = static_cast<int64_t>(blockIdx.x) * kTile, left = a.cols - c0;
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    Raw<DT> raw[4 * HALVES];
    const auto row_of = [&](int i) { return static_cast<int64_t>(group * 4 + (i & 3) + (i >> 2) * 64); };
#pragma unroll
    for (int i = 0; i < 4 * HALVES; ++i) raw[i] = load_columns<DT, false, 16, false>(a.x, min(row_of(i), a.rows - 1) * a.ld + c0, lane, left, a.cols);
    uint32_t top[kChunk] = {};
    float sum[kChunk] = {};
#pragma unroll
    for (int i = 0; i < 4 * HALVES; ++i) {
        mend_columns<DT, false, 16>(raw[i], a.x, min(row_of(i), a.rows - 1) * a.ld + c0, lane, left, a.cols);
        if (row_of(i) >= a.rows) raw[i] = zero_raw<DT>();
        float f[kChunk];
        unpack_raw<DT>(raw[i], f);
#pragma unroll
        for (int e = 0; e < kChunk; ++e) {
            top[e] = max(top[e], magnitude_bits(f[e]));
            sum[e] += f[e];
        }
    }
#pragma unroll
    for (int e = 0; e < kChunk; ++e) {
        tops[group][lane * kChunk + e] = top[e];
        sums[group][lane * kChunk + e] = sum[e];
    }
    __syncthreads();
    if (threadIdx.x < kTile) {
        uint32_t t = 0;
        float s = 0.0f;
#pragma unroll
        for (int g = 0; g < 16; ++g) {
            t = max(t, tops[g][threadIdx.x]);
            s += sums[g][threadIdx.x];
        }
        const CodeScale k = code_scale(t);
        inv_c[threadIdx.x] = k.inv;
        if (static_cast<int64_t>(threadIdx.x) < left) {
            a.col_scales[c0 + threadIdx.x] = k.scale;
            if (a.col_sums) a.col_sums[c0 + threadIdx.x] = s;
        }
    }
    __syncthreads();
    tile_codes<DT, ROUND, false, HALVES>(a, raw, true, 0, c0, inv_c, inv_c, turned);
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
    if (a.col_codes && a.rows <= 128) {
        const uint32_t tiles_c = static_cast<uint32_t>((a.cols + kTile - 1) / kTile);
        const dim3 grid(tiles_c + (a.row_codes ? static_cast<unsigned>(a.rows) : 0u));
        return a.rows <= 64 ? launch_kernel(quant8_short_kernel<DT, ROUND, 1>, grid, dim3(256), stream, a, tiles_c)
                            : launch_kernel(quant8_short_kernel<DT, ROUND, 2>, grid, dim3(256), stream, a, tiles_c);
    }
    ProfileSpan span;
    const bool tiles = a.col_codes != nullptr, rows = a.row_codes != nullptr;
    const ColumnPlan p = column_plan(a.rows, a.cols);
    const dim3 first(static_cast<unsigned>(p.blocks * p.spans)), first_block(32 * kSlots), block(256);
    hipError_t err;
    if (rows && tiles)
        err = a.col_sums ? launch_kernel(quant8_maxima_kernel<DT, true, true>, first, first_block, stream, a, p)
                         : launch_kernel(quant8_maxima_kernel<DT, true, false>, first, first_block, stream, a, p);
    else
        err = a.col_sums ? launch_kernel(quant8_maxima_kernel<DT, false, true>, first, first_block, stream, a, p)
                         : launch_kernel(quant8_maxima_kernel<DT, false, false>, first, first_block, stream, a, p);
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
    if (p.tile_rows == 64)
        return rows ? launch_kernel(quant8_tiles_kernel<DT, ROUND, true, 1>, second, block, stream, a, p)
                    : launch_kernel(quant8_tiles_kernel<DT, ROUND, false, 1>, second, block, stream, a, p);
    return rows ? launch_kernel(quant8_tiles_kernel<DT, ROUND, true, 2>, second, block, stream, a, p)
                : launch_kernel(quant8_tiles_kernel<DT, ROUND, false, 2>, second, block, stream, a, p);
}

}  // namespace aqsgd
