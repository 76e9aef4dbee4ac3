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


// What is left of the sums once they lie in LDS as rows of 32-bit integers: a lane takes four columns of every
// few rows, so that its scales and bias are read once and a row leaves in whole lines.
//   sums  LDS, [rows, pitch] of the wave's (or workgroup's) columns from virtual column n0 on
template <int KIND, int DT, int COLS>
struct Finish {
    static constexpr int wide = (KIND == kGated ? COLS / 2 : COLS) / 4;       // lanes to a row
    static constexpr int step_rows = kWave / wide;                            // rows a wave takes at a time
    static_assert(wide >= 1 && wide <= kWave && kWave % wide == 0, "a wave takes whole rows");
    const ProductArgs& p;
    int32_t n, left, half;       // first column (of h, where gated), columns that remain from there
    int place;                   // of the lane's first sum in a row
    f32x4_t step, bias, extra, step_u, bias_u;

    __device__ __forceinline__ f32x4_t steps(int32_t c) const {
        f32x4_t v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = p.b_scales[c + (e < left ? e : 0)] / kCodeHalf;
        return v;
    }
    __device__ __forceinline__ f32x4_t biases(int32_t c) const {
        f32x4_t v = {0, 0, 0, 0};
        if (p.bias) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = load_elem<DT>(p.bias, c + (e < left ? e : 0));
        }
        return v;
    }
    // ones: sums of the columns' codes of b (message)
    __device__ __forceinline__ Finish(const ProductArgs& args, int32_t n0, int lane, const int32_t* ones) : p(args) {
        const int c = (lane % wide) * 4;
        half = p.n >> 1;
        if constexpr (KIND == kGated) {
            n = (n0 >> 1) + c;
            left = half - n;
            place = ((c >> 4) << 5) + (c & 15);
        } else {
            n = n0 + c;
            left = p.n - n;
            place = c;
        }
        const int32_t at = left > 0 ? n : 0;
        step = steps(at);
        bias = biases(at);
        if constexpr (KIND == kGated) {
            step_u = steps(half + at);
            bias_u = biases(half + at);
        }
        if constexpr (KIND == kMessage) {
#pragma unroll
            for (int e = 0; e < 4; ++e) extra[e] = 0.5f * static_cast<float>(ones[place + e]);      // levels - 127.5
        }
    }
    __device__ __forceinline__ f32x4_t scaled(const i32x4_t& sum, float a_step, const f32x4_t& st, const f32x4_t& bi) const {
        f32x4_t v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = static_cast<float>(sum[e]);
            if constexpr (KIND == kMessage) x += extra[e];
            v[e] = x * a_step * st[e];
            if (p.bias) v[e] += bi[e];
        }
        return v;
    }
    __device__ __forceinline__ void put(void* base, int64_t at, const f32x4_t& v) const {
        if (left >= 4) {
            store4(DT, base, at, v);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < left) store_elem<DT>(base, at + e, v[e]);
        }
    }
    __device__ __forceinline__ void row(int32_t m, const int32_t* sums) const {
        if (m >= p.m || left <= 0) return;
        const float a_step = p.a_scales[m] / (KIND == kMessage ? kLevelHalf : kCodeHalf);
        f32x4_t v = scaled(*reinterpret_cast<const i32x4_t*>(sums + place), a_step, step, bias);
        if constexpr (KIND == kGated) {
            const f32x4_t u = scaled(*reinterpret_cast<const i32x4_t*>(sums + place + 16), a_step, step_u, bias_u);
            f32x4_t h;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = activation(p.act, v[e]) * u[e];
            put(p.out, static_cast<int64_t>(m) * half + n, h);
            if (p.pre) {
                put(p.pre, static_cast<int64_t>(m) * p.n + n, v);
                put(p.pre, static_cast<int64_t>(m) * p.n + half + n, u);
            }
        } else {
            const int64_t at = static_cast<int64_t>(m) * p.n + n;
            if constexpr (KIND == kActivation) {
                if (p.pre) put(p.pre, at, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = activation(p.act, v[e]);
            } else if (p.add) {
                if (left >= 4) {
                    v += load4(DT, p.add, at);
                } else {
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (e < left) v[e] += load_elem<DT>(p.add, at + e);
                }
            }
            put(p.out, at, v);
        }
    }
};

// A wave's TM x TN blocks of sums (lane l holds row l % 16 of a block and four columns from (l / 16) * 4 on), from
// row m0 and virtual column n0 on.  `own`: LDS of the wave's own, store_bytes() of it.
constexpr int kStoreBlocks = 2;                  // blocks of 16 rows that go through LDS at a time
constexpr int store_pitch(int tn) { return tn * 16 + 4; }
constexpr int store_bytes(int tn) { return (kStoreBlocks * 16 * store_pitch(tn) + 16 * tn) * 4; }

template <int KIND, int DT, int TM, int TN>
__device__ __forceinline__ void store_tile(const ProductArgs& p, const i32x4_t (&acc)[TM][TN], const int32_t (&ones)[TN], int32_t m0,
                                           int32_t n0, int lane, int32_t* own) {
    constexpr int pitch = store_pitch(TN);
    int32_t* sums_of_b = own + kStoreBlocks * 16 * pitch;
    if constexpr (KIND == kMessage) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            int32_t v = ones[j];
            v += __shfl_xor(v, 16, kWave);
            v += __shfl_xor(v, 32, kWave);
            if (lane < 16) sums_of_b[16 * j + lane] = v;
        }
    }
    using F = Finish<KIND, DT, TN * 16>;
    const F finish(p, n0, lane, sums_of_b);
    int32_t* to = own + (lane & 15) * pitch + (lane >> 4) * 4;
#pragma unroll
    for (int i0 = 0; i0 < TM; i0 += kStoreBlocks) {
#pragma unroll
        for (int i = 0; i < kStoreBlocks; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) *reinterpret_cast<i32x4_t*>(to + i * 16 * pitch + 16 * j) = acc[i0 + i][j];
        for (int r = lane / F::wide; r < kStoreBlocks * 16; r += F::step_rows) finish.row(m0 + i0 * 16 + r, own + r * pitch);
    }
}

// ---- large tiles ------------------------------------------------------------------------------
// TM x TN blocks of 16 x 16 sums to a wave, WM x WN waves to a workgroup, k in steps of 128 bytes.
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef const __attribute__((address_space(1))) void* global_ptr;

template <int TM, int TN, int WM, int WN>
struct TileShape {
    static constexpr int bm = 16 * TM * WM, bn = 16 * TN * WN, waves = WM * WN;
    static constexpr int row = 128;                               // bytes of k in a step
    static constexpr int stage = (bm + bn) * row;                 // bytes of a step's operands
    static constexpr int loads_a = bm / 8 / waves, loads_b = bn / 8 / waves;      // 1 KB each, per wave
};

// Tile of workgroup b: the eight XCDs take the workgroups in turn, so that b mod 8 is the XCD; each gets a
// contiguous run of the tiles, which go down in bands of kBand tile rows, so that the tiles an XCD works on
// at a time share rows of a and of b in its L2.
constexpr int kBand = 4;
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t total, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn) {
    const uint32_t q = total >> 3, r = total & 7, x = b & 7;
    const uint32_t t = x * q + min(x, r) + (b >> 3);
    const uint32_t band = t / (kBand * tiles_n), in = t - band * kBand * tiles_n;
    const uint32_t rows = min(static_cast<uint32_t>(kBand), tiles_m - band * kBand);
    tm = band * kBand + in % rows;
    tn = in / rows;
}

template <int KIND, int DT, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 1) void product_tile_kernel(const ProductArgs p, uint32_t tiles_m, uint32_t tiles_n) {
    using S = TileShape<TM, TN, WM, WN>;
    __shared__ __attribute__((aligned(128))) uint8_t lds[2 * S::stage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave / WN) * TM * 16, wn = (wave % WN) * TN * 16;
    uint32_t tm, tn;
    tile_of(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, tm, tn);
    const int32_t m0 = static_cast<int32_t>(tm) * S::bm, n0 = static_cast<int32_t>(tn) * S::bn;

    // A wave's load brings 8 rows of 128 bytes to 1 KB of LDS, lane l the 16 bytes at l * 16 there.  Piece c of
    // row r lies at place c ^ (r & 7), so that the 16 rows of a fragment spread over all banks.
    const uint8_t* base_a = p.a + static_cast<int64_t>(m0) * p.lda;
    const int32_t half = p.n >> 1;
    const int8_t* base_b = p.b + static_cast<int64_t>(KIND == kGated ? n0 >> 1 : n0) * p.ldb;
    const int8_t* base_u = KIND == kGated ? base_b + static_cast<int64_t>(half) * p.ldb : base_b;
    const int lr = lane >> 3, piece = ((lane & 7) ^ lr) * 16;
    uint32_t off_a[S::loads_a], off_b[S::loads_b];
#pragma unroll
    for (int i = 0; i < S::loads_a; ++i)
        off_a[i] = static_cast<uint32_t>(min((wave * S::loads_a + i) * 8 + lr, p.m - 1 - m0)) * static_cast<uint32_t>(p.lda);
#pragma unroll
    for (int i = 0; i < S::loads_b; ++i) {
        const int r = (wave * S::loads_b + i) * 8 + lr;
        if constexpr (KIND == kGated)
            off_b[i] = static_cast<uint32_t>(min(((r >> 5) << 4) + (r & 15), half - 1 - (n0 >> 1))) * static_cast<uint32_t>(p.ldb);
        else
            off_b[i] = static_cast<uint32_t>(min(r, p.n - 1 - n0)) * static_cast<uint32_t>(p.ldb);
    }
    const int32_t halves = (p.k + 63) / 64, steps = (halves + 1) / 2;
    const int32_t last_a = (KIND == kMessage ? p.k : halves * 64) - 16, last_b = halves * 64 - 16;
    auto bring = [&](int32_t step, int buf) {
        const int32_t k = step * S::row + piece;
        const uint32_t ka = min(k, last_a), kb = min(k, last_b);
        uint8_t* to = lds + buf * S::stage;
#pragma unroll
        for (int i = 0; i < S::loads_a; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(base_a + (off_a[i] + ka)), (lds_ptr)(to + (wave * S::loads_a + i) * 1024), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < S::loads_b; ++i) {
            const int8_t* b = KIND == kGated && (((wave * S::loads_b + i) * 8) & 16) ? base_u : base_b;
            __builtin_amdgcn_global_load_lds((global_ptr)(b + (off_b[i] + kb)), (lds_ptr)(to + S::bm * S::row + (wave * S::loads_b + i) * 1024), 16, 0, 0);
        }
    };
    // Fragments: lane l holds 16 bytes of row l % 16, piece (l / 16) of the half step.
    const int fr = lane & 15, fq = lane >> 4;
    const int at0 = fr * S::row + ((fq ^ (fr & 7)) * 16), at1 = at0 ^ 64;
    auto read_frags = [&](i32x4_t (&fa)[TM], i32x4_t (&fb)[TN], int buf, int h) {
        const uint8_t* from = lds + buf * S::stage + (h ? at1 : at0);
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[i] = *reinterpret_cast<const i32x4_t*>(from + (wm + 16 * i) * S::row);
#pragma unroll
        for (int j = 0; j < TN; ++j) fb[j] = *reinterpret_cast<const i32x4_t*>(from + (S::bm + wn + 16 * j) * S::row);
    };
    i32x4_t acc[TM][TN] = {};
    int32_t ones[TN] = {};
    auto multiply = [&](i32x4_t (&fa)[TM], i32x4_t (&fb)[TN]) {
        if constexpr (KIND == kMessage) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) fa[i][e] ^= static_cast<int32_t>(0x80808080u);      // level - 128
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) ones[j] = __builtin_amdgcn_sdot4(fb[j][e], 0x01010101, ones[j], false);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    };
    i32x4_t fa0[TM], fb0[TN], fa1[TM], fb1[TN];
    if (steps > 0) {
        bring(0, 0);
        __syncthreads();
        if (steps > 1) bring(1, 1);
        read_frags(fa0, fb0, 0, 0);
    }
    for (int32_t s = 0; s < steps; ++s) {
        const int buf = s & 1;
        read_frags(fa1, fb1, buf, 1);
        multiply(fa0, fb0);
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();                     // step s + 1 has arrived; no wave reads step s any more
        if (s + 2 < steps) bring(s + 2, buf);
        if (s + 1 < steps) read_frags(fa0, fb0, buf ^ 1, 0);
        if (2 * s + 1 < halves) multiply(fa1, fb1);
    }
    static_assert(store_bytes(TN) * S::waves <= 2 * S::stage && TM % kStoreBlocks == 0, "the stages' LDS serves the results");
    __syncthreads();                         // the last fragments have been read
    store_tile<KIND, DT, TM, TN>(p, acc, ones, m0 + wm, n0 + wn, lane, reinterpret_cast<int32_t*>(lds + wave * store_bytes(TN)));
}

template <int DT, int TM, int TN, int WM, int WN>
hipError_t launch_tiles_as(ProductKind kind, const ProductArgs& p, hipStream_t stream) {
    using S = TileShape<TM, TN, WM, WN>;
    const uint32_t tm = (static_cast<uint32_t>(p.m) + S::bm - 1) / S::bm, tn = (static_cast<uint32_t>(p.n) + S::bn - 1) / S::bn;
    const dim3 grid(tm * tn), block(64 * S::waves);
    switch (kind) {
    case kPlain:      return launch_kernel(product_tile_kernel<kPlain, DT, TM, TN, WM, WN>, grid, block, stream, p, tm, tn);
    case kMessage:    return launch_kernel(product_tile_kernel<kMessage, DT, TM, TN, WM, WN>, grid, block, stream, p, tm, tn);
    case kActivation: return launch_kernel(product_tile_kernel<kActivation, DT, TM, TN, WM, WN>, grid, block, stream, p, tm, tn);
    default:          return launch_kernel(product_tile_kernel<kGated, DT, TM, TN, WM, WN>, grid, block, stream, p, tm, tn);
    }
}

enum ProductTile { kTile256 = 0, kTile128 };

template <int DT>
hipError_t launch_product_dt(ProductTile tile, ProductKind kind, const ProductArgs& p, hipStream_t stream) {
    switch (tile) {
    case kTile256: return launch_tiles_as<DT, 8, 4, 2, 4>(kind, p, stream);
    default:       return launch_tiles_as<DT, 4, 4, 2, 2>(kind, p, stream);
    }
}

}  // namespace aqsgd
