// Kernels of aqsgd_matmul8 and aqsgd_ffn8: products of 8-bit codes on the matrix units, exact in 32-bit
// integers, with the scales, the bias and the activation applied to the sums before they are stored.
#pragma once

#include "aqsgd_products8.h"

namespace aqsgd {

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));

// Where column c of a tile whose columns start at n0 has its row of b, in rows from the tile's first (of the gate's
// half, where gated).  In the gated product the columns alternate in sixteens between the gate's rows and those it
// is multiplied with, n / 2 further on, so that one lane ends up with both sums of an element.  Columns past the
// last one read the last one's row.
template <int KIND>
__device__ __forceinline__ uint32_t row_from(int32_t n0, int32_t c, int32_t n) {
    if constexpr (KIND == kGated) return static_cast<uint32_t>(min(((c >> 5) << 4) + (c & 15), (n >> 1) - 1 - (n0 >> 1)));
    else return static_cast<uint32_t>(min(c, n - 1 - n0));
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
    __device__ __forceinline__ Finish(const ProductArgs& args, int32_t n0, int lane) : p(args) {
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
    }
    // A message's levels stand for level - 127.5; the sums are over level - 128, so half the sum of b's codes is
    // missing.  ones: those sums, `parts` of them `pitch` apart.
    __device__ __forceinline__ void take_ones(const int32_t* ones, int parts, int pitch) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            int32_t s = 0;
            for (int k = 0; k < parts; ++k) s += ones[k * pitch + place + e];
            extra[e] = 0.5f * static_cast<float>(s);
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
    template <bool FULL>
    __device__ __forceinline__ void put(void* base, int64_t at, const f32x4_t& v) const {
        if (FULL || left >= 4) {
            store4(DT, base, at, v);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < left) store_elem<DT>(base, at + e, v[e]);
        }
    }
    // A row's columns: its sums in LDS, in PARTS parts `pitch` apart.
    template <int PARTS>
    __device__ __forceinline__ i32x4_t sum_of(const int32_t* sums, int pitch) const {
        i32x4_t s = *reinterpret_cast<const i32x4_t*>(sums);
#pragma unroll
        for (int k = 1; k < PARTS; ++k) s += *reinterpret_cast<const i32x4_t*>(sums + k * pitch);
        return s;
    }
    static __device__ __forceinline__ float step_of_a(float scale) { return scale / (KIND == kMessage ? kLevelHalf : kCodeHalf); }
    // What is there already in a row's columns (the plain product with something to add to).
    template <bool FULL>
    __device__ __forceinline__ f32x4_t added(int32_t m) const {
        f32x4_t v = {0, 0, 0, 0};
        if constexpr (KIND == kPlain || KIND == kMessage) {
            if (p.add && (FULL || (m < p.m && left > 0))) {
                const int64_t at = static_cast<int64_t>(m) * p.n + n;
                if (FULL || left >= 4) {
                    v = load4(DT, p.add, at);
                } else {
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (e < left) v[e] = load_elem<DT>(p.add, at + e);
                }
            }
        }
        return v;
    }
    // FULL: the row and the four columns exist.
    template <bool FULL, int PARTS = 1>
    __device__ __forceinline__ void row(int32_t m, float a_step, const f32x4_t& there, const int32_t* sums, int pitch = 0) const {
        if (!FULL && (m >= p.m || left <= 0)) return;
        f32x4_t v = scaled(sum_of<PARTS>(sums + place, pitch), a_step, step, bias);
        if constexpr (KIND == kGated) {
            const f32x4_t u = scaled(sum_of<PARTS>(sums + place + 16, pitch), a_step, step_u, bias_u);
            f32x4_t h;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = activation(p.act, v[e]) * u[e];
            put<FULL>(p.out, static_cast<int64_t>(m) * half + n, h);
            if (p.pre) {
                put<FULL>(p.pre, static_cast<int64_t>(m) * p.n + n, v);
                put<FULL>(p.pre, static_cast<int64_t>(m) * p.n + half + n, u);
            }
        } else {
            const int64_t at = static_cast<int64_t>(m) * p.n + n;
            if constexpr (KIND == kActivation) {
                if (p.pre) put<FULL>(p.pre, at, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = activation(p.act, v[e]);
            } else if (p.add) {
                v += there;
            }
            put<FULL>(p.out, at, v);
        }
    }
};

// A wave's TM x TN blocks of sums (lane l holds row l % 16 of a block and four columns from (l / 16) * 4 on), from
// row m0 and virtual column n0 on.  `own`: LDS of the wave's own, store_bytes() of it.
constexpr int kStoreBlocks = 2;                  // blocks of 16 rows that go through LDS at a time
constexpr int store_pitch(int tn) { return tn * 16 + 4; }
constexpr int store_bytes(int tm, int tn) { return (kStoreBlocks * 16 * store_pitch(tn) + 16 * tn + 16 * tm) * 4; }

template <int KIND, int DT, int TM, int TN>
__device__ __forceinline__ void store_tile(const ProductArgs& p, const i32x4_t (&acc)[TM][TN], const int32_t (&ones)[TN], int32_t m0,
                                           int32_t n0, int lane, int32_t* own) {
    constexpr int pitch = store_pitch(TN);
    int32_t* sums_of_b = own + kStoreBlocks * 16 * pitch;
    float* steps_of_a = reinterpret_cast<float*>(sums_of_b + 16 * TN);
    using F = Finish<KIND, DT, TN * 16>;
#pragma unroll
    for (int i = 0; i < (16 * TM + 63) / 64; ++i) {
        const int r = 64 * i + lane;
        const float a_step = F::step_of_a(p.a_scales[min(m0 + r, p.m - 1)]);
        if (r < 16 * TM) steps_of_a[r] = a_step;
    }
    if constexpr (KIND == kMessage) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            int32_t v = ones[j];
            v += __shfl_xor(v, 16, kWave);
            v += __shfl_xor(v, 32, kWave);
            if (lane < 16) sums_of_b[16 * j + lane] = v;
        }
    }
    F finish(p, n0, lane);
    if constexpr (KIND == kMessage) finish.take_ones(sums_of_b, 1, 0);
    int32_t* to = own + (lane & 15) * pitch + (lane >> 4) * 4;
    constexpr int turns = kStoreBlocks * 16 / F::step_rows, ahead = turns < 4 ? turns : 4;
    const bool full = m0 + 16 * TM <= p.m && n0 + 16 * TN <= (KIND == kGated ? p.n & ~31 : p.n);     // h is whole sixteens there
    const int mine = lane / F::wide;
#pragma unroll
    for (int i0 = 0; i0 < TM; i0 += kStoreBlocks) {
#pragma unroll
        for (int i = 0; i < kStoreBlocks; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) *reinterpret_cast<i32x4_t*>(to + i * 16 * pitch + 16 * j) = acc[i0 + i][j];
        const int32_t first = m0 + i0 * 16 + mine;
        if (full) {
#pragma unroll 1
            for (int t = 0; t < turns; t += ahead) {
                f32x4_t there[ahead];
#pragma unroll
                for (int u = 0; u < ahead; ++u) there[u] = finish.template added<true>(first + (t + u) * F::step_rows);
#pragma unroll
                for (int u = 0; u < ahead; ++u) {
                    const int r = mine + (t + u) * F::step_rows;
                    finish.template row<true>(first + (t + u) * F::step_rows, steps_of_a[i0 * 16 + r], there[u], own + r * pitch);
                }
            }
        } else {
#pragma unroll 1
            for (int t = 0; t < turns; ++t) {
                const int r = mine + t * F::step_rows;
                const int32_t m = first + t * F::step_rows;
                finish.template row<false>(m, steps_of_a[i0 * 16 + r], finish.template added<false>(m), own + r * pitch);
            }
        }
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
        off_b[i] = row_from<KIND>(n0, r, p.n) * static_cast<uint32_t>(p.ldb);
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
        bring(min(1, steps - 1), 1);
        read_frags(fa0, fb0, 0, 0);
        for (int32_t s = 0; s < steps - 1; ++s) {
            const int buf = s & 1;
            read_frags(fa1, fb1, buf, 1);
            multiply(fa0, fb0);
            __builtin_amdgcn_sched_barrier(0);
            __syncthreads();                             // step s + 1 has arrived; no wave reads step s any more
            bring(min(s + 2, steps - 1), buf);           // the last one once more: nobody reads it
            read_frags(fa0, fb0, buf ^ 1, 0);
            multiply(fa1, fb1);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (halves % 2 == 0) read_frags(fa1, fb1, (steps - 1) & 1, 1);
        multiply(fa0, fb0);
        if (halves % 2 == 0) multiply(fa1, fb1);
    }
    static_assert(store_bytes(TM, TN) * S::waves <= 2 * S::stage && TM % kStoreBlocks == 0, "the stages' LDS serves the results");
    __syncthreads();                         // the last fragments have been read
    store_tile<KIND, DT, TM, TN>(p, acc, ones, m0 + wm, n0 + wn, lane, reinterpret_cast<int32_t*>(lds + wave * store_bytes(TM, TN)));
}

// ---- small products ---------------------------------------------------------------------------
// 16 R x 16 J sums to a workgroup, its W waves sharing out k in pieces of 128 bytes: nothing is staged, every wave
// loads the fragments of its pieces from memory into registers, the next ones while it multiplies, and the waves'
// sums meet in LDS once, at the end.
template <int R, int J> struct SplitShape {
    static constexpr int pieces = R + J >= 4 ? 1 : R + J == 3 ? 2 : 3;        // on their way at a time: registers
    static constexpr int pitch = 16 * J + 4;
};

template <int KIND, int DT, int R, int J, int W>
__global__ __launch_bounds__(64 * W) void product_split_kernel(const ProductArgs p, uint32_t tiles_n) {
    using S = SplitShape<R, J>;
    constexpr int P = S::pieces, slab = 16 * R * S::pitch;
    __shared__ __attribute__((aligned(16))) int32_t sums[W * slab];
    __shared__ int32_t ones_of[KIND == kMessage ? W * 16 * J : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t m0 = static_cast<int32_t>(blockIdx.x / tiles_n) * (16 * R), n0 = static_cast<int32_t>(blockIdx.x % tiles_n) * (16 * J);
    const int fr = lane & 15, fq = lane >> 4;
    // rows by their distance from the tile's first, in bytes: below 64 * 131072
    const int32_t half = p.n >> 1;
    const uint8_t* base_a = p.a + static_cast<int64_t>(m0) * p.lda;
    const int8_t* base_b = p.b + static_cast<int64_t>(KIND == kGated ? n0 >> 1 : n0) * p.ldb;
    const int8_t* base_u = KIND == kGated ? base_b + static_cast<int64_t>(half) * p.ldb : base_b;
    uint32_t off_a[R], off_b[J];
#pragma unroll
    for (int i = 0; i < R; ++i) off_a[i] = static_cast<uint32_t>(min(16 * i + fr, p.m - 1 - m0)) * static_cast<uint32_t>(p.lda);
#pragma unroll
    for (int j = 0; j < J; ++j) off_b[j] = row_from<KIND>(n0, 16 * j + fr, p.n) * static_cast<uint32_t>(p.ldb);
    const int32_t halves = (p.k + 63) / 64, whole = (halves + 1) / 2;
    const int32_t last_a = (KIND == kMessage ? p.k : halves * 64) - 16;
    struct Frags { i32x4_t a[P][2][R], b[P][2][J]; };
    auto load = [&](Frags& f, int32_t first) {
#pragma unroll
        for (int u = 0; u < P; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int32_t step = 2 * (first + u * W) + h, k = step * 64 + fq * 16;
                if (step < halves) {
#pragma unroll
                    for (int j = 0; j < J; ++j) 
                        f.b[u][h][j] = *reinterpret_cast<const i32x4_t*>((KIND == kGated && (j & 1) ? base_u : base_b) + (off_b[j] + static_cast<uint32_t>(k)));
#pragma unroll
                    for (int i = 0; i < R; ++i) 
                        f.a[u][h][i] = *reinterpret_cast<const i32x4_t*>(base_a + (off_a[i] + static_cast<uint32_t>(min(k, last_a))));
                } else {
#pragma unroll
                    for (int j = 0; j < J; ++j) f.b[u][h][j] = i32x4_t{0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < R; ++i) f.a[u][h][i] = i32x4_t{0, 0, 0, 0};
                }
            }
    };
    i32x4_t acc[R][J] = {};
    int32_t ones[J] = {};
    auto multiply = [&](Frags& f) {
#pragma unroll
        for (int u = 0; u < P; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (KIND == kMessage) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
#pragma unroll
                        for (int i = 0; i < R; ++i) f.a[u][h][i][e] ^= static_cast<int32_t>(0x80808080u);       // level - 128
#pragma unroll
                        for (int j = 0; j < J; ++j) ones[j] = __builtin_amdgcn_sdot4(f.b[u][h][j][e], 0x01010101, ones[j], false);
                    }
                }
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int j = 0; j < J; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.b[u][h][j], f.a[u][h][i], acc[i][j], 0, 0, 0);
            }
    };
    Frags x, y;
    load(x, wave);
    // what the end needs is asked for now
    using F = Finish<KIND, DT, 16 * J>;
    constexpr int lanes_rows = kWave * W / F::wide, turns = (16 * R + lanes_rows - 1) / lanes_rows;
    F finish(p, n0, lane);
    float a_step[turns];
#pragma unroll
    for (int t = 0; t < turns; ++t)
        a_step[t] = F::step_of_a(p.a_scales[min(m0 + static_cast<int>(threadIdx.x) / F::wide + t * lanes_rows, p.m - 1)]);
    for (int32_t at = wave; at < whole; at += 2 * P * W) {
        load(y, at + P * W);
        multiply(x);
        load(x, at + 2 * P * W);
        multiply(y);
    }
    int32_t* own = sums + wave * slab;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j)
            *reinterpret_cast<i32x4_t*>(own + (16 * i + fr) * S::pitch + 16 * j + 4 * fq) = acc[i][j];
    if constexpr (KIND == kMessage) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            int32_t v = ones[j];
            v += __shfl_xor(v, 16, kWave);
            v += __shfl_xor(v, 32, kWave);
            if (lane < 16) ones_of[(wave * J + j) * 16 + lane] = v;
        }
    }
    __syncthreads();
    if constexpr (KIND == kMessage) finish.take_ones(ones_of, W, 16 * J);
#pragma unroll
    for (int t = 0; t < turns; ++t) {
        const int r = static_cast<int>(threadIdx.x) / F::wide + t * lanes_rows;
        if (r < 16 * R) finish.template row<false, W>(m0 + r, a_step[t], finish.template added<false>(m0 + r), sums + r * S::pitch, slab);
    }
}

template <int DT, int R, int J, int W>
hipError_t launch_split_as(ProductKind kind, const ProductArgs& p, hipStream_t stream) {
    const uint32_t tm = (static_cast<uint32_t>(p.m) + 16 * R - 1) / (16 * R), tn = (static_cast<uint32_t>(p.n) + 16 * J - 1) / (16 * J);
    const dim3 grid(tm * tn), block(64 * W);
    switch (kind) {
    case kPlain:      return launch_kernel(product_split_kernel<kPlain, DT, R, J, W>, grid, block, stream, p, tn);
    case kMessage:    return launch_kernel(product_split_kernel<kMessage, DT, R, J, W>, grid, block, stream, p, tn);
    case kActivation: return launch_kernel(product_split_kernel<kActivation, DT, R, J, W>, grid, block, stream, p, tn);
    default:
        if constexpr (J % 2 == 0) return launch_kernel(product_split_kernel<kGated, DT, R, J, W>, grid, block, stream, p, tn);
        else return hipErrorInvalidValue;                       // the gate's columns come in pairs of sixteen
    }
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

enum ProductTile { kTile256 = 0, kTile128, kSplit64, kSplit64x32, kSplit32, kSplit16, kSplit16x32 };

template <int DT>
hipError_t launch_product_dt(ProductTile tile, ProductKind kind, const ProductArgs& p, hipStream_t stream) {
    switch (tile) {
    case kTile256: return launch_tiles_as<DT, 8, 4, 2, 4>(kind, p, stream);
    case kTile128: return launch_tiles_as<DT, 4, 4, 2, 2>(kind, p, stream);
    case kSplit64: return launch_split_as<DT, 4, 4, 8>(kind, p, stream);
    case kSplit64x32: return launch_split_as<DT, 4, 2, 8>(kind, p, stream);
    case kSplit32: return launch_split_as<DT, 2, 2, 8>(kind, p, stream);
    case kSplit16: return launch_split_as<DT, 1, 1, 8>(kind, p, stream);
    default:       return launch_split_as<DT, 1, 2, 8>(kind, p, stream);
    }
}

}  // namespace aqsgd
