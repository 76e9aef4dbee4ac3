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

// What is left of the sums once they lie in LDS as rows of 32-bit integers: a lane takes four columns of every few
// rows, so that its scales and bias are read once and a row leaves in whole lines.  COLS virtual columns from n0 on.
//
// STREAM: the results of large tiles go past the caches, in which they would take the room of the rows of a and b that
// other tiles still need, if rows of results are whole sectors of 32 bytes, so that no two waves share one: with ordinary
// stores and so, 4096 x 12800 x 1600 float16 gated, with what the backward pass needs, 124 us and 103; 8192 x 8192 x 2048
// float32 159 and 135, with 8200 columns 184 and 158; 2048 x 2048 x 1024 11.9 and 10.7; where sectors are shared, 5000 x
// 5001 x 512 bfloat16 27.7 and 33.5, 4096 x 6401 x 1600 float16 49.9 and 56.  Results of small tiles would
// only wait for memory then: 48 x 304 x 368 4.0 and 4.3.
template <int KIND, int DT, int COLS>
struct Finish {
    static constexpr int wide = (KIND == kGated ? COLS / 2 : COLS) / 4;       // lanes to a row
    static constexpr int step_rows = kWave / wide;                            // rows a wave takes at a time
    static_assert(wide >= 1 && wide <= kWave, "a wave takes whole rows");
    const ProductArgs& p;
    int32_t n, left, half;       // first column (of h, where gated), columns that remain from there
    int place;                   // of the lane's first sum in a row
    f32x4_t step, bias, extra, step_u, bias_u;

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
    }
    // Scales and bias of the lane's columns from memory (to be settled once they are needed) ...
    __device__ __forceinline__ f32x4_t scales(int32_t c, bool whole) const {
        if (whole) return *reinterpret_cast<const f32x4_any_t*>(p.b_scales + c);
        f32x4_t v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = p.b_scales[c + (e < left ? e : 0)];
        return v;
    }
    __device__ __forceinline__ f32x4_t biases(int32_t c, bool whole) const {          // bits, as they are stored
        f32x4_t v = {0, 0, 0, 0};
        if (!p.bias) return v;
        if constexpr (DT == AQSGD_F32) {
            const float* b = static_cast<const float*>(p.bias) + c;
            if (whole) return *reinterpret_cast<const f32x4_any_t*>(b);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = b[e < left ? e : 0];
        } else {
            const uint16_t* b = static_cast<const uint16_t*>(p.bias) + c;
            u16x4_any_t w;
            if (whole) {
                w = *reinterpret_cast<const u16x4_any_t*>(b);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = b[e < left ? e : 0];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(static_cast<uint32_t>(w[e]));
        }
        return v;
    }
    static __device__ __forceinline__ float value_of(float bits) {
        if constexpr (DT == AQSGD_F32) return bits;
        else if constexpr (DT == AQSGD_F16) return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(__float_as_uint(bits))));
        else return bf16_bits_to_f32(__float_as_uint(bits));
    }
    // whole: all of the tile's columns exist.
    __device__ __forceinline__ void ask_scales(bool whole) {
        const int32_t at = left > 0 ? n : 0;
        step = scales(at, whole);
        bias = biases(at, whole);
        if constexpr (KIND == kGated) {
            step_u = scales(half + at, whole);
            bias_u = biases(half + at, whole);
        }
    }
    __device__ __forceinline__ void settle_scales() {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            step[e] = step[e] / kCodeHalf;
            bias[e] = value_of(bias[e]);
            if constexpr (KIND == kGated) {
                step_u[e] = step_u[e] / kCodeHalf;
                bias_u[e] = value_of(bias_u[e]);
            }
        }
    }
    // ... or from LDS, by virtual column.
    __device__ __forceinline__ void take_scales(const float* b_step, const float* b_bias) {
        step = *reinterpret_cast<const f32x4_t*>(b_step + place);
        bias = *reinterpret_cast<const f32x4_t*>(b_bias + place);
        if constexpr (KIND == kGated) {
            step_u = *reinterpret_cast<const f32x4_t*>(b_step + place + 16);
            bias_u = *reinterpret_cast<const f32x4_t*>(b_bias + place + 16);
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
            v[e] = x * a_step * st[e] + bi[e];          // without a bias: 0
        }
        return v;
    }
    template <bool FULL, bool STREAM>
    __device__ __forceinline__ void put(void* base, int64_t at, const f32x4_t& v) const {
        if (FULL || left >= 4) {
            store4<DT, STREAM>(base, at, v);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < left) store_elem<DT>(base, at + e, v[e]);
        }
    }
    static __device__ __forceinline__ float step_of_a(float scale) { return scale / (KIND == kMessage ? kLevelHalf : kCodeHalf); }
    // What is there already in a row's columns, or 0.
    template <bool FULL, bool ADD>
    __device__ __forceinline__ f32x4_t added(int32_t m) const {
        f32x4_t v = {0, 0, 0, 0};
        if constexpr (ADD) {
            if (FULL || (m < p.m && left > 0)) {
                const int64_t at = static_cast<int64_t>(m) * p.n + n;
                if (FULL || left >= 4) {
                    v = load4<DT>(p.add, at);
                } else {
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (e < left) v[e] = load_elem<DT>(p.add, at + e);
                }
            }
        }
        return v;
    }
    // A row's columns: its sums in LDS, in PARTS parts `pitch` apart.
    template <int PARTS>
    __device__ __forceinline__ i32x4_t sum_of(const int32_t* sums, int pitch) const {
        i32x4_t s = *reinterpret_cast<const i32x4_t*>(sums);
#pragma unroll
        for (int k = 1; k < PARTS; ++k) s += *reinterpret_cast<const i32x4_t*>(sums + k * pitch);
        return s;
    }
    // FULL: the row and the four columns exist.
    template <bool FULL, int PARTS, bool STREAM>
    __device__ __forceinline__ void row(int32_t m, float a_step, const f32x4_t& there, const int32_t* sums, int pitch = 0) const {
        if (!FULL && (m >= p.m || left <= 0)) return;
        i32x4_t u = {0, 0, 0, 0};
        if constexpr (KIND == kGated) u = sum_of<PARTS>(sums + place + 16, pitch);
        finish<FULL, STREAM>(m, a_step, there, sum_of<PARTS>(sums + place, pitch), u);
    }
    template <bool FULL, bool STREAM>
    __device__ __forceinline__ void finish(int32_t m, float a_step, const f32x4_t& there, const i32x4_t& sum, const i32x4_t& sum_u) const {
        f32x4_t v = scaled(sum, a_step, step, bias);
        if constexpr (KIND == kGated) {
            const f32x4_t u = scaled(sum_u, a_step, step_u, bias_u);
            f32x4_t h;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = activation<DT>(p.act, v[e]) * u[e];
            put<FULL, STREAM>(p.out, static_cast<int64_t>(m) * half + n, h);
            if (p.pre) {
                put<FULL, STREAM>(p.pre, static_cast<int64_t>(m) * p.n + n, v);
                put<FULL, STREAM>(p.pre, static_cast<int64_t>(m) * p.n + half + n, u);
            }
        } else {
            const int64_t at = static_cast<int64_t>(m) * p.n + n;
            if constexpr (KIND == kActivation) {
                if (p.pre) put<FULL, STREAM>(p.pre, at, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = activation<DT>(p.act, v[e]);
            } else {
                v += there;
            }
            put<FULL, STREAM>(p.out, at, v);
        }
    }
};

// ---- large tiles ------------------------------------------------------------------------------
// A workgroup of WM x WN waves, each with TM x TN blocks of 16 x 16 sums (lane l holds row l % 16 of a block and four
// columns from (l / 16) * 4 on); k in steps of 128 bytes, two steps' operands in LDS.
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef const __attribute__((address_space(1))) void* global_ptr;

constexpr int kStoreBlocks = 2;                  // blocks of 16 rows that go through LDS at a time, at the end

template <int TM, int TN, int WM, int WN>
struct TileShape {
    static constexpr int bm = 16 * TM * WM, bn = 16 * TN * WN, waves = WM * WN;
    static constexpr int row = 128;                               // bytes of k in a step
    static constexpr int stage = (bm + bn) * row;                 // bytes of a step's operands
    static constexpr int loads_a = (bm / 8 + waves - 1) / waves, loads_b = (bn / 8 + waves - 1) / waves;    // 1 KB each, per wave
    static constexpr int loads_least = bm / 8 / waves + bn / 8 / waves;
    static constexpr int pitch = 16 * TN + 4;                     // words of a row of sums, at the end
    static constexpr int own = kStoreBlocks * 16 * pitch * 4;     // bytes of LDS of a wave, at the end
    static constexpr int work = 2 * stage > own * waves ? 2 * stage : own * waves;
    static constexpr int scales = (bm + 2 * bn) * 4;              // a's steps, b's steps, bias
    static constexpr int ones = WM * bn * 4;                      // sums of b's codes (message)
    static constexpr int lds = work + scales + ones;
    static_assert(TM % kStoreBlocks == 0, "the blocks leave in twos");
};

// Waits for all but the last N loads from memory of this wave, then for the workgroup.
template <int N>
__device__ __forceinline__ void barrier_but_last() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (0 << 8) | ((N >> 4) << 14));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int KIND, int DT, int TM, int TN, int WM, int WN>
__device__ __forceinline__ void product_tile(const ProductArgs& p, int32_t m0, int32_t n0, uint8_t* lds) {
    using S = TileShape<TM, TN, WM, WN>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave / WN) * TM * 16, wn = (wave % WN) * TN * 16;
    float* a_steps = reinterpret_cast<float*>(lds + S::work);
    float* b_steps = a_steps + S::bm;
    float* b_bias = b_steps + S::bn;
    int32_t* b_ones = reinterpret_cast<int32_t*>(b_bias + S::bn);

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
        off_a[i] = static_cast<uint32_t>(min((i * S::waves + wave) * 8 + lr, p.m - 1 - m0)) * static_cast<uint32_t>(p.lda);
#pragma unroll
    for (int i = 0; i < S::loads_b; ++i) off_b[i] = row_from<KIND>(n0, (i * S::waves + wave) * 8 + lr, p.n) * static_cast<uint32_t>(p.ldb);
    const int32_t halves = (p.k + 63) / 64, steps = (halves + 1) / 2;
    const int32_t last_a = (KIND == kMessage ? p.k : halves * 64) - 16, last_b = halves * 64 - 16;
    auto bring = [&](int32_t step, int buf) {
        const int32_t k = step * S::row + piece;
        const uint32_t ka = min(k, last_a), kb = min(k, last_b);
        uint8_t* to = lds + buf * S::stage;
#pragma unroll
        for (int i = 0; i < S::loads_a; ++i) {
            const int at = i * S::waves + wave;
            if (S::bm / 8 % S::waves == 0 || at < S::bm / 8)
                __builtin_amdgcn_global_load_lds((global_ptr)(base_a + (off_a[i] + ka)), (lds_ptr)(to + at * 1024), 16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < S::loads_b; ++i) {
            const int at = i * S::waves + wave;
            const int8_t* b = KIND == kGated && (at & 2) ? base_u : base_b;
            if (S::bn / 8 % S::waves == 0 || at < S::bn / 8)
                __builtin_amdgcn_global_load_lds((global_ptr)(b + (off_b[i] + kb)), (lds_ptr)(to + S::bm * S::row + at * 1024), 16, 0, 0);
        }
    };
    // What the end needs is asked for first and lies in LDS by then: nothing is waited for there.
    static_assert(S::bm <= 64 * S::waves && S::bn <= 64 * S::waves, "a lane for every row and column");
    const int t = threadIdx.x;
    float a_scale = 0.0f, b_scale = 0.0f, b_add = 0.0f;
    if (t < S::bm) a_scale = p.a_scales[min(m0 + t, p.m - 1)];
    if (t < S::bn) {
        const int32_t r = static_cast<int32_t>(row_from<KIND>(n0, t, p.n)) + (KIND == kGated ? (n0 >> 1) + ((t & 16) ? half : 0) : n0);
        b_scale = p.b_scales[r];
        if (p.bias) b_add = load_elem<DT>(p.bias, r);
    }
    if (steps > 0) {
        bring(0, 0);
        bring(min(1, steps - 1), 1);
    }
    if (t < S::bm) a_steps[t] = Finish<KIND, DT, 16 * TN>::step_of_a(a_scale);
    if (t < S::bn) {
        b_steps[t] = b_scale / kCodeHalf;
        b_bias[t] = b_add;
    }
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
    // Of the WM waves that hold the same columns of b, each adds up the codes of every WM-th half step.
    auto multiply = [&](i32x4_t (&fa)[TM], i32x4_t (&fb)[TN], int32_t h) {
        if constexpr (KIND == kMessage) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) fa[i][e] ^= static_cast<int32_t>(0x80808080u);      // level - 128
            if (h % WM == wave / WN) {
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) ones[j] = __builtin_amdgcn_sdot4(fb[j][e], 0x01010101, ones[j], false);
            }
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    };
    i32x4_t fa0[TM], fb0[TN], fa1[TM], fb1[TN];
    // The schedule of a half step: its products with the other accesses between them, so that none of them holds the
    // wave's products back (a load takes the memory pipe 16 cycles, and eight waves issue theirs at once).
    const auto interleave = [&](auto loads) {
        constexpr int ds = TM + TN, n = TM * TN, vm = decltype(loads)::value;
        constexpr int pairs = vm > 0 ? (ds + 1) / 2 : ds;                  // products between the reads
        constexpr int each = vm > 0 ? (n - pairs > vm ? (n - pairs) / (vm > 0 ? vm : 1) : 1) : (n / pairs > 1 ? 2 : 1);
#pragma unroll
        for (int i = 0; i < pairs; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, vm > 0 ? 2 : 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, vm > 0 ? 1 : each, 0);
        }
#pragma unroll
        for (int i = 0; i < vm; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, each, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, n, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    if (steps > 0) {
        barrier_but_last<S::loads_least>();
        read_frags(fa0, fb0, 0, 0);
        for (int32_t s = 0; s < steps - 1; ++s) {
            const int buf = s & 1;
            read_frags(fa1, fb1, buf, 1);
            multiply(fa0, fb0, 2 * s);
            interleave(std::integral_constant<int, 0>());
            barrier_but_last<0>();                       // step s + 1 has arrived; no wave reads step s any more
            read_frags(fa0, fb0, buf ^ 1, 0);
            bring(min(s + 2, steps - 1), buf);           // the last one once more: nobody reads it
            multiply(fa1, fb1, 2 * s + 1);
            interleave(std::integral_constant<int, S::loads_a + S::loads_b>());
        }
        if (halves % 2 == 0) read_frags(fa1, fb1, (steps - 1) & 1, 1);
        multiply(fa0, fb0, 2 * steps - 2);
        if (halves % 2 == 0) multiply(fa1, fb1, 2 * steps - 1);
    }
    if constexpr (KIND == kMessage) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            int32_t v = ones[j];
            v += __shfl_xor(v, 16, kWave);
            v += __shfl_xor(v, 32, kWave);
            if (lane < 16) b_ones[(wave / WN) * S::bn + wn + 16 * j + lane] = v;
        }
    }
    barrier_but_last<0>();                               // the last fragments have been read, the last loads are in

    using F = Finish<KIND, DT, TN * 16>;
    F finish(p, n0 + wn, lane);
    finish.take_scales(b_steps + wn, b_bias + wn);
    if constexpr (KIND == kMessage) finish.take_ones(b_ones + wn, WM, S::bn);
    int32_t* own = reinterpret_cast<int32_t*>(lds + wave * S::own);
    int32_t* to = own + fr * S::pitch + fq * 4;
    constexpr int rows = kStoreBlocks * 16, turns = (rows + F::step_rows - 1) / F::step_rows;
    constexpr int ahead = turns % 8 == 0 ? 8 : turns % 4 == 0 ? 4 : turns % 2 == 0 ? 2 : 1;
    const bool full = m0 + wm + 16 * TM <= p.m && n0 + wn + 16 * TN <= (KIND == kGated ? p.n & ~31 : p.n);     // h is whole sixteens there
    const int mine = lane / F::wide;
    const bool busy = F::step_rows * F::wide == kWave || mine < F::step_rows;
    const auto store = [&](auto adds, auto streams) {
        constexpr bool ADD = decltype(adds)::value, STREAM = decltype(streams)::value;
#pragma unroll
        for (int i0 = 0; i0 < TM; i0 += kStoreBlocks) {
#pragma unroll
            for (int i = 0; i < kStoreBlocks; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) *reinterpret_cast<i32x4_t*>(to + i * 16 * S::pitch + 16 * j) = acc[i0 + i][j];
            const int32_t first = m0 + wm + i0 * 16 + mine;
            const float* a_step = a_steps + wm + i0 * 16 + mine;
            if (full && rows % F::step_rows == 0) {
                if (busy) {
#pragma unroll 1
                    for (int t = 0; t < turns; t += ahead) {
                        f32x4_t there[ahead];
#pragma unroll
                        for (int u = 0; u < ahead; ++u) there[u] = finish.template added<true, ADD>(first + (t + u) * F::step_rows);
#pragma unroll
                        for (int u = 0; u < ahead; ++u) {
                            const int r = (t + u) * F::step_rows;
                            finish.template row<true, 1, STREAM>(first + r, a_step[r], there[u], own + (mine + r) * S::pitch);
                        }
                    }
                }
            } else {
                // several rows' sums at a time (12072 x 944 x 136 13.5 us, one at a time 13.7; the gated product is 2 % slower so)
                constexpr int most = KIND == kGated ? 1 : 4, few = ahead < most ? ahead : most;
#pragma unroll 1
                for (int t = 0; t < turns; t += few) {
                    f32x4_t there[few];
                    i32x4_t sum[few], sum_u[few] = {};
                    float step[few];
#pragma unroll
                    for (int u = 0; u < few; ++u) {
                        const int r = (t + u) * F::step_rows, at = min(r, rows - 1 - mine);
                        there[u] = finish.template added<false, ADD>(first + r);
                        sum[u] = *reinterpret_cast<const i32x4_t*>(own + (mine + at) * S::pitch + finish.place);
                        if constexpr (KIND == kGated) sum_u[u] = *reinterpret_cast<const i32x4_t*>(own + (mine + at) * S::pitch + finish.place + 16);
                        step[u] = a_step[at];
                    }
#pragma unroll
                    for (int u = 0; u < few; ++u) {
                        const int r = (t + u) * F::step_rows;
                        if (busy && mine + r < rows && first + r < p.m && finish.left > 0) finish.template finish<false, STREAM>(first + r, step[u], there[u], sum[u], sum_u[u]);
                    }
                }
            }
        }
    };
    if ((KIND == kPlain || KIND == kMessage) && p.add) {
        if (p.stream) store(std::true_type(), std::true_type());
        else store(std::true_type(), std::false_type());
    } else {
        if (p.stream) store(std::false_type(), std::true_type());
        else store(std::false_type(), std::false_type());
    }
}

// Tile t of a grid of tiles: they go down in bands of kBand tile rows, so that the tiles an XCD works on at a time
// share rows of a and of b in its L2.
constexpr uint32_t kBand = 4;
__device__ __forceinline__ void tile_of(uint32_t t, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn) {
    const uint32_t band = t / (kBand * tiles_n), in = t - band * kBand * tiles_n;
    const uint32_t rows = min(kBand, tiles_m - band * kBand);
    tm = band * kBand + in % rows;
    tn = in / rows;
}
// The eight XCDs take the workgroups in turn, so that b mod 8 is the XCD; each gets a contiguous run of 0 .. total - 1.
__device__ __forceinline__ uint32_t spread_over_xcds(uint32_t b, uint32_t total) {
    const uint32_t q = total >> 3, r = total & 7, x = b & 7;
    return x * q + min(x, r) + (b >> 3);
}

// Workgroups 0 .. wide_tiles_n * tiles_m - 1 take tiles of full width, the others narrower ones (NARROW blocks to a
// wave) of the columns that are left.
template <int KIND, int DT, int TM, int TN, int WM, int WN, int NARROW>
__global__ __launch_bounds__(64 * WM * WN, 1) void product_tile_kernel(const ProductArgs p, uint32_t tiles_m, uint32_t wide_tiles_n,
                                                                       uint32_t narrow_tiles_n) {
    using S = TileShape<TM, TN, WM, WN>;
    __shared__ __attribute__((aligned(128))) uint8_t lds[S::lds];
    const uint32_t wide = tiles_m * wide_tiles_n;
    uint32_t tm, tn;
    if (NARROW == 0 || blockIdx.x < wide) {
        tile_of(spread_over_xcds(blockIdx.x, wide), tiles_m, wide_tiles_n, tm, tn);
        product_tile<KIND, DT, TM, TN, WM, WN>(p, static_cast<int32_t>(tm) * S::bm, static_cast<int32_t>(tn) * S::bn, lds);
    } else if constexpr (NARROW > 0) {
        tile_of(spread_over_xcds(blockIdx.x - wide, tiles_m * narrow_tiles_n), tiles_m, narrow_tiles_n, tm, tn);
        product_tile<KIND, DT, TM, NARROW, WM, WN>(p, static_cast<int32_t>(tm) * S::bm,
                                                   static_cast<int32_t>(wide_tiles_n) * S::bn + static_cast<int32_t>(tn) * (16 * NARROW * WN), lds);
    }
}

// ---- small products ---------------------------------------------------------------------------
// 16 R x 16 J sums to a workgroup, its W waves sharing out k in pieces of 128 bytes: nothing is staged, every wave
// loads the fragments of its pieces from memory into registers, the next ones while it multiplies, and the waves'
// sums meet in LDS once, at the end.  Where tiles are few and k is long, the pieces of a tile are shared out over several
// workgroups (SLICED): each leaves its sums in the workspace, and a second kernel joins and finishes them.
struct Slices {
    int32_t* sums;             // [slices, m, pitch], then the sums of b's codes [slices, pitch]
    int32_t count, pieces;     // of slices; of 128 bytes of k to a slice
    int32_t pitch;
};

template <int KIND, int R, int J> struct SplitShape {
    // Pieces that are asked for together, twice over: as many as leave the registers of four waves to a SIMD.
    static constexpr int most = R + J >= 4 ? 1 : R + J == 3 ? 2 : 3;
    static constexpr int pieces = most > 1 && (KIND == kMessage || KIND == kGated) ? most - 1 : most;
    static constexpr int waves = R + J <= 4 ? 4 : 2;                          // of a SIMD: two workgroups to a CU, or one
    static constexpr int pitch = 16 * J + 4;
};

template <int KIND, int DT, int R, int J, int W, bool SLICED>
__global__ __launch_bounds__(64 * W, (SplitShape<KIND, R, J>::waves)) void product_split_kernel(const ProductArgs p, uint32_t tiles_n, Slices slices) {
    using S = SplitShape<KIND, R, J>;
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
    const int32_t last_a = (KIND == kMessage ? p.k : (p.k + 63) / 64 * 64) - 16;
    const int32_t slice = SLICED ? static_cast<int32_t>(blockIdx.y) : 0, begin = SLICED ? slice * slices.pieces : 0;
    const int32_t halves = SLICED ? min((p.k + 63) / 64, 2 * (begin + slices.pieces)) : (p.k + 63) / 64, whole = (halves + 1) / 2;
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
    load(x, begin + wave);
    // what the end needs is asked for now
    using F = Finish<KIND, DT, 16 * J>;
    constexpr int lanes_rows = kWave * W / F::wide, turns = (16 * R + lanes_rows - 1) / lanes_rows;
    F finish(p, n0, lane);
    if (!SLICED) finish.ask_scales(n0 + 16 * J <= (KIND == kGated ? p.n & ~31 : p.n));         // h is whole sixteens there
    float a_step[turns];
#pragma unroll
    for (int t = 0; t < turns && !SLICED; ++t)
        a_step[t] = p.a_scales[min(m0 + static_cast<int>(threadIdx.x) / F::wide + t * lanes_rows, p.m - 1)];
    for (int32_t at = begin + wave; at < whole; at += 2 * P * W) {
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
    if constexpr (SLICED) {
#pragma unroll
        for (int t = 0; t < turns; ++t) {
            const int r = static_cast<int>(threadIdx.x) / F::wide + t * lanes_rows;
            if (r < 16 * R && m0 + r < p.m)
                *reinterpret_cast<i32x4_t*>(slices.sums + (static_cast<int64_t>(slice) * p.m + m0 + r) * slices.pitch + n0 + finish.place) =
                    finish.template sum_of<W>(sums + r * S::pitch + finish.place, slab);
        }
        if constexpr (KIND == kMessage) {
            if (m0 == 0 && threadIdx.x < 16 * J) {
                int32_t s = 0;
                for (int w = 0; w < W; ++w) s += ones_of[w * 16 * J + threadIdx.x];
                slices.sums[(static_cast<int64_t>(slices.count) * p.m + slice) * slices.pitch + n0 + threadIdx.x] = s;
            }
        }
        return;
    }
    if constexpr (KIND == kMessage) finish.take_ones(ones_of, W, 16 * J);
    finish.settle_scales();
#pragma unroll
    for (int t = 0; t < turns; ++t) {
        const int r = static_cast<int>(threadIdx.x) / F::wide + t * lanes_rows;
        if (r >= 16 * R) continue;
        const bool adds = (KIND == kPlain || KIND == kMessage) && p.add;
        finish.template row<false, W, false>(m0 + r, F::step_of_a(a_step[t]), adds ? finish.template added<false, true>(m0 + r) : f32x4_t{0, 0, 0, 0},
                                      sums + r * S::pitch, slab);
    }
}

// The slices' sums joined: a lane takes four columns of a row.
template <int KIND, int DT>
__global__ __launch_bounds__(256) void product_join_kernel(const ProductArgs p, Slices slices) {
    const uint32_t fours = (static_cast<uint32_t>(p.n) + 3) / 4, i = blockIdx.x * 256 + threadIdx.x;
    const int32_t m = static_cast<int32_t>(i / fours), n = static_cast<int32_t>(i % fours) * 4;
    if (m >= p.m) return;
    using F = Finish<KIND, DT, 256>;
    F finish(p, n, 0);
    finish.ask_scales(n + 4 <= p.n);
    const float a_scale = p.a_scales[m];
    const f32x4_t there = p.add ? finish.template added<false, true>(m) : f32x4_t{0, 0, 0, 0};
    i32x4_t sum = {0, 0, 0, 0}, ones = {0, 0, 0, 0};
    for (int32_t s = 0; s < slices.count; ++s) {
        sum += *reinterpret_cast<const i32x4_t*>(slices.sums + (static_cast<int64_t>(s) * p.m + m) * slices.pitch + n);
        if constexpr (KIND == kMessage)
            ones += *reinterpret_cast<const i32x4_t*>(slices.sums + (static_cast<int64_t>(slices.count) * p.m + s) * slices.pitch + n);
    }
    if constexpr (KIND == kMessage) finish.take_ones(reinterpret_cast<const int32_t*>(&ones), 1, 0);
    finish.settle_scales();
    finish.template finish<false, false>(m, F::step_of_a(a_scale), there, sum, sum);
}

template <int KIND, int DT, int R, int J, int W>
hipError_t launch_split_kind(const ProductArgs& p, const Slices& slices, hipStream_t stream) {
    const uint32_t tm = (static_cast<uint32_t>(p.m) + 16 * R - 1) / (16 * R), tn = (static_cast<uint32_t>(p.n) + 16 * J - 1) / (16 * J);
    if constexpr (KIND == kPlain || KIND == kMessage) {
        if (slices.count > 1) {
            ProfileSpan span;
            const hipError_t err = launch_kernel(product_split_kernel<KIND, DT, R, J, W, true>, dim3(tm * tn, static_cast<unsigned>(slices.count)),
                                                 dim3(64 * W), stream, p, tn, slices);
            span.last();
            if (err != hipSuccess) return err;
            const uint32_t fours = static_cast<uint32_t>(p.m) * ((static_cast<uint32_t>(p.n) + 3) / 4);
            return launch_kernel(product_join_kernel<KIND, DT>, dim3((fours + 255) / 256), dim3(256), stream, p, slices);
        }
    }
    return launch_kernel(product_split_kernel<KIND, DT, R, J, W, false>, dim3(tm * tn), dim3(64 * W), stream, p, tn, slices);
}

template <int DT, int R, int J, int W>
hipError_t launch_split_as(ProductKind kind, const ProductArgs& p, const Slices& slices, hipStream_t stream) {
    switch (kind) {
    case kPlain:      return launch_split_kind<kPlain, DT, R, J, W>(p, slices, stream);
    case kMessage:    return launch_split_kind<kMessage, DT, R, J, W>(p, slices, stream);
    case kActivation: return launch_split_kind<kActivation, DT, R, J, W>(p, slices, stream);
    default:
        if constexpr (J % 2 == 0) return launch_split_kind<kGated, DT, R, J, W>(p, slices, stream);
        else return hipErrorInvalidValue;                       // the gate's columns come in pairs of sixteen
    }
}

// How a product is cut: rows of tiles, columns of tiles of full width, columns of narrower ones.
struct TilePlan {
    uint32_t tiles_m, wide_n, narrow_n;
    int narrow;                                  // blocks to a wave of the narrower ones, 0: none
};

template <int DT, int TM, int TN, int WM, int WN, int NARROW>
hipError_t launch_tiles_as(ProductKind kind, const TilePlan& t, const ProductArgs& p, hipStream_t stream) {
    const dim3 grid(t.tiles_m * (t.wide_n + t.narrow_n)), block(64 * WM * WN);
    switch (kind) {
    case kPlain:
        return launch_kernel(product_tile_kernel<kPlain, DT, TM, TN, WM, WN, NARROW>, grid, block, stream, p, t.tiles_m, t.wide_n, t.narrow_n);
    case kMessage:
        return launch_kernel(product_tile_kernel<kMessage, DT, TM, TN, WM, WN, NARROW>, grid, block, stream, p, t.tiles_m, t.wide_n, t.narrow_n);
    case kActivation:
        return launch_kernel(product_tile_kernel<kActivation, DT, TM, TN, WM, WN, NARROW>, grid, block, stream, p, t.tiles_m, t.wide_n, t.narrow_n);
    default:
        if constexpr (NARROW % 2 == 0)           // the gate's columns come in pairs of sixteen
            return launch_kernel(product_tile_kernel<kGated, DT, TM, TN, WM, WN, NARROW>, grid, block, stream, p, t.tiles_m, t.wide_n, t.narrow_n);
        else return hipErrorInvalidValue;
    }
}

template <int DT>
hipError_t launch_tiles256_dt(ProductKind kind, const TilePlan& t, const ProductArgs& p, hipStream_t stream) {
    switch (t.narrow) {
    case 0: return launch_tiles_as<DT, 4, 8, 4, 2, 0>(kind, t, p, stream);
    case 2: return launch_tiles_as<DT, 4, 8, 4, 2, 2>(kind, t, p, stream);
    case 3: return launch_tiles_as<DT, 4, 8, 4, 2, 3>(kind, t, p, stream);
    case 4: return launch_tiles_as<DT, 4, 8, 4, 2, 4>(kind, t, p, stream);
    case 5: return launch_tiles_as<DT, 4, 8, 4, 2, 5>(kind, t, p, stream);
    case 6: return launch_tiles_as<DT, 4, 8, 4, 2, 6>(kind, t, p, stream);
    default: return launch_tiles_as<DT, 4, 8, 4, 2, 7>(kind, t, p, stream);
    }
}

// Tiles of 128 rows and 128 or 64 columns, two or three workgroups to a CU.
template <int DT>
hipError_t launch_tiles128_dt(int cols, ProductKind kind, const ProductArgs& p, hipStream_t stream) {
    const TilePlan t{(static_cast<uint32_t>(p.m) + 127) / 128, (static_cast<uint32_t>(p.n) + cols - 1) / cols, 0, 0};
    return cols == 128 ? launch_tiles_as<DT, 4, 4, 2, 2, 0>(kind, t, p, stream) : launch_tiles_as<DT, 4, 2, 2, 2, 0>(kind, t, p, stream);
}

enum SplitTile { kSplit64 = 0, kSplit64x32, kSplit32, kSplit16, kSplit16x32 };

template <int DT>
hipError_t launch_split_dt(SplitTile tile, ProductKind kind, const ProductArgs& p, const Slices& slices, hipStream_t stream) {
    switch (tile) {
    case kSplit64: return launch_split_as<DT, 4, 4, 8>(kind, p, slices, stream);
    case kSplit64x32: return launch_split_as<DT, 4, 2, 8>(kind, p, slices, stream);
    case kSplit32: return launch_split_as<DT, 2, 2, 8>(kind, p, slices, stream);
    case kSplit16: return launch_split_as<DT, 1, 1, 8>(kind, p, slices, stream);
    default:       return launch_split_as<DT, 1, 2, 8>(kind, p, slices, stream);
    }
}

#define AQSGD_PRODUCT_DT(EXTERN, DT)                                                                                        \
    EXTERN template hipError_t launch_tiles256_dt<DT>(ProductKind, const TilePlan&, const ProductArgs&, hipStream_t);      \
    EXTERN template hipError_t launch_tiles128_dt<DT>(int, ProductKind, const ProductArgs&, hipStream_t);                  \
    EXTERN template hipError_t launch_split_dt<DT>(SplitTile, ProductKind, const ProductArgs&, const Slices&, hipStream_t);

}  // namespace aqsgd
