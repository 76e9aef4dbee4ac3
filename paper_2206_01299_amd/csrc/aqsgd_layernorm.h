// Kernels of aqsgd_layernorm and aqsgd_layernorm_grad.
//
// Both read a row once into the registers of a team of lanes (a fraction of a wave, a wave, or a workgroup of up to
// 1024), which forms the row's sums between the load and the store.  What bounds them is memory, and in small calls a launch and
// one chain of load, two sums and store: one row of 1600 float16 2.9 us, 4096 such rows with residual, codes and statistics 12.0 (4.9
// TB/s), 16384 of 4096 float32 96 (5.6 TB/s); their gradients 2.4, 16.4 and 189.  The forward pass sums in
// binary64, which costs little here: statistics then depend on the order, and with it on the launch, only where a sum's last places in
// binary64 decide how it rounds to binary32.  Lanes take pieces of 16 bytes side by side.
#pragma once

#include <optional>
#include <utility>

#include "aqsgd_norms.h"
#include "aqsgd_quant8.h"

namespace aqsgd {

template <int DT> constexpr int kPiece = 16 / ElemBytes<DT>::value;            // elements of a piece

template <int DT>
__device__ __forceinline__ void piece_values(const u32x4_t& r, float (&f)[kPiece<DT>]) {
    if constexpr (DT == AQSGD_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(r[e]);
    } else {
        unpack_raw<DT>(Raw<DT>{r}, f);
    }
}

template <int DT>
__device__ __forceinline__ u32x4_t values_piece(const float (&f)[kPiece<DT>]) {
    if constexpr (DT == AQSGD_F32) return u32x4_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    else return pack_raw<DT>(f).v;
}

// The piece from column c on of a row that starts at element `at`.  Rows have at least a piece's elements.  LAST: a piece
// that may lie across the row's end (RAGGED) or behind it; such a lane reads the row's last elements instead.
template <int DT, bool LAST>
__device__ __forceinline__ u32x4_t load_piece(const void* base, int64_t at, int32_t c, int32_t cols) {
    const char* row = element_at<DT>(base, at);
    return *reinterpret_cast<const u32x4_any_t*>(row + (LAST ? min(c, cols - kPiece<DT>) : c) * ElemBytes<DT>::value);
}

// What was so read, each element at its column.  Where there is no column: some other element of the row.
template <int DT, bool LAST, bool RAGGED>
__device__ __forceinline__ u32x4_t placed_piece(u32x4_t r, int32_t c, int32_t cols) {
    if constexpr (LAST && RAGGED) {
        const int down = c + kPiece<DT> - cols;          // columns that do not exist
        if (down > 0 && down < kPiece<DT>) {
            if constexpr (DT == AQSGD_F32) {
                if (down & 2) r = u32x4_t{r[2], r[3], r[0], r[1]};
                if (down & 1) r = u32x4_t{r[1], r[2], r[3], r[0]};
            } else {
                if (down & 4) r = u32x4_t{r[2], r[3], r[0], r[1]};
                if (down & 2) r = u32x4_t{r[1], r[2], r[3], r[0]};
                if (down & 1) r = u32x4_t{r[0] >> 16 | r[1] << 16, r[1] >> 16 | r[2] << 16, r[2] >> 16 | r[3] << 16, r[3] >> 16 | r[0] << 16};
            }
        }
    }
    return r;
}

// The same with 0 where there is no column.
template <int DT, bool LAST, bool RAGGED>
__device__ __forceinline__ u32x4_t whole_piece(u32x4_t r, int32_t c, int32_t cols) {
    if constexpr (!LAST) return r;
    if constexpr (RAGGED) {
        const int down = c + kPiece<DT> - cols;
        if (down > 0 && down < kPiece<DT>) {
            if constexpr (DT == AQSGD_F32) {
                if (down & 2) r = u32x4_t{r[2], r[3], 0, 0};
                if (down & 1) r = u32x4_t{r[1], r[2], r[3], 0};
            } else {
                if (down & 4) r = u32x4_t{r[2], r[3], 0, 0};
                if (down & 2) r = u32x4_t{r[1], r[2], r[3], 0};
                if (down & 1) r = u32x4_t{r[0] >> 16 | r[1] << 16, r[1] >> 16 | r[2] << 16, r[2] >> 16 | r[3] << 16, r[3] >> 16};
            }
        }
    }
    return c < cols ? r : u32x4_t{0, 0, 0, 0};
}

// A value as the type holds it.
template <int DT>
__device__ __forceinline__ float rounded_to(float f) {
    if constexpr (DT == AQSGD_F16) return static_cast<float>(static_cast<_Float16>(f));
    else if constexpr (DT == AQSGD_BF16) return bf16_bits_to_f32(f32_to_bf16_bits(f));
    return f;
}

template <int DT>
__device__ __forceinline__ char* element_at(void* base, int64_t i) {
    return static_cast<char*>(base) + i * ElemBytes<DT>::value;
}

// Stores what exists of a piece, past the caches: 4096 x 1600 float16 with residual and codes 14.2 us, with ordinary
// stores 16.0; 16384 x 4096 float32 96.6 and 101.4.
template <int DT, bool LAST, bool RAGGED>
__device__ __forceinline__ void store_piece_of(void* base, int64_t at, int32_t c, int32_t cols, const u32x4_t& r) {
    char* row = element_at<DT>(base, at);
    if (!LAST || c + (RAGGED ? kPiece<DT> : 1) <= cols) {
        stream16(row + c * ElemBytes<DT>::value, r);
    } else if constexpr (RAGGED) {
#pragma unroll
        for (int e = 0; e < kPiece<DT> - 1; ++e) {
            if (c + e >= cols) continue;
            if constexpr (DT == AQSGD_F32) reinterpret_cast<uint32_t*>(row)[c + e] = r[e];
            else reinterpret_cast<uint16_t*>(row)[c + e] = static_cast<uint16_t>(r[e >> 1] >> (16 * (e & 1)));
        }
    }
}

// A team's number in its workgroup: the same for all of a wave, where the team has a wave's lanes or more.
template <int TEAM>
__device__ __forceinline__ int team_number() {
    const int t = static_cast<int>(threadIdx.x) / TEAM;
    return TEAM >= kWave ? __builtin_amdgcn_readfirstlane(t) : t;
}

// f(i, whether it may lie across or behind the row's end) for each of a lane's pieces: its last one, of eight the last four.
template <typename F, int... I>
__device__ __forceinline__ void each_of(F& f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>(), std::bool_constant<I == sizeof...(I) - 1 || (sizeof...(I) == 8 && I >= 4)>()), ...);
}
template <int CPL, typename F>
__device__ __forceinline__ void each_piece(F&& f) { each_of(f, std::make_integer_sequence<int, CPL>()); }

// ---- sums over a team, the same bits in all of its lanes ---------------------------------------
template <int CTRL> __device__ __forceinline__ float dpp_moved(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <int CTRL> __device__ __forceinline__ double dpp_moved(double v) {
    const int lo = __double2loint(v), hi = __double2hiint(v);
    return __hiloint2double(__builtin_amdgcn_update_dpp(hi, hi, CTRL, 0xf, 0xf, false), __builtin_amdgcn_update_dpp(lo, lo, CTRL, 0xf, 0xf, false));
}

// v plus its counterpart in the other half of 32 lanes (HALF 16), or of the wave (HALF 32): a swap of two registers'
// halves, which costs no trip through LDS.
template <int HALF>
__device__ __forceinline__ uint2 halves_swapped(uint32_t v) {
    const auto r = HALF == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return uint2{r[0], r[1]};
}
template <int HALF> __device__ __forceinline__ float halves_sum(float v) {
    const uint2 r = halves_swapped<HALF>(__float_as_uint(v));
    return __uint_as_float(r.x) + __uint_as_float(r.y);
}
template <int HALF> __device__ __forceinline__ double halves_sum(double v) {
    const uint2 lo = halves_swapped<HALF>(static_cast<uint32_t>(__double2loint(v))), hi = halves_swapped<HALF>(static_cast<uint32_t>(__double2hiint(v)));
    return __hiloint2double(static_cast<int>(hi.x), static_cast<int>(lo.x)) + __hiloint2double(static_cast<int>(hi.y), static_cast<int>(lo.y));
}

template <int LANES, typename T>
__device__ __forceinline__ T lanes_sum(T v) {
    if constexpr (LANES >= 2) v += dpp_moved<0xB1>(v);     // quad_perm [1,0,3,2]
    if constexpr (LANES >= 4) v += dpp_moved<0x4E>(v);     // quad_perm [2,3,0,1]
    if constexpr (LANES >= 8) v += dpp_moved<0x141>(v);    // row_half_mirror
    if constexpr (LANES >= 16) v += dpp_moved<0x140>(v);   // row_mirror
    if constexpr (LANES >= 32) v = halves_sum<16>(v);
    if constexpr (LANES >= 64) v = halves_sum<32>(v);
    return v;
}

// `part`: a word for each of the workgroup's waves, not in use otherwise since the last barrier.
template <int TEAM, typename T>
__device__ __forceinline__ T team_sum(T v, T* part) {
    if constexpr (TEAM <= kWave) {
        return lanes_sum<TEAM>(v);
    } else {
        v = lanes_sum<kWave>(v);
        if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = v;
        __syncthreads();
        const T* of = part + threadIdx.x / TEAM * (TEAM / kWave);
        T sum = of[0];
#pragma unroll
        for (int w = 1; w < TEAM / kWave; ++w) sum += of[w];
        return sum;
    }
}

template <int TEAM>
__device__ __forceinline__ uint32_t team_top(uint32_t v, uint32_t* part) {
    v = __float_as_uint(team_max<(TEAM < kWave ? TEAM : kWave)>(__uint_as_float(v)));
    if constexpr (TEAM > kWave) {
        if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = v;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TEAM / kWave; ++w) v = max(v, part[w]);
    }
    return v;
}

struct TeamSpace {                       // of a workgroup that is one team
    double first[16], second[16];
    uint32_t top[16];
};

// A sum over the columns by their number, the quotient rounded once.  Its product with the rounded inverse `each` is up to 1.5 units
// of the last place off, which at a width of 49, 300 or 1537 puts a quotient in the middle between two binary32 numbers on
// one side of it.  The residual is a multiple of that unit below 1.5 cols of them, so it has no error, and the step by it none of
// 2^-52 units.  A quotient that is not in the middle between two binary64 numbers is 1 / (2 cols) units or more from it, cols being
// at most 2^24, and none is in the middle: that has 54 bits, and its product with cols, the sum, no fewer.
__device__ __forceinline__ double column_mean(double sum, int32_t cols, double each) {
    const double q = sum * each;
    return fabs(q) < __builtin_inf() ? fma(fma(-q, static_cast<double>(cols), sum), each, q) : q;
}

// 1 / sqrt of the variance, in binary64 to its last places and then rounded: the hardware's (2^-24 of it off at most) and two steps of Newton's, ten
// operations instead of some sixty for a root and a quotient (4096 x 1600 float16 with residual and codes 12.8 -> 12.2 us).
__device__ __forceinline__ float inverse_deviation(double squares, int32_t cols, double each, double eps) {
    const double v = column_mean(squares, cols, each) + eps;
    double y = __builtin_amdgcn_rsq(v);
    if (v > 0.0 && v < __builtin_inf()) {
#pragma unroll
        for (int i = 0; i < 2; ++i) y = fma(0.5 * y, fma(-v * y, y, 1.0), y);
    }
    return static_cast<float>(y);
}

// The codes of a piece of y.
template <int DT>
__device__ __forceinline__ void store_codes(int8_t* to, const u32x4_t& y, float inv) {
    constexpr int V = kPiece<DT>;
    float f[V];
    piece_values<DT>(y, f);
    uint32_t k[V / 4];
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
        int32_t c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = code_of<AQSGD_ROUND_NEAREST>(f[4 * q + e], inv, 0.5f);
        k[q] = pack_codes(c[0], c[1], c[2], c[3]);
    }
    if constexpr (V == 8) *reinterpret_cast<u32x2_t*>(to) = u32x2_t{k[0], k[1]};
    else *reinterpret_cast<uint32_t*>(to) = k[0];
}

// ---- forward -----------------------------------------------------------------------------------
template <int DT, int TEAM, int CPL, bool RAGGED>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void layernorm_kernel(const LayernormArgs a) {
    constexpr int kRows = (TEAM < 256 ? 256 : TEAM) / TEAM, V = kPiece<DT>;
    static_assert(TEAM * V % kCodePad == 0, "the lanes that write a row's codes write the zeros behind them");
    __shared__ TeamSpace space;
    const int lane = threadIdx.x % TEAM, team = team_number<TEAM>();
    const auto column = [&](int i) { return (i * TEAM + lane) * V; };
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * kRows; first < a.rows; first += static_cast<int64_t>(gridDim.x) * kRows) {
        const bool here = first + team < a.rows;
        const int64_t row = here ? first + team : a.rows - 1;          // the last row again: its lanes store nothing
        // Weight and bias are asked for with the row where registers allow (4096 x 1600 float16 with residual and codes
        // 13.0 us, 14.3 without; 16384 x 4096 float32, four pieces of 256 lanes, 102 so and 98.9 without).
        constexpr bool kEarly = TEAM < 256 || (TEAM == 256 && CPL < 4);
        u32x4_t held[CPL], w[CPL], b[CPL];
        each_piece<CPL>([&](auto i, auto last) { held[i] = load_piece<DT, last>(a.x, row * a.ld, column(i), a.cols); });
        if (a.residual) {
            u32x4_t more[CPL];
            each_piece<CPL>([&](auto i, auto last) { more[i] = load_piece<DT, last>(a.residual, row * a.cols, column(i), a.cols); });
            if (kEarly && a.weight) each_piece<CPL>([&](auto i, auto last) { w[i] = load_piece<DT, last>(a.weight, 0, column(i), a.cols); });
            if (kEarly && a.bias) each_piece<CPL>([&](auto i, auto last) { b[i] = load_piece<DT, last>(a.bias, 0, column(i), a.cols); });
            each_piece<CPL>([&](auto i, auto) {
                float f[V], r[V];
                piece_values<DT>(held[i], f);
                piece_values<DT>(more[i], r);
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] += r[e];
                held[i] = values_piece<DT>(f);
            });
        } else {
            if (kEarly && a.weight) each_piece<CPL>([&](auto i, auto last) { w[i] = load_piece<DT, last>(a.weight, 0, column(i), a.cols); });
            if (kEarly && a.bias) each_piece<CPL>([&](auto i, auto last) { b[i] = load_piece<DT, last>(a.bias, 0, column(i), a.cols); });
        }
        double total = 0.0;
        each_piece<CPL>([&](auto i, auto last) {
            held[i] = whole_piece<DT, last, RAGGED>(held[i], column(i), a.cols);
            float f[V];
            piece_values<DT>(held[i], f);
#pragma unroll
            for (int e = 0; e < V; ++e) total += static_cast<double>(f[e]);
        });
        if (a.sum && here) each_piece<CPL>([&](auto i, auto last) { store_piece_of<DT, last, RAGGED>(a.sum, row * a.cols, column(i), a.cols, held[i]); });
        const float mean = static_cast<float>(column_mean(team_sum<TEAM>(total, space.first), a.cols, a.each));
        double squares = 0.0;
        each_piece<CPL>([&](auto i, auto last) {
            if (last && column(i) >= a.cols) return;
            float f[V];
            piece_values<DT>(held[i], f);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const double d = static_cast<double>(!(last && RAGGED) || column(i) + e < a.cols ? f[e] - mean : 0.0f);
                squares = fma(d, d, squares);
            }
        });
        const float rstd = inverse_deviation(team_sum<TEAM>(squares, space.second), a.cols, a.each, a.eps);
        if (a.mean && here && lane == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
        each_piece<CPL>([&](auto i, auto last) {
            float f[V], more[V];
            piece_values<DT>(held[i], f);
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = (f[e] - mean) * rstd;
            if (a.weight) {
                if (!kEarly) w[i] = load_piece<DT, last>(a.weight, 0, column(i), a.cols);
                piece_values<DT>(whole_piece<DT, last, RAGGED>(w[i], column(i), a.cols), more);
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] = f[e] * more[e];
            }
            if (a.bias) {
                if (!kEarly) b[i] = load_piece<DT, last>(a.bias, 0, column(i), a.cols);
                piece_values<DT>(whole_piece<DT, last, RAGGED>(b[i], column(i), a.cols), more);
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] = f[e] + more[e];
            }
            if constexpr (last) {                        // zeros behind the row's end: codes' rows have them, and they are no maximum
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] = column(i) + (RAGGED ? e : 0) < a.cols ? f[e] : 0.0f;
            }
            held[i] = values_piece<DT>(f);
            if (a.y && here) store_piece_of<DT, last, RAGGED>(a.y, row * a.cols, column(i), a.cols, held[i]);
        });
        if (a.codes) {
            uint32_t top = 0;
            each_piece<CPL>([&](auto i, auto) {
                float f[V];
                piece_values<DT>(held[i], f);
#pragma unroll
                for (int e = 0; e < V; ++e) top = max(top, magnitude_bits(f[e]));
            });
            const CodeScale s = code_scale(team_top<TEAM>(top, space.top));
            if (here) {
                if (lane == 0) a.scales[row] = s.scale;
                int8_t* const to = a.codes + row * a.code_stride;
                each_piece<CPL>([&](auto i, auto last) {
                    if (!last || column(i) < a.code_stride) store_codes<DT>(to + column(i), held[i], s.inv);
                });
            }
        }
        if constexpr (TEAM > kWave) __syncthreads();      // the words of `space` are free again
    }
}

// Rows wider than a workgroup holds in registers: read again for each sum and for the result, from the caches as far as those go.
// A lane always comes back to its own columns, so that sum and y may lie where x or the residual do.
constexpr int kWideLanes = 1024;

template <int DT>
__global__ __launch_bounds__(kWideLanes) void layernorm_wide_kernel(const LayernormArgs a) {
    constexpr int V = kPiece<DT>;
    __shared__ TeamSpace space;
    const int32_t begin = threadIdx.x * V, step = kWideLanes * V;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t at = row * a.cols;
        const auto piece = [&](const void* base, int64_t from, int32_t c) { return whole_piece<DT, true, true>(load_piece<DT, true>(base, from, c, a.cols), c, a.cols); };
        const auto values = [&](int32_t c, float (&f)[V]) {              // as they are stored
            piece_values<DT>(piece(a.x, row * a.ld, c), f);
            if (!a.residual) return;
            float r[V];
            piece_values<DT>(piece(a.residual, at, c), r);
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] += r[e];
            piece_values<DT>(values_piece<DT>(f), f);
        };
        const auto again = [&](int32_t c, float (&f)[V]) {
            if (a.sum) piece_values<DT>(piece(a.sum, at, c), f);
            else values(c, f);
        };
        double total = 0.0, squares = 0.0;
        for (int32_t c = begin; c < a.cols; c += step) {
            float f[V];
            values(c, f);
            if (a.sum) store_piece_of<DT, true, true>(a.sum, at, c, a.cols, values_piece<DT>(f));
#pragma unroll
            for (int e = 0; e < V; ++e) total += static_cast<double>(f[e]);
        }
        const float mean = static_cast<float>(column_mean(team_sum<kWideLanes>(total, space.first), a.cols, a.each));
        for (int32_t c = begin; c < a.cols; c += step) {
            float f[V];
            again(c, f);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const double d = static_cast<double>(c + e < a.cols ? f[e] - mean : 0.0f);
                squares = fma(d, d, squares);
            }
        }
        const float rstd = inverse_deviation(team_sum<kWideLanes>(squares, space.second), a.cols, a.each, a.eps);
        if (a.mean && threadIdx.x == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
        const auto result = [&](int32_t c) {
            float f[V], more[V];
            again(c, f);
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = (f[e] - mean) * rstd;
            if (a.weight) {
                piece_values<DT>(piece(a.weight, 0, c), more);
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] = f[e] * more[e];
            }
            if (a.bias) {
                piece_values<DT>(piece(a.bias, 0, c), more);
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] = f[e] + more[e];
            }
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = c + e < a.cols ? f[e] : 0.0f;
            return values_piece<DT>(f);
        };
        CodeScale s = {};
        if (a.codes) {                                    // before y is stored: it may be what `again` reads
            uint32_t top = 0;
            for (int32_t c = begin; c < a.cols; c += step) {
                float f[V];
                piece_values<DT>(result(c), f);
#pragma unroll
                for (int e = 0; e < V; ++e) top = max(top, magnitude_bits(f[e]));
            }
            s = code_scale(team_top<kWideLanes>(top, space.top));
            if (threadIdx.x == 0) a.scales[row] = s.scale;
        }
        const int32_t end = a.codes ? static_cast<int32_t>(a.code_stride) : a.cols;
        if (a.codes || a.y) {
            for (int32_t c = begin; c < end; c += step) {
                const u32x4_t y = c < a.cols ? result(c) : u32x4_t{0, 0, 0, 0};
                if (a.codes) store_codes<DT>(a.codes + row * a.code_stride + c, y, s.inv);
                if (a.y) store_piece_of<DT, true, true>(a.y, at, c, a.cols, y);
            }
        }
        __syncthreads();
    }
}

// Rows narrower than a piece: a wave to a row, a lane to an element.
template <int DT>
__global__ __launch_bounds__(256) void layernorm_narrow_kernel(const LayernormArgs a) {
    const int lane = threadIdx.x % kWave;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / kWave; row < a.rows; row += static_cast<int64_t>(gridDim.x) * 4) {
        const int64_t at = row * a.cols;
        const bool exists = lane < a.cols;
        float f = 0.0f;
        if (exists) {
            f = load_elem<DT>(a.x, row * a.ld + lane);
            if (a.residual) f = rounded_to<DT>(f + load_elem<DT>(a.residual, at + lane));
            if (a.sum) store_elem<DT>(a.sum, at + lane, f);
        }
        const float mean = static_cast<float>(column_mean(lanes_sum<kWave>(static_cast<double>(f)), a.cols, a.each));
        const double d = static_cast<double>(exists ? f - mean : 0.0f);
        const float rstd = inverse_deviation(lanes_sum<kWave>(d * d), a.cols, a.each, a.eps);
        if (a.mean && lane == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
        float y = (f - mean) * rstd;
        if (exists && a.weight) y = y * load_elem<DT>(a.weight, lane);
        if (exists && a.bias) y = y + load_elem<DT>(a.bias, lane);
        y = exists ? rounded_to<DT>(y) : 0.0f;
        if (a.y && exists) store_elem<DT>(a.y, at + lane, y);
        if (a.codes) {
            const CodeScale s = code_scale(__float_as_uint(team_max<kWave>(__uint_as_float(magnitude_bits(y)))));
            if (lane == 0) a.scales[row] = s.scale;
            a.codes[row * a.code_stride + lane] = static_cast<int8_t>(code_of<AQSGD_ROUND_NEAREST>(y, s.inv, 0.5f));      // a stride of 64
        }
    }
}

// ---- backward ----------------------------------------------------------------------------------
// Three ways.  Many rows: a workgroup takes many and keeps the columns' sums of them, which a second launch joins.  Few rows,
// or rows wider than a workgroup has lanes: the columns' sums by workgroups of their own, which read dy and x a second time.
// Rows narrower than a piece: the same, element by element.
enum GradWay { kGradBlocks, kGradColumns, kGradNarrow };

constexpr int kGradLanes = 1024;          // of a workgroup that takes many rows
constexpr int kGradBlocksMost = 256;      // workgroups that take many rows: one to a CU

// The workspace of the first way: sums of blocks of rows, for the weight [blocks, cols] and for the bias [blocks, cols].
struct GradPlan {
    GradWay way;
    int team;                             // lanes to a row
    int64_t blocks;                       // workgroups, and sums of each column
};

// Up to how many rows the columns go by workgroups of their own.  By blocks costs the join's launch, 4 us; by columns the second read,
// which grows with the rows and is shared by a workgroup for every 32 to 128 bytes of a row.  So the limit is where the read has
// become the longer one: lower for 65 to 128 pieces, whose 17 to 32 workgroups take 64 bytes of every row each, and higher for wide 16-bit rows, which have more
// than 64 of them and go one at a time through a workgroup of the blocks.  It is fitted (us, by blocks and by columns): 1024 x 1600 float16 10.7 and 7.3, 1400 x 1600 11.2 and 9.3, 2048 x 1600 11.7 and 12.7; 1280 x 400
// 6.8 and 5.8, 2048 x 400 7.2 and 8.5; 1100 x 768 bfloat16 7.3 and 7.8; 1400 x 4096 float32 23.8 and 22.6, 2048 x 4096 32.2 and 32.9; 2048 x 5120
// bfloat16 30.0 and 25.3, 2048 x 8192 43.9 and 33.2, 6000 x 8192 86 and 94; and misses 1280 x 768 float32, 9.0 and 9.4, and 3000 x 8192
// bfloat16, 54 and 49.  Without sums rows alone are left, which blocks would only hold up.
template <int DT>
inline int64_t most_rows_by_columns(int64_t pieces) {
    return DT != AQSGD_F32 && pieces > kGradLanes / 2 ? 2048 : pieces > 64 && pieces <= 128 ? 1024 : 1408;
}

template <int DT>
inline GradPlan grad_plan(int64_t rows, int64_t cols, bool sums) {
    const int64_t pieces = (cols + kPiece<DT> - 1) / kPiece<DT>;
    GradPlan p = {kGradNarrow, 0, 0};
    if (cols < kPiece<DT>) return p;
    p.way = kGradColumns;
    if (!sums || rows <= most_rows_by_columns<DT>(pieces) || pieces > kGradLanes) return p;
    p.way = kGradBlocks;
    p.team = 16;
    while (p.team < pieces) p.team *= 2;
    const int64_t teams = kGradLanes / p.team, want = (rows + teams - 1) / teams;
    p.blocks = want < kGradBlocksMost ? want : kGradBlocksMost;
    return p;
}

// Two sums over a team.
template <int TEAM>
__device__ __forceinline__ void team_sums(float& a, float& b, float2* part) {
    a = lanes_sum<(TEAM < kWave ? TEAM : kWave)>(a);
    b = lanes_sum<(TEAM < kWave ? TEAM : kWave)>(b);
    if constexpr (TEAM > kWave) {
        if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = float2{a, b};
        __syncthreads();
        const float2* of = part + threadIdx.x / TEAM * (TEAM / kWave);
        a = of[0].x;
        b = of[0].y;
#pragma unroll
        for (int w = 1; w < TEAM / kWave; ++w) {
            a += of[w].x;
            b += of[w].y;
        }
    }
}

// A row of what the gradient reads, on its way.
template <int DT, int TEAM, int CPL>
struct GradRow {
    u32x4_t x[CPL], dy[CPL], more[CPL];
    float mean, rstd;

    __device__ __forceinline__ void ask(const LayernormGradArgs& a, int64_t row, int lane) {
        mean = a.mean[row];
        rstd = a.rstd[row];
        each_piece<CPL>([&](auto i, auto last) { x[i] = load_piece<DT, last>(a.x, row * a.ld, (i * TEAM + lane) * kPiece<DT>, a.cols); });
        each_piece<CPL>([&](auto i, auto last) { dy[i] = load_piece<DT, last>(a.dy, row * a.cols, (i * TEAM + lane) * kPiece<DT>, a.cols); });
        if (a.add) each_piece<CPL>([&](auto i, auto last) { more[i] = load_piece<DT, last>(a.add, row * a.cols, (i * TEAM + lane) * kPiece<DT>, a.cols); });
    }
};

// A workgroup takes every blocks-th set of rows, a piece a lane, asks for the next one before it computes one, and keeps the
// columns' sums in registers to its end.
template <int DT, int TEAM, bool RAGGED>
__global__ __launch_bounds__(kGradLanes) void layernorm_grad_kernel(const LayernormGradArgs a, const int64_t blocks) {
    constexpr int kTeams = kGradLanes / TEAM, V = kPiece<DT>;
    __shared__ float2 part[2][kGradLanes / kWave];
    __shared__ float joined[kTeams > 1 ? kTeams : 1][kTeams > 1 ? TEAM * V : 1];
    const int lane = threadIdx.x % TEAM, team = team_number<TEAM>();
    const int32_t c = lane * V;
    float dw[V] = {}, db[V] = {}, w[V];
    const int64_t stride = blocks * kTeams;
    const auto row_of = [&](int64_t first) { return min(first + team, a.rows - 1); };
    int64_t first = static_cast<int64_t>(blockIdx.x) * kTeams;
    GradRow<DT, TEAM, 1> now, next;
    now.ask(a, row_of(first), lane);
    if (a.weight) {
        piece_values<DT>(whole_piece<DT, true, RAGGED>(load_piece<DT, true>(a.weight, 0, c, a.cols), c, a.cols), w);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = 1.0f;
    }
    const float each = 1.0f / static_cast<float>(a.cols);
    int turn = 0;
    for (; first < a.rows; first += stride, turn ^= 1) {
        const bool here = first + team < a.rows, more = first + stride < a.rows;
        const int64_t row = row_of(first);
        if (more) next.ask(a, row_of(first + stride), lane);
        // Where there is no column or no row dy is 0, and with it whatever is summed: xh is then that of another of the row's
        // elements, or of the last row's, so it is finite unless that row's own sums are NaN anyway.
        float along = 0.0f, across = 0.0f, g[V], xh[V], gw[V];
        piece_values<DT>(placed_piece<DT, true, RAGGED>(now.x[0], c, a.cols), xh);
        piece_values<DT>(here ? whole_piece<DT, true, RAGGED>(now.dy[0], c, a.cols) : u32x4_t{0, 0, 0, 0}, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            xh[e] = (xh[e] - now.mean) * now.rstd;
            gw[e] = g[e] * w[e];
            along += gw[e];
            across = fmaf(gw[e], xh[e], across);
            dw[e] = fmaf(g[e], xh[e], dw[e]);
            db[e] += g[e];
        }
        team_sums<TEAM>(along, across, part[turn]);
        along *= each;
        across *= each;
        float out[V] = {};
        if (a.add) piece_values<DT>(whole_piece<DT, true, RAGGED>(now.more[0], c, a.cols), out);
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = fmaf(now.rstd, fmaf(-xh[e], across, gw[e] - along), out[e]);
        if (here) store_piece_of<DT, true, RAGGED>(a.dx, row * a.cols, c, a.cols, values_piece<DT>(out));
        if (more) now = next;
    }
    float* to = a.workspace + static_cast<int64_t>(blockIdx.x) * a.cols;
    const auto leave = [&](const float (&sums)[V], float* at) {
        if constexpr (kTeams > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e) joined[team][lane * V + e] = sums[e];
            __syncthreads();
            for (int k = threadIdx.x; k < TEAM * V; k += kGradLanes) {
                float s = joined[0][k];
#pragma unroll
                for (int t = 1; t < kTeams; ++t) s += joined[t][k];
                if (k < a.cols) at[k] = s;
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (c + e < a.cols) at[c + e] = sums[e];
        }
    };
    if (a.dweight) leave(dw, to);
    if (a.dbias) leave(db, to + blocks * a.cols);
}

// The second way in one launch: the first workgroups take the columns, PIECES of every row, the others the rows; neither needs
// the other's sums.  Where dx is dy itself the columns go first, in a launch of their own.
constexpr int kFewLanes = 512;

template <int DT, int PIECES, bool RAGGED>
__device__ __forceinline__ void columns_of_few(const LayernormGradArgs& a, int64_t block) {
    constexpr int V = kPiece<DT>, kCols = PIECES * V, kGroups = kFewLanes / kCols, kFewSlots = kFewLanes / PIECES, kAhead = 4;
    __shared__ float part[2][kFewSlots][kCols + 1];
    __shared__ float last[2][kGroups][kCols + 1];
    const int slot = threadIdx.x / PIECES, across = threadIdx.x % PIECES;
    const int32_t c = static_cast<int32_t>(block * kCols) + across * V;
    float dw[V] = {}, db[V] = {};
    for (int64_t first = slot; first < a.rows; first += kFewSlots * kAhead) {
        u32x4_t x[kAhead], dy[kAhead];
        float mean[kAhead], rstd[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t row = min(first + i * kFewSlots, a.rows - 1);
            x[i] = load_piece<DT, true>(a.x, row * a.ld, c, a.cols);
            dy[i] = load_piece<DT, true>(a.dy, row * a.cols, c, a.cols);
            mean[i] = a.mean[row];
            rstd[i] = a.rstd[row];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (first + i * kFewSlots >= a.rows) break;
            float xf[V], g[V];
            piece_values<DT>(placed_piece<DT, true, RAGGED>(x[i], c, a.cols), xf);
            piece_values<DT>(whole_piece<DT, true, RAGGED>(dy[i], c, a.cols), g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                dw[e] = fmaf(g[e], (xf[e] - mean[i]) * rstd[i], dw[e]);
                db[e] += g[e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        part[0][slot][across * V + e] = dw[e];
        part[1][slot][across * V + e] = db[e];
    }
    __syncthreads();
    const int col = threadIdx.x % kCols, group = threadIdx.x / kCols;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kFewSlots / kGroups; ++i) sum += part[k][group * (kFewSlots / kGroups) + i][col];
        last[k][group][col] = sum;
    }
    __syncthreads();
    const int64_t at = block * kCols + col;
    float* out = group == 0 ? a.dweight : group == 1 ? a.dbias : nullptr;
    if (!out || at >= a.cols) return;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) sum += last[group][i][col];
    out[at] = a.accumulate ? out[at] + sum : sum;
}

template <int DT, int TEAM, int CPL, int PIECES, bool RAGGED>
__global__ __launch_bounds__(kFewLanes) void layernorm_grad_few_kernel(const LayernormGradArgs a, const uint32_t column_blocks) {
    if (blockIdx.x < column_blocks) {
        columns_of_few<DT, PIECES, RAGGED>(a, blockIdx.x);
        return;
    }
    constexpr int kTeams = kFewLanes / TEAM, V = kPiece<DT>;
    __shared__ float2 part[2][kFewLanes / kWave];
    const int lane = threadIdx.x % TEAM, team = team_number<TEAM>();
    const auto column = [&](int i) { return (i * TEAM + lane) * V; };
    const float each = 1.0f / static_cast<float>(a.cols);
    const int64_t stride = static_cast<int64_t>(gridDim.x - column_blocks) * kTeams;
    int turn = 0;
    // A team of one wave goes by its own rows and waits for nobody.  Of several waves, all go on to team_sums' barrier, a team without a row
    // with the last one again: what it reads there, dx perhaps over dy by then, is not used.
    constexpr bool kAlone = TEAM <= kWave;
    for (int64_t first = static_cast<int64_t>(blockIdx.x - column_blocks) * kTeams + (kAlone ? team : 0); first < a.rows; first += stride, turn ^= 1) {
        const bool here = kAlone || first + team < a.rows;
        const int64_t row = kAlone ? first : here ? first + team : a.rows - 1;
        GradRow<DT, TEAM, CPL> now;
        now.ask(a, row, lane);
        u32x4_t w[CPL];
        if (a.weight) each_piece<CPL>([&](auto i, auto last) { w[i] = load_piece<DT, last>(a.weight, 0, column(i), a.cols); });
        float along = 0.0f, across = 0.0f, xh[CPL][V], gw[CPL][V];
        each_piece<CPL>([&](auto i, auto last) {
            piece_values<DT>(placed_piece<DT, last, RAGGED>(now.x[i], column(i), a.cols), xh[i]);
            piece_values<DT>(whole_piece<DT, last, RAGGED>(now.dy[i], column(i), a.cols), gw[i]);
            if (a.weight) {
                float wf[V];
                piece_values<DT>(whole_piece<DT, last, RAGGED>(w[i], column(i), a.cols), wf);
#pragma unroll
                for (int e = 0; e < V; ++e) gw[i][e] *= wf[e];
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                xh[i][e] = (xh[i][e] - now.mean) * now.rstd;
                along += gw[i][e];
                across = fmaf(gw[i][e], xh[i][e], across);
            }
        });
        team_sums<TEAM>(along, across, part[turn]);
        along *= each;
        across *= each;
        each_piece<CPL>([&](auto i, auto last) {
            float out[V] = {};
            if (a.add) piece_values<DT>(whole_piece<DT, last, RAGGED>(now.more[i], column(i), a.cols), out);
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = fmaf(now.rstd, fmaf(-xh[i][e], across, gw[i][e] - along), out[e]);
            if (here) store_piece_of<DT, last, RAGGED>(a.dx, row * a.cols, column(i), a.cols, values_piece<DT>(out));
        });
    }
}

// Rows wider than a workgroup holds in registers: read once for the sums and once for dx.
template <int DT>
__global__ __launch_bounds__(kWideLanes) void layernorm_grad_wide_kernel(const LayernormGradArgs a) {
    constexpr int V = kPiece<DT>;
    __shared__ float2 part[2][kWideLanes / kWave];
    const int32_t begin = threadIdx.x * V, step = kWideLanes * V;
    const float each = 1.0f / static_cast<float>(a.cols);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const int64_t at = row * a.cols;
        const float mean = a.mean[row], rstd = a.rstd[row];
        const auto piece = [&](const void* base, int64_t from, int32_t c) { return whole_piece<DT, true, true>(load_piece<DT, true>(base, from, c, a.cols), c, a.cols); };
        const auto read = [&](int32_t c, float (&xh)[V], float (&gw)[V]) {
            piece_values<DT>(placed_piece<DT, true, true>(load_piece<DT, true>(a.x, row * a.ld, c, a.cols), c, a.cols), xh);
            piece_values<DT>(piece(a.dy, at, c), gw);
            if (a.weight) {
                float w[V];
                piece_values<DT>(piece(a.weight, 0, c), w);
#pragma unroll
                for (int e = 0; e < V; ++e) gw[e] *= w[e];
            }
#pragma unroll
            for (int e = 0; e < V; ++e) xh[e] = (xh[e] - mean) * rstd;
        };
        float along = 0.0f, across = 0.0f;
        for (int32_t c = begin; c < a.cols; c += step) {
            float xh[V], gw[V];
            read(c, xh, gw);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                along += gw[e];
                across = fmaf(gw[e], xh[e], across);
            }
        }
        team_sums<kWideLanes>(along, across, part[turn]);
        along *= each;
        across *= each;
        for (int32_t c = begin; c < a.cols; c += step) {
            float xh[V], gw[V], out[V] = {};
            read(c, xh, gw);
            if (a.add) piece_values<DT>(piece(a.add, at, c), out);
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = fmaf(rstd, fmaf(-xh[e], across, gw[e] - along), out[e]);
            store_piece_of<DT, true, true>(a.dx, at, c, a.cols, values_piece<DT>(out));
        }
    }
}

// Rows narrower than a piece.  The columns' sums, in binary64 for a lane adds as many rows as there are: a workgroup to a column.
template <int DT>
__global__ __launch_bounds__(kWideLanes) void layernorm_grad_narrow_columns_kernel(const LayernormGradArgs a) {
    __shared__ double part[2][kWideLanes / kWave];
    const int32_t c = blockIdx.x;
    double dw = 0.0, db = 0.0;
#pragma unroll 4
    for (int64_t row = threadIdx.x; row < a.rows; row += kWideLanes) {
        const float g = load_elem<DT>(a.dy, row * a.cols + c);
        dw += static_cast<double>(g * ((load_elem<DT>(a.x, row * a.ld + c) - a.mean[row]) * a.rstd[row]));
        db += static_cast<double>(g);
    }
    dw = team_sum<kWideLanes>(dw, part[0]);
    db = team_sum<kWideLanes>(db, part[1]);
    if (threadIdx.x != 0) return;
    if (a.dweight) a.dweight[c] = a.accumulate ? a.dweight[c] + static_cast<float>(dw) : static_cast<float>(dw);
    if (a.dbias) a.dbias[c] = a.accumulate ? a.dbias[c] + static_cast<float>(db) : static_cast<float>(db);
}

// A wave to a row, a lane to an element.
template <int DT>
__global__ __launch_bounds__(256) void layernorm_grad_narrow_kernel(const LayernormGradArgs a) {
    const int lane = threadIdx.x % kWave;
    const float each = 1.0f / static_cast<float>(a.cols);
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / kWave; row < a.rows; row += static_cast<int64_t>(gridDim.x) * 4) {
        const int64_t at = row * a.cols + lane;
        const bool exists = lane < a.cols;
        float xh = 0.0f, gw = 0.0f;
        if (exists) {
            xh = (load_elem<DT>(a.x, row * a.ld + lane) - a.mean[row]) * a.rstd[row];
            gw = load_elem<DT>(a.dy, at);
            if (a.weight) gw *= load_elem<DT>(a.weight, lane);
        }
        const float along = lanes_sum<kWave>(gw) * each, across = lanes_sum<kWave>(gw * xh) * each;
        if (!exists) continue;
        const float more = a.add ? load_elem<DT>(a.add, at) : 0.0f;
        store_elem<DT>(a.dx, at, fmaf(a.rstd[row], fmaf(-xh, across, gw - along), more));
    }
}

// ---- launches ----------------------------------------------------------------------------------
template <int DT>
hipError_t launch_layernorm_as(const LayernormArgs& a, hipStream_t stream) {
    const auto go = [&](void (*kernel)(const LayernormArgs), int team) {
        const int threads = team < 256 ? 256 : team;
        const int64_t per = threads / team, blocks = (a.rows + per - 1) / per, most = (int64_t{1} << 30) / threads;
        return launch_kernel(kernel, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), dim3(static_cast<unsigned>(threads)), stream, a);
    };
    const int64_t pieces = (a.cols + kPiece<DT> - 1) / kPiece<DT>;
    // Few rows of three or four pieces a lane are better shared by four waves: 256 rows of 1600 float16 3.7 us, with a wave to a row
    // 4.4; 512 rows 4.3 and 4.7, 1024 rows 6.0 and 5.1.
    const bool ragged = a.cols % kPiece<DT> != 0, few = a.rows <= 512;
#define AQSGD_NORM(TEAM, CPL) \
    return ragged ? go(layernorm_kernel<DT, TEAM, CPL, true>, TEAM) : go(layernorm_kernel<DT, TEAM, CPL, false>, TEAM)
    if (a.cols < kPiece<DT>) return go(layernorm_narrow_kernel<DT>, kWave);
    // Many narrow rows: few lanes with several pieces each, so that a wave's sums and statistics serve several rows.  32768 rows (us; with a
    // piece or two a lane in brackets): 130 float16 6.9 (10.7), 300 bfloat16 11.0 (17.7), 768 float16 17.8 (23.2), 129 float32 9.0 (13.9);
    // 4096 rows: 3.2 (3.6), 3.5 (4.5), 4.1 (4.7), 2.9 (3.9); 1024 rows: 3.1 (3.1), 3.1 (3.1), 3.1 (2.9), 2.7 (2.9).
    if (a.rows >= 4096) {
        if constexpr (DT != AQSGD_F32) {
            if (pieces <= 8) AQSGD_NORM(8, 1);
            if (pieces <= 16) AQSGD_NORM(8, 2);
            if (pieces <= 24) AQSGD_NORM(8, 3);
            if (pieces <= 32) AQSGD_NORM(8, 4);
        } else {
            if (pieces <= 16) AQSGD_NORM(16, 1);
            if (pieces <= 32) AQSGD_NORM(16, 2);
        }
        if (pieces <= 48) AQSGD_NORM(16, 3);
        if (pieces <= 64) AQSGD_NORM(16, 4);
        if (pieces <= 96) AQSGD_NORM(32, 3);
        if (pieces <= 128) AQSGD_NORM(32, 4);
    }
    if (pieces <= 16) AQSGD_NORM(16, 1);
    if (pieces <= 32) AQSGD_NORM(32, 1);
    if (pieces <= 64) AQSGD_NORM(64, 1);
    if (pieces <= 128) AQSGD_NORM(64, 2);
    if (pieces <= 256 && few) AQSGD_NORM(256, 1);
    if (pieces <= 192) AQSGD_NORM(64, 3);
    if (pieces <= 256) AQSGD_NORM(64, 4);
    if (pieces <= 512) AQSGD_NORM(256, 2);
    if (pieces <= 768) AQSGD_NORM(256, 3);
    if (pieces <= 1024) AQSGD_NORM(256, 4);
    // Rows of 16384 bfloat16: 2048 of them 29.9 us, by 1024 lanes 36.3; 16 rows 4.9 and 4.5, 256 rows 5.9 and 5.7.
    if (pieces <= 2048 && a.rows <= 256) AQSGD_NORM(1024, 2);
    if (pieces <= 1536) AQSGD_NORM(512, 3);
    if (pieces <= 2048) AQSGD_NORM(512, 4);
    if (pieces <= 3 * 1024) AQSGD_NORM(1024, 3);
    if (pieces <= 4096) AQSGD_NORM(1024, 4);
#undef AQSGD_NORM
    return go(layernorm_wide_kernel<DT>, kWideLanes);
}

hipError_t launch_layernorm_join(const LayernormGradArgs& a, int64_t blocks, hipStream_t stream);

// The columns' launch, if the sums are asked for, and the rows' behind it.
template <typename C, typename R>
hipError_t launch_columns_and_rows(bool sums, C&& columns, R&& rows) {
    std::optional<ProfileSpan> span;
    if (sums) {
        span.emplace();
        const hipError_t err = columns();
        if (err != hipSuccess) return err;
        span->last();
    }
    return rows();
}

template <int DT>
hipError_t launch_layernorm_grad_columns(const LayernormGradArgs& a, hipStream_t stream) {
    const int64_t pieces = (a.cols + kPiece<DT> - 1) / kPiece<DT>;
    const bool ragged = a.cols % kPiece<DT> != 0, sums = a.dweight || a.dbias;
    const int64_t most = int64_t{1} << 21;                                     // workgroups of up to 1024 lanes
    const auto column_blocks = [&](int each) { return sums ? static_cast<uint32_t>((pieces + each - 1) / each) : 0; };
    const auto launch = [&](void (*kernel)(const LayernormGradArgs, const uint32_t), int64_t blocks, uint32_t columns) {
        return launch_kernel(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kFewLanes), stream, a, columns);
    };
    const auto go = [&](void (*kernel)(const LayernormGradArgs, const uint32_t), int team, int each) {
        const int64_t per = kFewLanes / team, want = (a.rows + per - 1) / per, rows = want < most ? want : most;
        const uint32_t columns = column_blocks(each);
        if (a.dx != a.dy) return launch(kernel, columns + rows, columns);
        return launch_columns_and_rows(sums, [&] { return launch(kernel, columns, columns); }, [&] { return launch(kernel, rows, 0); });
    };
#define AQSGD_NORM(TEAM, CPL, PIECES) \
    if (pieces <= TEAM * CPL) \
        return ragged ? go(layernorm_grad_few_kernel<DT, TEAM, CPL, PIECES, true>, TEAM, PIECES) \
                      : go(layernorm_grad_few_kernel<DT, TEAM, CPL, PIECES, false>, TEAM, PIECES);
    // Few rows go by four waves each where one would take several pieces a lane: 8 rows of 1600 float16 2.6 us, by a wave 3.8; 256 rows
    // 3.1 and 4.1, 512 rows 4.6 and 4.5, 4096 rows without sums 8.6 and 7.6.
    if (a.rows <= 256 && pieces > 64) AQSGD_NORM(256, 1, 4)
    // Columns: 64 bytes of a row to a workgroup, 128 where that still makes 100 workgroups, 32 where the rows are many and their
    // columns' workgroups would be the last to end.  2, 4 and 8 pieces (us): 1000 x 200 float16 3.7, 4.5, 6.5; 1024 x 1600 7.6, 7.4, 10.0;
    // 1000 x 6144 bfloat16 23.4, 15.4, 16.0; 1024 x 4096 float32 31.7, 19.5, 17.0; 2048 x 8192 float32 122, 80, 62.
    if (a.rows > 256) AQSGD_NORM(64, 1, 2)
    AQSGD_NORM(64, 1, 4) AQSGD_NORM(64, 2, 4) AQSGD_NORM(64, 3, 4) AQSGD_NORM(64, 4, 4) AQSGD_NORM(512, 1, 4)
    if (pieces < 800) AQSGD_NORM(512, 2, 4)
    AQSGD_NORM(512, 2, 8) AQSGD_NORM(512, 3, 8) AQSGD_NORM(512, 4, 8)
    if constexpr (DT == AQSGD_F32) AQSGD_NORM(512, 8, 8)
#undef AQSGD_NORM
    const auto few = ragged ? layernorm_grad_few_kernel<DT, 64, 1, 8, true> : layernorm_grad_few_kernel<DT, 64, 1, 8, false>;      // its columns alone
    return launch_columns_and_rows(sums, [&] { const uint32_t columns = column_blocks(8); return launch(few, columns, columns); },
                                   [&] { return launch_kernel(layernorm_grad_wide_kernel<DT>, dim3(static_cast<unsigned>(a.rows < most ? a.rows : most)), dim3(kWideLanes), stream, a); });
}

template <int DT>
hipError_t launch_layernorm_grad_blocks(const LayernormGradArgs& a, const GradPlan& p, hipStream_t stream) {
    const bool ragged = a.cols % kPiece<DT> != 0;
    ProfileSpan span;
    const auto go = [&](void (*kernel)(const LayernormGradArgs, const int64_t)) {
        return launch_kernel(kernel, dim3(static_cast<unsigned>(p.blocks)), dim3(kGradLanes), stream, a, p.blocks);
    };
    hipError_t err = hipErrorInvalidValue;
#define AQSGD_NORM(TEAM) \
    if (p.team == TEAM) err = ragged ? go(layernorm_grad_kernel<DT, TEAM, true>) : go(layernorm_grad_kernel<DT, TEAM, false>);
    AQSGD_NORM(16) AQSGD_NORM(32) AQSGD_NORM(64) AQSGD_NORM(128) AQSGD_NORM(256) AQSGD_NORM(512) AQSGD_NORM(1024)
#undef AQSGD_NORM
    if (err != hipSuccess) return err;
    span.last();
    return launch_layernorm_join(a, p.blocks, stream);
}

template <int DT>
hipError_t launch_layernorm_grad_narrow(const LayernormGradArgs& a, hipStream_t stream) {
    const int64_t blocks = (a.rows + 3) / 4, most = int64_t{1} << 20;
    return launch_columns_and_rows(a.dweight || a.dbias,
                                   [&] { return launch_kernel(layernorm_grad_narrow_columns_kernel<DT>, dim3(static_cast<unsigned>(a.cols)), dim3(kWideLanes), stream, a); },
                                   [&] { return launch_kernel(layernorm_grad_narrow_kernel<DT>, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), dim3(256), stream, a); });
}

template <int DT>
hipError_t launch_layernorm_grad_as(const LayernormGradArgs& a, hipStream_t stream) {
    if (a.rows == 0) return launch_layernorm_join(a, 0, stream);
    const GradPlan p = grad_plan<DT>(a.rows, a.cols, a.dweight || a.dbias);
    switch (p.way) {
    case kGradBlocks:  return launch_layernorm_grad_blocks<DT>(a, p, stream);
    case kGradColumns: return launch_layernorm_grad_columns<DT>(a, stream);
    default:           return launch_layernorm_grad_narrow<DT>(a, stream);
    }
}

}  // namespace aqsgd
