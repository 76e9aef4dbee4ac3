// Kernels of aqsgd_adamw: one step of many tensors in one launch.
//
// Every element is read and written once, past the caches.  With states in 32 bits memory bounds the step: 30.7 M float16
// weights with binary32 copies and gradients 154 us, 6.0 TB/s.  In 8 bits what is moved halves and the arithmetic doubles (a root and a
// quotient for the step, two roots for the codes): 123 M such weights 362 us, 6.1 TB/s, with vector instructions in 90 % of the cycles, and
// 28.3 M bfloat16 ones without copies 75 us, 3.8 TB/s, or 84 with draws, where it is they that bound it (95 %).
//
// Lanes take four neighbouring elements at a time, so that binary32 accesses are contiguous.  With states in 8 bits half a wave
// takes a group in two such pieces: what a lane does once for its group (four quotients, two maxima over the lanes) is shared by eight
// elements (28.3 M bfloat16 weights 110 us with a wave to a group and four elements a lane, 77 so, before the next step).  Root and quotient
// by a step from the hardware's reciprocals, where a vote says that their ranges allow it: with draws 83 us, 87 by the compiler's quotient.
// Everything stays in registers between the loads and the stores.  A workgroup's tensor is found in the launch's table by one load and a
// vote of the wave.
#pragma once

#include "aqsgd_norms.h"

namespace aqsgd {

constexpr int kUpdateWaves = 4, kUpdatePieces = 2;                        // waves of a workgroup, pieces of four elements a lane
constexpr int64_t kUpdateSpan = int64_t{4} * kWave * kUpdateWaves * kUpdatePieces;      // elements of a workgroup
constexpr float kStateFloor = 0x1p-100f;                                  // a group below this is held as zeros: T^2 / s is finite from here on
constexpr float kMTop = 127.0f, kRTop = 255.0f;

// Where the parts of a tensor's state lie, in bytes.
__host__ __device__ inline int64_t whole64(int64_t bytes) { return (bytes + 63) / 64 * 64; }
__host__ __device__ inline int64_t state_groups(int64_t n) { return (n + kStateGroup - 1) / kStateGroup; }
__host__ __device__ inline int64_t state_bytes(int64_t n, int bits) {
    return bits == 32 ? 2 * whole64(4 * n) : 2 * whole64(n) + 2 * whole64(4 * state_groups(n));
}

typedef uint16_t u16x4_t __attribute__((ext_vector_type(4)));

// Four elements at any element's address, of which `count` exist (FULL: all four).
template <int DT, bool FULL>
__device__ __forceinline__ void load_four(const void* base, int64_t i, int count, float (&f)[4]) {
    if (FULL || count >= 4) {
        if constexpr (DT == AQSGD_F32) {
            const f32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const f32x4_any_t*>(static_cast<const float*>(base) + i));
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = v[e];
        } else {
            typedef uint16_t u16x4_at_t __attribute__((ext_vector_type(4), aligned(2)));
            const u16x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u16x4_at_t*>(static_cast<const uint16_t*>(base) + i));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                f[e] = DT == AQSGD_F16 ? static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(v[e]))) : bf16_bits_to_f32(v[e]);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = e < count ? load_elem<DT>(base, i + e) : 0.0f;
}

template <int DT, bool FULL>
__device__ __forceinline__ void store_four(void* base, int64_t i, int count, const float (&f)[4]) {
    if (FULL || count >= 4) {
        if constexpr (DT == AQSGD_F32) {
            __builtin_nontemporal_store(f32x4_t{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4_any_t*>(static_cast<float*>(base) + i));
        } else {
            typedef uint32_t u32x2_at_t __attribute__((ext_vector_type(2), aligned(2)));
            uint32_t lo, hi;
            if constexpr (DT == AQSGD_F16) {
                typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
                lo = __builtin_bit_cast(uint32_t, half2_t{static_cast<_Float16>(f[0]), static_cast<_Float16>(f[1])});
                hi = __builtin_bit_cast(uint32_t, half2_t{static_cast<_Float16>(f[2]), static_cast<_Float16>(f[3])});
            } else {
                lo = f32x2_to_bf16x2(f[0], f[1]);
                hi = f32x2_to_bf16x2(f[2], f[3]);
            }
            __builtin_nontemporal_store(u32x2_at_t{lo, hi}, reinterpret_cast<u32x2_at_t*>(static_cast<uint16_t*>(base) + i));
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < count) store_elem<DT>(base, i + e, f[e]);
}

// What all of a tensor's elements share.
struct UpdateFactors {
    float decay, length, correct;         // 1 - lr * weight_decay, lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    float scale;                          // 1 where there is none
};

// The moments of one element after this step.
__device__ __forceinline__ void step_moments(const AdamwArgs& a, const UpdateFactors& k, float g, float& m, float& v) {
    g = g * k.scale;
    m = m * a.beta1f + g * a.rest1;
    v = v * a.beta2f + (g * a.rest2) * g;
}

__device__ __forceinline__ float stepped_weight(const AdamwArgs& a, const UpdateFactors& k, float w, float m, float r) {
    return w * k.decay - (m / (r * k.correct + a.eps)) * k.length;
}

// The root of a v that is 0 or between 2^-96 and 2^127, rounded once: v times the hardware's reciprocal root is within two ulps, and
// one step by the residual, which is exact, ends at the right one (tried on every significand of twelve binades).
__device__ __forceinline__ float root_of(float v) {
    const float y = __builtin_amdgcn_rsqf(fmaxf(v, 0x1p-126f)), s = v * y;
    return fmaf(fmaf(-s, s, v), 0.5f * y, s);
}

// A quotient, rounded once, of an m that is 0 or between 2^-70 and 2^60 in magnitude by a d between 2^-48 and 2^50.  The reciprocal is the
// rounded one after a step (tried on every significand of d); from that, a residual without error, which these ranges grant, leads
// to the rounded quotient (Markstein's theorem).  The residual is formed the other way round so that a zero keeps its sign.
__device__ __forceinline__ float quotient_of(float m, float d) {
    const float y = __builtin_amdgcn_rcpf(d), inverse = fmaf(fmaf(-d, y, 1.0f), y, y), q = m * inverse;
    return fmaf(-fmaf(d, q, -m), inverse, q);
}

// ---- states in 8 bits ----------------------------------------------------------------------------
struct HeldScale {
    float scale;          // stored
    float inv;            // T^2 / scale, or 0
    bool live;
};

__device__ __forceinline__ HeldScale held_scale(uint32_t bits, float top) {
    const float s = __uint_as_float(bits);
    const bool finite = bits < 0x7f800000u;
    HeldScale h;
    h.live = finite && !(s < kStateFloor);
    h.scale = h.live ? s : finite ? 0.0f : __uint_as_float(0x7fc00000u);
    h.inv = h.live ? (top * top) / (h.live ? s : 1.0f) : 0.0f;
    return h;
}

// The code of one magnitude of a live group: the whole number below u's root, and one more where the distance says so.  The
// hardware's root may be off by an ulp, so that its whole part is one off where u is next to a square.  To the nearest that
// changes nothing: from either side the distance leads to the same neighbour.  Draws ask for the right one: the
// root is taken a little low, and raised where the next square is not above u (both checked on every u to 255^2, draws with the
// smallest and largest z).  No code passes T: u is at most T^2 (1 + 2^-23), nearer to T^2 than any threshold (z (2 T + 1), z at
// least 2^-16).  z is (word + 1) / 65536; its product with 2 k + 1 is one fused step.
template <int ROUND>
__device__ __forceinline__ float held_code(float x, float inv, float word) {
    const float u = x * inv;
    if constexpr (ROUND == AQSGD_ROUND_NEAREST) {
        const float k = floorf(__builtin_amdgcn_sqrtf(u));
        return fmaf(-k, k, u) >= k + 0.5f ? k + 1.0f : k;
    } else {
        float k = floorf(__builtin_amdgcn_sqrtf(u) * (1.0f - 0x1p-21f));
        const float next = k + 1.0f;
        k = next * next <= u ? next : k;
        const float width = fmaf(k, 0x1p-15f, 0x1p-16f);
        return fmaf(-k, k, u) >= fmaf(word, width, width) ? k + 1.0f : k;
    }
}

// The largest of 32 lanes, in all of them.
__device__ __forceinline__ uint32_t half_wave_max(uint32_t v) {
    v = dpp_max_step<0xB1>(v);
    v = dpp_max_step<0x4E>(v);
    v = dpp_max_step<0x141>(v);
    v = dpp_max_step<0x140>(v);
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return max(r[0], r[1]);
}

// A quotient by a constant, rounded once for every s whose quotient is a normal number (all 2^23 significands were tried, for
// 127^2 and 255^2).
template <int N>
__device__ __forceinline__ float divided_by(float s) {
    constexpr float inv = 1.0f / N;
    const float q = s * inv;
    return fmaf(fmaf(-static_cast<float>(N), q, s), inv, q);
}

// Half a wave's group, elements 4 l .. 4 l + 3 and 128 + 4 l .. of it a lane l.
template <int DT, int GT, int ROUND, bool FULL>
__device__ __forceinline__ void adamw8_group(const UpdateTensor& t, const AdamwArgs& a, const UpdateFactors& k, uint64_t key, int64_t group, int l) {
    const int64_t first = group * kStateGroup + l * 4;
    int count[2];
    float g[2][4], w[2][4], m[2][4], v[2][4], r[2][4];
    uint32_t mc[2], rc[2];
    char* const m_at = t.state + first;
    char* const r_at = m_at + whole64(t.n);
    float* const m_scale = reinterpret_cast<float*>(t.state + 2 * whole64(t.n)) + group;
    float* const r_scale = m_scale + whole64(4 * state_groups(t.n)) / 4;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int64_t i = first + 128 * p, left = t.n - i;
        count[p] = FULL || left >= 4 ? 4 : left > 0 ? static_cast<int>(left) : 0;
        load_four<GT, FULL>(t.grad, i, count[p], g[p]);
        if (t.master) load_four<AQSGD_F32, FULL>(t.master, i, count[p], w[p]);
        else load_four<DT, FULL>(t.param, i, count[p], w[p]);
        mc[p] = rc[p] = 0;
        if (FULL || count[p] > 0) {
            mc[p] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(m_at + 128 * p));
            rc[p] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(r_at + 128 * p));
        }
    }
    const float m_step = divided_by<127 * 127>(*m_scale), r_step = divided_by<255 * 255>(*r_scale);
    uint32_t m_least = 0xffffffffu, v_least = 0xffffffffu, m_top = 0, r_top = 0;      // patterns of magnitudes; of the smallest that is not 0, less one
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        mc[p] ^= 0x80808080u;                              // code + 128 as bytes
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float mk = static_cast<float>((mc[p] >> (8 * e)) & 0xffu) - 128.0f, rk = static_cast<float>((rc[p] >> (8 * e)) & 0xffu);
            const float root = (rk * rk) * r_step;
            m[p][e] = (mk * fabsf(mk)) * m_step;
            v[p][e] = root * root;
            step_moments(a, k, g[p][e], m[p][e], v[p][e]);
            if (!FULL && e >= count[p]) m[p][e] = v[p][e] = 0.0f;
            r[p][e] = root_of(v[p][e]);
            const uint32_t size = __float_as_uint(m[p][e]) & 0x7fffffffu;
            m_least = min(m_least, size - 1u);
            m_top = max(m_top, size);
            v_least = min(v_least, __float_as_uint(v[p][e]) - 1u);
            r_top = max(r_top, __float_as_uint(r[p][e]));  // not below 0; a NaN of either sign lies above all numbers
        }
    }
    // What root_of and quotient_of ask for holds of any usual step; d is eps or more, and "1 / sqrt(1 - beta2^t)" below 2^27.
    const bool usual = m_least >= 0x1c800000u - 1u && m_top < 0x5d800000u && v_least >= 0x0f800000u - 1u && r_top < 0x49800000u &&
                       a.eps >= 0x1p-48f && a.eps <= 0x1p48f;      // m 2^-70, 2^60; v 2^-96; r 2^20
    if (__all(usual)) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int e = 0; e < 4; ++e) w[p][e] = w[p][e] * k.decay - quotient_of(m[p][e], r[p][e] * k.correct + a.eps) * k.length;
    } else {
        r_top = 0;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                r[p][e] = sqrtf(v[p][e]);
                r_top = max(r_top, __float_as_uint(r[p][e]));
                w[p][e] = stepped_weight(a, k, w[p][e], m[p][e], r[p][e]);
            }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int64_t i = first + 128 * p;
        if (t.master) store_four<AQSGD_F32, FULL>(t.master, i, count[p], w[p]);
        store_four<DT, FULL>(t.param, i, count[p], w[p]);
    }
    const HeldScale ms = held_scale(half_wave_max(m_top), kMTop), rs = held_scale(half_wave_max(r_top), kRTop);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        float m_word[4], r_word[4];
        if constexpr (ROUND == AQSGD_ROUND_STOCHASTIC) {
            const uint64_t block = static_cast<uint64_t>(t.group0 + group) * (kStateGroup / 4) + static_cast<uint32_t>(32 * p + l);
            uint32_t words[4];
            philox4x32_10(static_cast<uint32_t>(block), static_cast<uint32_t>(block >> 32), static_cast<uint32_t>(key),
                          static_cast<uint32_t>(key >> 32), words);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m_word[e] = static_cast<float>(words[e] & 0xffffu);
                r_word[e] = static_cast<float>(words[e] >> 16);
            }
        }
        mc[p] = rc[p] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float mk = held_code<ROUND>(fabsf(m[p][e]), ms.inv, m_word[e]);
            const float rk = fmaxf(held_code<ROUND>(r[p][e], rs.inv, r_word[e]), fminf(fmaxf(r[p][e] * 0x1p100f, 0.0f), 1.0f));
            mc[p] = __builtin_amdgcn_cvt_pk_u8_f32(copysignf(mk, m[p][e]) + 128.0f, e, mc[p]);
            rc[p] = __builtin_amdgcn_cvt_pk_u8_f32(rk, e, rc[p]);
        }
        mc[p] = ms.live ? mc[p] ^ 0x80808080u : 0;
        rc[p] = rs.live ? rc[p] : 0;
        if (FULL || count[p] > 0) {
            __builtin_nontemporal_store(mc[p], reinterpret_cast<uint32_t*>(m_at + 128 * p));
            __builtin_nontemporal_store(rc[p], reinterpret_cast<uint32_t*>(r_at + 128 * p));
        }
    }
    if (l == 0) {
        *m_scale = ms.scale;
        *r_scale = rs.scale;
    }
}

// Four elements with states in 32 bits.
template <int DT, int GT, bool FULL>
__device__ __forceinline__ void adamw32_pieces(const UpdateTensor& t, const AdamwArgs& a, const UpdateFactors& k, int64_t first) {
    int count[kUpdatePieces];
    float g[kUpdatePieces][4], w[kUpdatePieces][4], m[kUpdatePieces][4], v[kUpdatePieces][4];
    char* const v_at = t.state + whole64(4 * t.n);
#pragma unroll
    for (int p = 0; p < kUpdatePieces; ++p) {
        const int64_t i = first + 4 * kWave * p, left = t.n - i;
        count[p] = FULL || left >= 4 ? 4 : left > 0 ? static_cast<int>(left) : 0;
        load_four<GT, FULL>(t.grad, i, count[p], g[p]);
        if (t.master) load_four<AQSGD_F32, FULL>(t.master, i, count[p], w[p]);
        else load_four<DT, FULL>(t.param, i, count[p], w[p]);
        load_four<AQSGD_F32, FULL>(t.state, i, count[p], m[p]);
        load_four<AQSGD_F32, FULL>(v_at, i, count[p], v[p]);
    }
#pragma unroll
    for (int p = 0; p < kUpdatePieces; ++p) {
        const int64_t i = first + 4 * kWave * p;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            step_moments(a, k, g[p][e], m[p][e], v[p][e]);
            w[p][e] = stepped_weight(a, k, w[p][e], m[p][e], sqrtf(v[p][e]));
        }
        if (t.master) store_four<AQSGD_F32, FULL>(t.master, i, count[p], w[p]);
        store_four<DT, FULL>(t.param, i, count[p], w[p]);
        store_four<AQSGD_F32, FULL>(t.state, i, count[p], m[p]);
        store_four<AQSGD_F32, FULL>(v_at, i, count[p], v[p]);
    }
}

// ---- the kernel ----------------------------------------------------------------------------------
template <int DT, int GT, int BITS, int ROUND>
__global__ __launch_bounds__(kWave * kUpdateWaves) void adamw_kernel(const UpdateTable table, const AdamwArgs a) {
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    UpdateFactors k;
    k.scale = a.scale ? *a.scale : 1.0f;
    if (!(fabsf(k.scale) < __builtin_inff())) return;                     // a step that is skipped
    const int which = __builtin_amdgcn_readfirstlane(__popcll(__ballot(table.first[lane] <= blockIdx.x)) - 1);
    const UpdateTensor& t = table.tensor[which];
    k.decay = t.decay;
    k.length = a.length;
    k.correct = a.correct;
    uint64_t key = a.key;
    if (a.lr_at || a.step_at) {                                           // some 150 instructions in binary64, a fifth of a wave's
        const int64_t now = a.step_at ? max(*a.step_at, int64_t{1}) : a.step;
        const double lr = a.lr_at ? static_cast<double>(*a.lr_at) : a.lr;
        k.decay = decay_factor(lr, t.weight_decay);
        k.length = length_factor(lr, a.beta1, now);
        k.correct = correct_factor(a.beta2, now);
        key = a.seed + static_cast<uint64_t>(now);
    }
    const int64_t begin = static_cast<int64_t>(blockIdx.x - table.first[which]) * kUpdateSpan + wave * (4 * kWave * kUpdatePieces);
    const int64_t left = t.n - begin;                                     // for the wave, which takes 512 elements
    if (left <= 0) return;
    if constexpr (BITS == 32) {
        if (left >= 4 * kWave * kUpdatePieces) adamw32_pieces<DT, GT, true>(t, a, k, begin + 4 * lane);
        else adamw32_pieces<DT, GT, false>(t, a, k, begin + 4 * lane);
    } else {
        const int64_t group = begin / kStateGroup + lane / 32;
        if (left >= 2 * kStateGroup) adamw8_group<DT, GT, ROUND, true>(t, a, k, key, group, lane & 31);
        else if (group * kStateGroup < t.n) adamw8_group<DT, GT, ROUND, false>(t, a, k, key, group, lane & 31);
    }
}

// The table goes to the runtime from where it is: launch_kernel's copies of its arguments would cost the host more here than elsewhere.
template <int DT, int GT>
hipError_t launch_adamw_as(const AdamwKind& kind, const UpdateTable& table, uint32_t blocks, const AdamwArgs& a, hipStream_t stream) {
    void (*const kernel)(const UpdateTable, const AdamwArgs) = kind.state_bits == 32                     ? adamw_kernel<DT, GT, 32, AQSGD_ROUND_NEAREST>
                                                               : kind.rounding == AQSGD_ROUND_NEAREST ? adamw_kernel<DT, GT, 8, AQSGD_ROUND_NEAREST>
                                                                                                      : adamw_kernel<DT, GT, 8, AQSGD_ROUND_STOCHASTIC>;
    void* argv[] = {const_cast<UpdateTable*>(&table), const_cast<AdamwArgs*>(&a)};
    return launch_with(reinterpret_cast<const void*>(kernel), dim3(blocks), dim3(kWave * kUpdateWaves), stream, argv);
}

}  // namespace aqsgd
