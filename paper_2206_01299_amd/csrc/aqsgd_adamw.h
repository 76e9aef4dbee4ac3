// Kernels of aqsgd_adamw: one step of many tensors in one launch.
//
// Every element is read and written once, so memory bounds the step.  A wave takes a group of 256 elements, four
// neighbouring ones a lane: with states in 8 bits the group's new scale is a maximum over the wave, and everything
// stays in registers between the loads and the stores.  A workgroup's tensor is found in the launch's table by one load
// and a vote of the wave.
#pragma once

#include "aqsgd_norms.h"

namespace aqsgd {

constexpr int kUpdateWaves = 4, kUpdateGroups = 2;                        // waves of a workgroup, groups of a wave
constexpr int64_t kUpdateSpan = int64_t{kStateGroup} * kUpdateWaves * kUpdateGroups;
constexpr float kStateFloor = 0x1p-100f;                                  // a group below this is held as zeros: T^2 / s is finite from here on
constexpr float kMTop = 127.0f, kRTop = 255.0f;

// Where the parts of a tensor's state lie, in bytes.
__host__ __device__ inline int64_t whole64(int64_t bytes) { return (bytes + 63) / 64 * 64; }
__host__ __device__ inline int64_t state_groups(int64_t n) { return (n + kStateGroup - 1) / kStateGroup; }
__host__ __device__ inline int64_t state_bytes(int64_t n, int bits) {
    return bits == 32 ? 2 * whole64(4 * n) : 2 * whole64(n) + 2 * whole64(4 * state_groups(n));
}

typedef uint16_t u16x4_t __attribute__((ext_vector_type(4)));

// Four elements at any element's address, of which `count` exist.
template <int DT>
__device__ __forceinline__ void load_four(const void* base, int64_t i, int count, float (&f)[4]) {
    if (count >= 4) {
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

template <int DT>
__device__ __forceinline__ void store_four(void* base, int64_t i, int count, const float (&f)[4]) {
    if (count >= 4) {
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
    float scale;
    bool scaled;
};

__device__ __forceinline__ void step_element(const AdamwArgs& a, const UpdateFactors& k, float g, float& w, float& m, float& v, float& r) {
    if (k.scaled) g = g * k.scale;
    m = m * a.beta1f + g * a.rest1;
    v = v * a.beta2f + (g * a.rest2) * g;
    r = sqrtf(v);
    const float denominator = r * k.correct + a.eps;
    w = w * k.decay - (m / denominator) * k.length;
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

// The code of one magnitude: the neighbour below u's root and the choice between it and the next.
__device__ __forceinline__ float held_code(float x, const HeldScale& h, float top, float least, float z) {
    const float u = x * h.inv;
    float k = floorf(sqrtf(u));
    if (k * k > u) k -= 1.0f;             // the root is rounded: it may be a whole number that u's own is just below
    k = fminf(k, top);
    if (u - k * k >= z * (2.0f * k + 1.0f)) k += 1.0f;
    k = fminf(k, top);
    return h.live && x > 0.0f ? fmaxf(k, least) : 0.0f;
}

__device__ __forceinline__ uint32_t magnitude_of(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// ---- the kernel ----------------------------------------------------------------------------------
template <int DT, int GT, int BITS, int ROUND>
__global__ __launch_bounds__(kWave * kUpdateWaves) void adamw_kernel(const UpdateTable table, const AdamwArgs a) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    UpdateFactors k;
    k.scaled = a.scale != nullptr;
    k.scale = k.scaled ? *a.scale : 1.0f;
    if (!(fabsf(k.scale) < __builtin_inff())) return;                     // a step that is skipped
    const int which = __builtin_amdgcn_readfirstlane(__popcll(__ballot(table.first[lane] <= blockIdx.x)) - 1);
    const UpdateTensor& t = table.tensor[which];
    int64_t now = a.step_at ? *a.step_at : a.step;
    if (now < 1) now = 1;
    const double lr = a.lr_at ? static_cast<double>(*a.lr_at) : a.lr;
    k.decay = static_cast<float>(1.0 - lr * t.weight_decay);
    k.length = static_cast<float>(lr / (1.0 - power_of(a.beta1, now)));
    k.correct = static_cast<float>(1.0 / sqrt(1.0 - power_of(a.beta2, now)));
    const uint64_t key = a.seed + static_cast<uint64_t>(now);
    const int64_t span = static_cast<int64_t>(blockIdx.x - table.first[which]) * (kUpdateWaves * kUpdateGroups);
#pragma unroll
    for (int q = 0; q < kUpdateGroups; ++q) {
        const int64_t group = span + wave * kUpdateGroups + q, i = group * kStateGroup + lane * 4;
        if (group * kStateGroup >= t.n) return;
        const int64_t left = t.n - i;
        const int count = left >= 4 ? 4 : left > 0 ? static_cast<int>(left) : 0;
        float g[4], w[4], m[4], v[4], r[4];
        load_four<GT>(t.grad, i, count, g);
        if (t.master) load_four<AQSGD_F32>(t.master, i, count, w);
        else load_four<DT>(t.param, i, count, w);
        char* const m_at = t.state;
        char* const r_at = t.state + whole64(BITS == 32 ? 4 * t.n : t.n);
        float* const m_scales = reinterpret_cast<float*>(t.state + 2 * whole64(t.n));
        float* const r_scales = m_scales + whole64(4 * state_groups(t.n)) / 4;
        if constexpr (BITS == 32) {
            load_four<AQSGD_F32>(m_at, i, count, m);
            load_four<AQSGD_F32>(r_at, i, count, v);
        } else {
            uint32_t mc = 0, rc = 0;
            if (count > 0) {
                mc = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(m_at + i));
                rc = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(r_at + i));
            }
            const float m_step = m_scales[group] / (kMTop * kMTop), r_step = r_scales[group] / (kRTop * kRTop);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float mk = static_cast<float>(static_cast<int8_t>(mc >> (8 * e))), rk = static_cast<float>((rc >> (8 * e)) & 0xffu);
                m[e] = (mk * fabsf(mk)) * m_step;
                const float root = (rk * rk) * r_step;
                v[e] = root * root;
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) step_element(a, k, g[e], w[e], m[e], v[e], r[e]);
        if (t.master) store_four<AQSGD_F32>(t.master, i, count, w);
        store_four<DT>(t.param, i, count, w);
        if constexpr (BITS == 32) {
            store_four<AQSGD_F32>(m_at, i, count, m);
            store_four<AQSGD_F32>(r_at, i, count, v);
        } else {
            uint32_t m_top = 0, r_top = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (e >= count) m[e] = r[e] = 0.0f;
                m_top = max(m_top, magnitude_of(m[e]));
                r_top = max(r_top, magnitude_of(r[e]));
            }
            const HeldScale ms = held_scale(__float_as_uint(team_max<kWave>(__uint_as_float(m_top))), kMTop);
            const HeldScale rs = held_scale(__float_as_uint(team_max<kWave>(__uint_as_float(r_top))), kRTop);
            float zm[4], zr[4];
            if constexpr (ROUND == AQSGD_ROUND_STOCHASTIC) {
                const uint64_t block = static_cast<uint64_t>((t.group0 + group) * (kStateGroup / 4) + lane);
                uint32_t words[4];
                philox4x32_10(static_cast<uint32_t>(block), static_cast<uint32_t>(block >> 32), static_cast<uint32_t>(key),
                              static_cast<uint32_t>(key >> 32), words);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    zm[e] = static_cast<float>((words[e] & 0xffffu) + 1u) * 0x1p-16f;
                    zr[e] = static_cast<float>((words[e] >> 16) + 1u) * 0x1p-16f;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) zm[e] = zr[e] = 0.5f;
            }
            uint32_t mc = 0, rc = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float mk = held_code(fabsf(m[e]), ms, kMTop, 0.0f, zm[e]);
                mc |= (static_cast<uint32_t>(static_cast<int32_t>(m[e] < 0.0f ? -mk : mk)) & 0xffu) << (8 * e);
                rc |= static_cast<uint32_t>(held_code(r[e], rs, kRTop, 1.0f, zr[e])) << (8 * e);
            }
            if (count > 0) {
                __builtin_nontemporal_store(mc, reinterpret_cast<uint32_t*>(m_at + i));
                __builtin_nontemporal_store(rc, reinterpret_cast<uint32_t*>(r_at + i));
            }
            if (lane == 0) {
                m_scales[group] = ms.scale;
                r_scales[group] = rs.scale;
            }
        }
    }
}

template <int DT, int GT>
hipError_t launch_adamw_as(const AdamwKind& kind, const UpdateTable& table, uint32_t blocks, const AdamwArgs& a, hipStream_t stream) {
    const dim3 grid(blocks), block(kWave * kUpdateWaves);
    if (kind.state_bits == 32) return launch_kernel(adamw_kernel<DT, GT, 32, AQSGD_ROUND_NEAREST>, grid, block, stream, table, a);
    if (kind.rounding == AQSGD_ROUND_NEAREST) return launch_kernel(adamw_kernel<DT, GT, 8, AQSGD_ROUND_NEAREST>, grid, block, stream, table, a);
    return launch_kernel(adamw_kernel<DT, GT, 8, AQSGD_ROUND_STOCHASTIC>, grid, block, stream, table, a);
}

}  // namespace aqsgd
