// Backward pass of a feed-forward block's first half, to the gradient of its projections: every element by
// itself, read and written once, so memory bounds it; the activation is a constant of the kernel, and its
// exponential and reciprocal are the hardware's, or arithmetic would weigh as much.
#include "aqsgd_products8.h"

namespace aqsgd {

// A lane's elements: 16 bytes, at any element's address, of which the first `count` exist.  Results go past the caches:
// 4096 x 6400 float16 gated 48.4 us, with ordinary stores 52.2.
template <int DT> constexpr int kPiece = DT == AQSGD_F32 ? 4 : 8;

template <int DT>
__device__ __forceinline__ void load_values(const void* base, int64_t at, int count, float (&f)[kPiece<DT>]) {
    const char* p = static_cast<const char*>(base) + at * ElemBytes<DT>::value;
    if (count < kPiece<DT>) {
#pragma unroll
        for (int e = 0; e < kPiece<DT>; ++e) f[e] = e < count ? load_elem<DT>(base, at + e) : 0.0f;
    } else if constexpr (DT == AQSGD_F32) {
        const f32x4_t v = *reinterpret_cast<const f32x4_any_t*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = v[e];
    } else {
        Raw<DT> r;
        r.v = *reinterpret_cast<const u32x4_any_t*>(p);
        unpack_raw<DT>(r, f);
    }
}

template <int DT>
__device__ __forceinline__ void store_values(void* base, int64_t at, int count, const float (&f)[kPiece<DT>]) {
    char* p = static_cast<char*>(base) + at * ElemBytes<DT>::value;
    if (count < kPiece<DT>) {
#pragma unroll
        for (int e = 0; e < kPiece<DT> - 1; ++e)
            if (e < count) store_elem<DT>(base, at + e, f[e]);
    } else if constexpr (DT == AQSGD_F32) {
        stream16(p, f32x4_t{f[0], f[1], f[2], f[3]});
    } else {
        stream16(p, pack_raw<DT>(f).v);
    }
}

// A workgroup takes `across` pieces of a row, of as many rows as 256 lanes hold.
template <int DT, int ACT, bool GATED>
__global__ __launch_bounds__(256) void ffn8_grad_kernel(const Ffn8GradArgs a, uint32_t across) {
    constexpr int N = kPiece<DT>;
    const uint32_t ty = threadIdx.x / across, tx = threadIdx.x - ty * across, rows = 256 / across;
    const int64_t c = (static_cast<int64_t>(blockIdx.x) * across + tx) * N, w = GATED ? 2 * a.f : a.f;
    if (ty >= rows || c >= a.f) return;
    const int count = static_cast<int>(min(a.f - c, static_cast<int64_t>(N)));
    for (int64_t m = static_cast<int64_t>(blockIdx.y) * rows + ty; m < a.m; m += static_cast<int64_t>(gridDim.y) * rows) {
        float d[N], g[N], u[N];
        load_values<DT>(a.dh, m * a.f + c, count, d);
        load_values<DT>(a.pre, m * w + c, count, g);
        if constexpr (GATED) load_values<DT>(a.pre, m * w + a.f + c, count, u);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float value, slope;
            activation_slope<DT>(ACT, g[e], value, slope);
            g[e] = GATED ? d[e] * u[e] * slope : d[e] * slope;
            u[e] = d[e] * value;
        }
        store_values<DT>(a.dpre, m * w + c, count, g);
        if constexpr (GATED) store_values<DT>(a.dpre, m * w + a.f + c, count, u);
    }
}

template <int DT, int ACT>
hipError_t launch_ffn8_grad_as(const Ffn8GradArgs& a, hipStream_t stream) {
    const int64_t pieces = (a.f + kPiece<DT> - 1) / kPiece<DT>, across = pieces < 256 ? pieces : 256;
    const int64_t rows = 256 / across, bands = (a.m + rows - 1) / rows;
    const dim3 grid(static_cast<unsigned>((pieces + across - 1) / across), static_cast<unsigned>(bands < 65535 ? bands : 65535)), block(256);
    return a.gated ? launch_kernel(ffn8_grad_kernel<DT, ACT, true>, grid, block, stream, a, static_cast<uint32_t>(across))
                   : launch_kernel(ffn8_grad_kernel<DT, ACT, false>, grid, block, stream, a, static_cast<uint32_t>(across));
}

template <int DT>
hipError_t launch_ffn8_grad_dt(const Ffn8GradArgs& a, hipStream_t stream) {
    switch (a.act) {
    case AQSGD_ACT_SILU: return launch_ffn8_grad_as<DT, AQSGD_ACT_SILU>(a, stream);
    case AQSGD_ACT_GELU: return launch_ffn8_grad_as<DT, AQSGD_ACT_GELU>(a, stream);
    default:             return launch_ffn8_grad_as<DT, AQSGD_ACT_GELU_TANH>(a, stream);
    }
}

hipError_t launch_ffn8_grad(const Ffn8GradArgs& a, hipStream_t stream) {
    switch (a.dtype) {
    case AQSGD_F32: return launch_ffn8_grad_dt<AQSGD_F32>(a, stream);
    case AQSGD_F16: return launch_ffn8_grad_dt<AQSGD_F16>(a, stream);
    default:        return launch_ffn8_grad_dt<AQSGD_BF16>(a, stream);
    }
}

}  // namespace aqsgd
