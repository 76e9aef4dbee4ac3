// Backward pass of a feed-forward block's first half, to the gradient of its projections.
#include "aqsgd_products8.h"

namespace aqsgd {

__global__ __launch_bounds__(256) void ffn8_grad_kernel(const Ffn8GradArgs a) {
    const int64_t w = a.gated ? 2 * a.f : a.f, pieces = (a.f + 3) / 4, total = a.m * pieces;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t row = i / pieces, c = (i - row * pieces) * 4;
        for (int64_t f = c; f < min(c + 4, a.f); ++f) {
            const float d = load1(a.dtype, a.dh, row * a.f + f);
            float value, slope;
            activation_slope(a.act, load1(a.dtype, a.pre, row * w + f), value, slope);
            if (a.gated) {
                const float up = load1(a.dtype, a.pre, row * w + a.f + f);
                store1(a.dtype, a.dpre, row * w + f, d * up * slope);
                store1(a.dtype, a.dpre, row * w + a.f + f, d * value);
            } else {
                store1(a.dtype, a.dpre, row * w + f, d * slope);
            }
        }
    }
}

hipError_t launch_ffn8_grad(const Ffn8GradArgs& a, hipStream_t stream) {
    const int64_t blocks = (a.m * ((a.f + 3) / 4) + 255) / 256;
    return launch_kernel(ffn8_grad_kernel, dim3(static_cast<unsigned>(blocks < 8192 ? blocks : 8192)), dim3(256), stream, a);
}

}  // namespace aqsgd
