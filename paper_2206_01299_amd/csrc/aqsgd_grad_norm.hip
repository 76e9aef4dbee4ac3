// The 2-norm over many tensors' gradients and the factor that clips them: a pass that leaves a sum of squares for each
// workgroup, and one workgroup that joins them; what one workgroup reads faster than a second launch comes, it takes alone.  Squares
// are summed in binary64, in which none overflows and no order shows.  Memory bounds the first pass.
#include "aqsgd_adamw.h"
#include "aqsgd_layernorm.h"

namespace aqsgd {
namespace {

constexpr int kLanes = 256, kJoinLanes = 1024;

template <int LANES>
__device__ __forceinline__ double workgroup_sum(double v, double* part) {
    v = lanes_sum<kWave>(v);
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    double sum = part[0];
#pragma unroll
    for (int w = 1; w < LANES / kWave; ++w) sum += part[w];
    return sum;
}

template <int GT>
__device__ __forceinline__ double added_squares(const u32x4_t& piece, double sum) {
    float f[kPiece<GT>];
    piece_values<GT>(piece, f);
#pragma unroll
    for (int e = 0; e < kPiece<GT>; ++e) sum = fma(static_cast<double>(f[e]), static_cast<double>(f[e]), sum);
    return sum;
}

// Pieces of 16 bytes, kAhead of a lane's on their way at a time; spans are whole pieces, so that only the last one of a tensor
// ends inside one.
template <int GT>
__global__ __launch_bounds__(kLanes) void grad_squares_kernel(const NormTable table, const int64_t span, double* partial) {
    constexpr int V = kPiece<GT>, kAhead = 4;
    __shared__ double part[kLanes / kWave];
    const int which = __builtin_amdgcn_readfirstlane(__popcll(__ballot(table.first[threadIdx.x & (kWave - 1)] <= blockIdx.x)) - 1);
    const int64_t n = table.n[which], begin = static_cast<int64_t>(blockIdx.x - table.first[which]) * span;
    const int64_t end = begin + span < n ? begin + span : n;
    const char* const grad = element_at<GT>(table.grad[which], 0);
    // Past the caches: 123 M float16 41.2 us, with ordinary loads 47.2; float32 78.1 and 89.2.
    const auto piece_at = [&](int64_t i) -> u32x4_t { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_any_t*>(grad + i * ElemBytes<GT>::value)); };
    double sum[2] = {};
    int64_t i = begin + threadIdx.x * V;
    for (; i + (kAhead - 1) * kLanes * V + V <= end; i += kAhead * kLanes * V) {
        u32x4_t piece[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) piece[k] = piece_at(i + k * kLanes * V);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) sum[k & 1] = added_squares<GT>(piece[k], sum[k & 1]);
    }
    for (; i + V <= end; i += kLanes * V) sum[0] = added_squares<GT>(piece_at(i), sum[0]);
    for (; i < end; ++i) {                                   // one lane's, of the tensor's last piece
        const double f = static_cast<double>(load_elem<GT>(grad, i));
        sum[1] = fma(f, f, sum[1]);
    }
    const double all = workgroup_sum<kLanes>(sum[0] + sum[1], part);
    if (threadIdx.x == 0) partial[blockIdx.x] = all;
}

// The results, by one lane.
__device__ __forceinline__ void leave_norm(double sum, double max_norm, const float* loss_scale, float* result) {
    const double inverse = loss_scale ? 1.0 / static_cast<double>(*loss_scale) : 1.0, norm = sqrt(sum) * inverse;
    const double clip = max_norm / norm;                    // 0 / 0, of no gradient at all: nothing to clip
    result[0] = static_cast<float>(norm);
    result[1] = norm < __builtin_inf() ? static_cast<float>((clip < 1.0 ? clip : 1.0) * inverse) : __builtin_nanf("");
}

// A wave to a chunk of 64 pieces, each wave's four asked for at once.  A tensor's last piece is moved back to end with it, what lies in
// front of its place counts nothing.  1000 bfloat16 2.0 us (in two launches 3.6), 16384 float32 3.1 (3.8), 32768 bfloat16 3.8 (3.9), and
// the host is done up to 3.5 us earlier; twice as many, with eight chunks a wave, 4.6 (3.9).
template <int GT>
__global__ __launch_bounds__(kJoinLanes) void grad_norm_few_kernel(const NormTable table, const uint32_t chunks, const double max_norm, const float* loss_scale, float* result) {
    constexpr int V = kPiece<GT>, kWaves = kJoinLanes / kWave, kEach = kFewChunks / kWaves;
    __shared__ double part[kWaves];
    const int lane = threadIdx.x & (kWave - 1);
    const uint32_t first = table.first[lane], wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    u32x4_t piece[kEach];
    int skip[kEach];                                        // elements of the piece that are not to count
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const uint32_t chunk = wave + k * kWaves;
        if (chunk >= chunks) break;
        const int which = __builtin_amdgcn_readfirstlane(__popcll(__ballot(first <= chunk)) - 1);
        const int64_t n = table.n[which], i = static_cast<int64_t>(chunk - table.first[which]) * (kWave * V) + lane * V;
        if (n >= V) {
            const int64_t at = i + V <= n ? i : n - V;
            skip[k] = i - at < V ? static_cast<int>(i - at) : V;
            piece[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any_t*>(element_at<GT>(table.grad[which], at)));
        } else {
            float f[V];
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = i + e < n ? load_elem<GT>(table.grad[which], i + e) : 0.0f;
            skip[k] = 0;
            piece[k] = values_piece<GT>(f);
        }
    }
    double sums[2] = {};
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        if (wave + k * kWaves >= chunks) break;
        float f[V];
        piece_values<GT>(piece[k], f);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const double d = static_cast<double>(e < skip[k] ? 0.0f : f[e]);
            sums[e & 1] = fma(d, d, sums[e & 1]);
        }
    }
    double sum = sums[0] + sums[1];
    sum = workgroup_sum<kJoinLanes>(sum, part);
    if (threadIdx.x == 0) leave_norm(sum, max_norm, loss_scale, result);
}

__global__ __launch_bounds__(kJoinLanes) void grad_norm_kernel(const double* partial, const int64_t count, const double max_norm, const float* loss_scale, float* result) {
    __shared__ double part[kJoinLanes / kWave];
    double sum = 0.0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < count; i += kJoinLanes) sum += partial[i];
    sum = workgroup_sum<kJoinLanes>(sum, part);
    if (threadIdx.x == 0) leave_norm(sum, max_norm, loss_scale, result);
}

}  // namespace

hipError_t launch_grad_squares(int dtype, const NormTable& table, uint32_t blocks, int64_t span, double* partial, hipStream_t stream) {
    const dim3 grid(blocks), block(kLanes);
    switch (dtype) {
    case AQSGD_F32:  return launch_kernel(grad_squares_kernel<AQSGD_F32>, grid, block, stream, table, span, partial);
    case AQSGD_F16:  return launch_kernel(grad_squares_kernel<AQSGD_F16>, grid, block, stream, table, span, partial);
    default:         return launch_kernel(grad_squares_kernel<AQSGD_BF16>, grid, block, stream, table, span, partial);
    }
}

int64_t norm_chunk(int dtype) { return kWave * (dtype == AQSGD_F32 ? kPiece<AQSGD_F32> : kPiece<AQSGD_F16>); }

hipError_t launch_grad_norm_few(int dtype, const NormTable& table, uint32_t chunks, double max_norm, const float* loss_scale, float* result, hipStream_t stream) {
    const dim3 grid(1), block(kJoinLanes);
    switch (dtype) {
    case AQSGD_F32:  return launch_kernel(grad_norm_few_kernel<AQSGD_F32>, grid, block, stream, table, chunks, max_norm, loss_scale, result);
    case AQSGD_F16:  return launch_kernel(grad_norm_few_kernel<AQSGD_F16>, grid, block, stream, table, chunks, max_norm, loss_scale, result);
    default:         return launch_kernel(grad_norm_few_kernel<AQSGD_BF16>, grid, block, stream, table, chunks, max_norm, loss_scale, result);
    }
}

hipError_t launch_grad_norm(const double* partial, int64_t count, double max_norm, const float* loss_scale, float* result, hipStream_t stream) {
    return launch_kernel(grad_norm_kernel, dim3(1), dim3(kJoinLanes), stream, partial, count, max_norm, loss_scale, result);
}

}  // namespace aqsgd
