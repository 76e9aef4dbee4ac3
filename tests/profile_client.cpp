// A client of the C ABI that stands in for the device runtime's launch calls: AdamW steps, gradients' norms and layer norms' gradients whose
// time is asked for.  Every launch is printed with the stamps it is to make, 1 its begin, 2 its end (the pointers are never followed).
// Calls: a,dtype,n,tensors (adamw, n elements each), r,dtype,n,tensors (grad_norm), g,dtype,rows,cols (layernorm_grad).
#include <cstdio>
#include <vector>

#include <hip/hip_runtime_api.h>

#include "aqsgd.h"

static int stamps(hipEvent_t start, hipEvent_t stop) { return (start ? 1 : 0) + (stop ? 2 : 0); }

extern "C" hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) {
    std::printf("launch 0\n");
    return hipSuccess;
}
extern "C" hipError_t hipExtLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t, hipEvent_t start, hipEvent_t stop, int) {
    std::printf("launch %d\n", stamps(start, stop));
    return hipSuccess;
}

int main(int argc, char** argv) {
    char* at = reinterpret_cast<char*>(uintptr_t{1} << 20);
    char* other = at + (uintptr_t{1} << 40);
    auto* floats = reinterpret_cast<float*>(at);
    for (int i = 1; i < argc; ++i) {
        char what;
        int dtype;
        long x, y;
        if (std::sscanf(argv[i], "%c,%d,%ld,%ld", &what, &dtype, &x, &y) != 4) return 2;
        aqsgd_profile_next_launch(at, other);
        int status;
        if (what == 'g') {
            aqsgd_layernorm_desc d = {x, y, y, dtype, 0, 1e-5};
            status = aqsgd_layernorm_grad(&d, at, at, floats, floats, at, nullptr, other, floats, floats, at, size_t{1} << 40, nullptr);
        } else {
            std::vector<aqsgd_adamw_tensor> tensors(static_cast<size_t>(y), {at, at, at, nullptr, x, 0.0});
            aqsgd_adamw_desc d = {1e-3, 0.9, 0.999, 1e-8, 1, dtype, dtype, 32, AQSGD_ROUND_NEAREST, 0};
            status = what == 'a' ? aqsgd_adamw(&d, tensors.data(), static_cast<int32_t>(y), nullptr, nullptr, nullptr, nullptr)
                                 : aqsgd_grad_norm(dtype, tensors.data(), static_cast<int32_t>(y), 1.0, nullptr, floats, at, size_t{1} << 40, nullptr);
        }
        std::printf("call %d\n", status);
    }
    return 0;
}
