// A client of the C ABI that stands in for the device runtime's launch call: layer norms, their gradients, AdamW steps and
// gradients' norms go through the library's checks and its choice of kernels, and every launch is printed instead of made
// (the pointers are never followed).  Calls: n,dtype,0,rows,cols (layernorm), g,dtype,which,rows,cols (layernorm_grad; which:
// 1 with sums, 2 dx over dy), a,dtype,kind,n,tensors (adamw; kind: the gradients' dtype, + 4 in 8 bits, + 8 stochastic),
// r,dtype,0,n,tensors (grad_norm).  A line "call <status>" follows the launches of each.
#include <dlfcn.h>
#include <cxxabi.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include <hip/hip_runtime_api.h>

#include "aqsgd.h"

extern "C" hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
    Dl_info info = {};
    char* name = nullptr;
    if (dladdr(f, &info) && info.dli_sname) name = abi::__cxa_demangle(info.dli_sname, nullptr, nullptr, nullptr);
    std::printf("launch %u %u %u x %u %s\n", grid.x, grid.y, grid.z, block.x, name ? name : "?");
    std::free(name);
    return hipSuccess;
}

int main(int argc, char** argv) {
    char* at = reinterpret_cast<char*>(uintptr_t{1} << 20);
    char* other = at + (uintptr_t{1} << 30);
    char* third = other + (uintptr_t{1} << 30);
    auto* floats = reinterpret_cast<float*>(at);
    const size_t plenty = size_t{1} << 40;
    for (int i = 1; i < argc; ++i) {
        char what;
        int dtype, kind;
        long x, y;
        if (std::sscanf(argv[i], "%c,%d,%d,%ld,%ld", &what, &dtype, &kind, &x, &y) != 5) return 2;
        int status;
        if (what == 'n' || what == 'g') {
            aqsgd_layernorm_desc d = {x, y, y, dtype, 0, 1e-5};
            status = what == 'n' ? aqsgd_layernorm(&d, at, nullptr, at, at, nullptr, other, floats, floats, nullptr, nullptr, nullptr)
                                 : aqsgd_layernorm_grad(&d, at, third, floats, floats, at, nullptr, kind & 2 ? at : other, kind & 1 ? floats : nullptr,
                                                        kind & 1 ? floats : nullptr, at, plenty, nullptr);
        } else {
            std::vector<aqsgd_adamw_tensor> tensors(static_cast<size_t>(y), {at, at, at, nullptr, x, 0.0});
            const int n = static_cast<int>(y);
            aqsgd_adamw_desc d = {1e-3, 0.9, 0.999, 1e-8, 1, dtype, kind & 3, kind & 4 ? 8 : 32, kind & 8 ? AQSGD_ROUND_STOCHASTIC : AQSGD_ROUND_NEAREST, 1};
            status = what == 'a' ? aqsgd_adamw(&d, tensors.data(), n, nullptr, nullptr, nullptr, nullptr)
                                 : aqsgd_grad_norm(dtype, tensors.data(), n, 1.0, nullptr, floats, at, plenty, nullptr);
        }
        std::printf("call %d\n", status);
    }
    return 0;
}
