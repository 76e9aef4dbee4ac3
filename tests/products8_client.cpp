// A client of the C ABI that stands in for the device runtime's launch call: 8-bit products, blocks and quantisers go
// through the library's checks and its choice of kernels, and every launch is printed instead of made (the pointers
// are never followed).  Calls: m,dtype,message,m,n,k (matmul8), f,dtype,gated,m,f,k (ffn8), q,dtype,which,rows,cols,ld
// (quant8; which: 1 rows, 2 columns, 4 sums, 8 stochastic).  A line "call <status>" follows the launches of each.
#include <dlfcn.h>
#include <cxxabi.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>

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
    auto* codes = reinterpret_cast<int8_t*>(at);
    auto* floats = reinterpret_cast<float*>(at);
    const size_t plenty = size_t{1} << 40;
    for (int i = 1; i < argc; ++i) {
        char what;
        int dtype, kind;
        long x, y, z;
        if (std::sscanf(argv[i], "%c,%d,%d,%ld,%ld,%ld", &what, &dtype, &kind, &x, &y, &z) != 6) return 2;
        int status;
        if (what == 'm') {
            aqsgd_matmul8_desc d = {x, y, z, dtype, kind};
            status = aqsgd_matmul8(&d, at, floats, codes, floats, nullptr, nullptr, at, at, plenty, nullptr);
        } else if (what == 'f') {
            aqsgd_ffn8_desc d = {x, y, z, dtype, AQSGD_ACT_SILU, kind, 0};
            status = aqsgd_ffn8(&d, codes, floats, codes, floats, nullptr, at, at, nullptr);
        } else {
            aqsgd_quant8_desc d = {x, y, z, dtype, kind & 8 ? AQSGD_ROUND_STOCHASTIC : AQSGD_ROUND_NEAREST, 1};
            status = aqsgd_quant8(&d, at, kind & 1 ? codes : nullptr, kind & 1 ? floats : nullptr, kind & 2 ? codes : nullptr,
                                  kind & 2 ? floats : nullptr, kind & 4 ? floats : nullptr, at, plenty, nullptr);
        }
        std::printf("call %d\n", status);
    }
    return 0;
}
