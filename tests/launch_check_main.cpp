// Driver for the CPU test of what the policy's memory launches: layer_norm.hip's and linear_attention.hip's host side, linked with the few
// runtime calls below instead of the HIP runtime.  They note each launch and check it against what a launch may have:
// 1 to 1024 threads a workgroup, 2^32 - 1 threads along a dimension, 65535 workgroups along the second and third, 160 KB of LDS,
// and more than 64 KB of it only for kernels that have been allowed it.  Built and run by tests/test_host_launches.py;
// prints "ok <launches> <kernels> <launches above 64 KB>", or the launches that are wrong.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>
#include <map>
#include <set>
#include <string>

#include "../paper_2502_00021_amd/csrc/pxr_internal.h"

namespace {

struct Launch {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
};
Launch pushed;
std::map<const void*, std::string>& names() {
    static std::map<const void*, std::string> m;
    return m;
}
std::map<const void*, size_t> allowed;
std::set<const void*> launched;
uint64_t launches = 0, large = 0, wrong = 0;
std::string what;  // the call that is made

}  // namespace

extern "C" {

void** __hipRegisterFatBinary(const void*) {
    static void* modules = nullptr;
    return &modules;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* function, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[function] = name; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
    pushed = {grid, block, lds, stream};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
    *grid = pushed.grid;
    *block = pushed.block;
    *lds = pushed.lds;
    *stream = pushed.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void* function, dim3 grid, dim3 block, void**, size_t lds, hipStream_t) {
    const uint64_t threads = (uint64_t)block.x * block.y * block.z;
    const bool fits = grid.x && grid.y && grid.z && threads && threads <= 1024 && (uint64_t)grid.x * block.x < (1ull << 32) && grid.y <= 65535 && grid.z <= 65535;
    const auto cap = allowed.find(function);
    const size_t most = cap == allowed.end() ? 64 * 1024 : cap->second;
    ++launches;
    large += lds > 64 * 1024;
    launched.insert(function);
    if ((!fits || lds > most || lds > 160 * 1024) && wrong++ < 10)
        std::printf("%s: %s: grid %u x %u x %u, block %u x %u x %u, %zu bytes of LDS (allowed %zu)\n", what.c_str(), names()[function].c_str(), grid.x, grid.y, grid.z,
                    block.x, block.y, block.z, lds, most);
    return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void* function, hipFuncAttribute attribute, int value) {
    if (attribute == hipFuncAttributeMaxDynamicSharedMemorySize) allowed[function] = (size_t)value;
    return hipSuccess;
}
hipError_t hipGetDevice(int* device) {
    *device = 0;
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "no error"; }
}

namespace {

float* const p = reinterpret_cast<float*>(4096);  // (nothing is read through it)

void layer_norms() {
    const uint32_t widths[] = {1,    3,    4,    7,    8,     64,    256,   333,   512,   1000,   1024,   1300,    2048,    4096,      5000,          8192,           12345,     16384,
                               30752, 32768, 32769, 34001, 65536, 65537, 70001, 131072, 131073, 1000003, 1 << 24, 1 << 26, (1u << 27) - 1, (1u << 27) + 1000, 1u << 30};
    const uint64_t rows[] = {1, 2, 3, 4, 5, 50, 999, 1024, 5000, 65536, 500000, 4000000, 0x7FFFFFFF};
    for (uint32_t width : widths)
        for (uint64_t n : rows)
            for (uint32_t types = 0; types < 3; ++types) {
                const pxr_layer_norm_desc d{types ? PXR_BF16 : PXR_F32, types == 2 ? PXR_BF16 : PXR_F32, n, width, 1e-5f, width, width, width};
                if ((double)n * width * (types ? 2 : 4) > 288e9) continue;  // (more than the memory of a device)
                std::string err;
                what = "layer norm " + std::to_string(n) + " x " + std::to_string(width) + " types " + std::to_string(types);
                pxr::launch_layer_norm_forward(d, p, p, p, p, p, p, nullptr, err);
                pxr::launch_layer_norm_backward(d, p, p, p, p, p, p, p, p, p, nullptr, err);
                pxr::launch_layer_norm_backward(d, p, p, p, p, p, p, nullptr, nullptr, nullptr, nullptr, err);
            }
}

void attentions() {
    std::string err;
    pxr::prepare_linear_attention_kernels(err);
    const uint32_t sizes[] = {1, 8, 31, 32, 33, 64, 65, 100, 128, 129, 200, 256};
    const uint32_t rollouts[][2] = {{1, 0}, {1, 1}, {1, 33}, {1, 20000}, {1, 0x7FFFFFFF}, {3, 700}, {40, 1000}, {512, 256}, {4000, 2}, {1u << 21, 40}};
    for (uint32_t dk : sizes)
        for (uint32_t dv : sizes)
            for (uint32_t heads : {1u, 3u, 8u})
                for (const auto& size : rollouts)
                    for (uint32_t dtype : {(uint32_t)PXR_F32, (uint32_t)PXR_BF16}) {
                        const uint32_t envs = size[0] == 1u << 21 ? (1u << 21) / heads : size[0];
                        const pxr::LinearAttentionConsts c{heads, dk, dv, 256u, 1.0f, nullptr};
                        const pxr_tokens t{p, 1, 1, 1};
                        pxr_rollout r{dtype, envs, size[1], t, t, t, nullptr, 0, 0, p};
                        what = "linear attention " + std::to_string(envs) + " x " + std::to_string(size[1]) + ", " + std::to_string(heads) + " heads of " + std::to_string(dk) + " x " +
                               std::to_string(dv) + " type " + std::to_string(dtype);
                        pxr::launch_linear_attention_forward(c, r, t, p, p, nullptr, err);
                        pxr::launch_linear_attention_backward(c, r, t, p, t, t, t, p, p, nullptr, err);
                        r.n_steps = 1;
                        pxr::launch_linear_attention_step(c, r, p, t, nullptr, err);
                    }
}

}  // namespace

int main() {
    layer_norms();
    attentions();
    if (wrong) {
        std::printf("%llu launches of %llu are wrong\n", (unsigned long long)wrong, (unsigned long long)launches);
        return 1;
    }
    std::printf("ok %llu %zu %llu\n", (unsigned long long)launches, launched.size(), (unsigned long long)large);
    return 0;
}
