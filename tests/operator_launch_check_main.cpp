// Driver for the CPU test of what the gated recurrence, the turned heads and the orthogonalised updates launch: their host side, with the stand-in for
// the runtime of launch_check_main.cpp and its limits of a launch.  Sizes run up to the largest that the calls take.  The workspaces that the calls ask
// for are compared with what a device has, so that no size that fits one is left out.  Built and run by tests/test_host_operator_launches.py.
#define main memory_main
#include "launch_check_main.cpp"
#undef main

#include <algorithm>

namespace {

constexpr double kMemory = 288e9;

void recurrences() {
    std::string err;
    const uint32_t widths[] = {1, 2, 3, 15, 16, 31, 33, 63, 64, 65, 128, 129, 257, 1024, 4099, 65536, 1u << 20, 1u << 28};
    const uint32_t steps[] = {0, 1, 2, 16, 17, 127, 128, 129, 255, 256, 257, 1000, 4096, 50000, 1000003, 1u << 29};
    const uint32_t envs[] = {1, 2, 3, 4, 5, 33, 512, 4000, 16384, 1u << 20, 1u << 22};
    for (uint32_t width : widths)
        for (uint32_t t : steps)
            for (uint32_t e : envs)
                for (uint32_t dtype : {(uint32_t)PXR_F32, (uint32_t)PXR_BF16})
                    for (int64_t apart : {(int64_t)t * width, (int64_t)0, (int64_t)-5, (int64_t)1 << 40}) {
                        const uint64_t wide = (uint64_t)e * ((width + 63) / 64), parts = std::max(1u, (t + 127) / 128);
                        if (wide * parts > (1ull << 22)) continue;  // (refused)
                        if ((double)e * t * width * (dtype == PXR_F32 ? 4 : 2) > kMemory) continue;
                        const pxr_steps v{p, apart, width};
                        pxr_gated_rollout r{dtype, e, t, width, t & 1u, v, v, nullptr, 0, 0, p};
                        what = "gated recurrence " + std::to_string(e) + " x " + std::to_string(t) + " x " + std::to_string(width) + " type " + std::to_string(dtype) + " apart " + std::to_string(apart);
                        pxr::launch_gated_recurrence_forward(r, v, p, p, nullptr, err);
                        pxr::launch_gated_recurrence_backward(r, v, p, v, v, p, p, nullptr, err);
                        r.n_steps = 1;
                        pxr::launch_gated_recurrence_step(r, p, v, nullptr, err);
                    }
}

void heads() {
    std::string err;
    const uint64_t tokens[][2] = {{0, 5}, {1, 0}, {1, 1}, {16, 1}, {3, 77}, {256, 128}, {16384, 1}, {1, 0x7FFFFFFF}, {0x7FFFFFFF, 1}};
    for (uint32_t d : {1u, 2u, 3u, 8u, 33u, 48u, 64u, 100u, 128u, 200u, 255u, 256u})
        for (uint32_t r : {0u, 2u, d / 4 * 2, d / 2 * 2})
            for (const auto& n : tokens)
                for (uint32_t h : {0u, 1u, 5u, 16u, 65535u})
                    for (uint32_t hk : {0u, 1u, 4u, 65535u})
                        for (uint32_t types = 0; types < 3; ++types) {
                            if (r > d) continue;
                            const pxr::HeadNormConsts c{d, r, 1e-6f, nullptr};
                            const pxr_tokens t{p, 1, 1, 1};
                            const pxr_heads a{types ? PXR_BF16 : PXR_F32, types == 2 ? PXR_BF16 : PXR_F32, (uint32_t)n[0], (uint32_t)n[1], h, hk, t, t, nullptr, nullptr, nullptr, 32, 0, 0, 0};
                            what = "heads " + std::to_string(h) + " + " + std::to_string(hk) + " of " + std::to_string(d) + ", " + std::to_string(n[0]) + " x " + std::to_string(n[1]);
                            pxr::launch_head_norm_forward(c, a, &t, &t, nullptr, err);
                            pxr::launch_head_norm_backward(c, a, &t, &t, &t, &t, p, p, p, nullptr, err);
                        }
}

void updates() {
    std::string err;
    const float c[9] = {3.4445f, -4.775f, 2.0315f, 3.4445f, -4.775f, 2.0315f, 3.4445f, -4.775f, 2.0315f};
    const uint32_t sizes[] = {1, 2, 7, 31, 32, 33, 64, 65, 96, 97, 127, 128, 129, 200, 256, 448, 512, 1000, 1130, 1500, 2048, 2900, 4096, 5000, 10000, 1u << 15, 200000, 1u << 20, 1u << 28};
    for (uint32_t rows : sizes)
        for (uint32_t cols : sizes)
            for (uint32_t n : {1u, 2u, 3u, 8u, 300u, 65535u})
                for (uint32_t dtype : {(uint32_t)PXR_F32, (uint32_t)PXR_BF16}) {
                    if (std::min(rows, cols) > (1u << 15) || (uint64_t)rows * cols > (1ull << 32)) continue;  // (refused)
                    const pxr_orthogonalise_desc d{dtype, n, rows, cols, (int64_t)rows * cols, cols, (int64_t)rows * cols, cols, 3, c, 1e-7f};
                    const double need = (double)n * rows * cols * (dtype == PXR_F32 ? 4 : 2) + (double)pxr::orthogonalise_workspace(d);
                    if (need > kMemory) continue;
                    what = "orthogonalise " + std::to_string(n) + " x " + std::to_string(rows) + " x " + std::to_string(cols) + " type " + std::to_string(dtype);
                    pxr::launch_orthogonalise(d, p, p, p, nullptr, err);
                }
}

}  // namespace

int main() {
    recurrences();
    heads();
    updates();
    if (wrong) {
        std::printf("%llu launches of %llu are wrong\n", (unsigned long long)wrong, (unsigned long long)launches);
        return 1;
    }
    std::printf("ok %llu %zu %llu\n", (unsigned long long)launches, launched.size(), (unsigned long long)large);
    return 0;
}
