// Driver for the CPU test of the steps that the scan kernels ask for (csrc/steps.h): every request of every lane of every kernel, for the
// chunks that rollouts are cut into, forward and in reverse, against the rows that the view has.  Built and run by
// tests/test_host_steps.py; prints "ok <requests> <kernels>", or the first requests outside.
#include <cstdint>
#include <cstdio>
#include <initializer_list>

#include "../paper_2502_00021_amd/csrc/steps.h"

namespace {

uint64_t requests = 0, outside = 0, misplaced = 0, kernels = 0;

// All lanes' requests for the chunk that holds rows [first, first + n) of a view of `rows` rows of d values, `step` apart.
template <int kBytes, int kWidth, int kThreads>
void chunk(int64_t first, uint32_t n, int64_t rows, uint32_t d, int64_t step) {
    typedef pxr::Dealt<kBytes, kWidth, kThreads> D;
    for (uint32_t thread = 0; thread < (uint32_t)kThreads; ++thread) {
        const uint32_t row = D::row(thread), col = D::col(thread);
        const int64_t offset = D::offset(row, col, d, step);
        for (uint32_t i = 0; i < D::kCount; ++i) {
            const int64_t at = D::request(first * step, i, n, row, col, d, step, offset);
            ++requests;
            if (at < 0 || at / step >= rows || at % step + D::N > d) {
                if (outside++ < 5)
                    std::printf("%d-byte values, %d wide, %d threads: thread %u, request %u: value %lld of row %lld of %lld (d %u, chunk of %u from %lld)\n", kBytes, kWidth,
                                kThreads, thread, i, (long long)(at % step), (long long)(at / step), (long long)rows, d, n, (long long)first);
                continue;
            }
            // what is written to the tile is the vector of that place
            const uint32_t r = row + i * D::kRowsEach;
            const int64_t c = (int64_t)(col + D::N <= d ? col : d - D::N);
            if (r < n && col < d && at != (first + r) * step + c) ++misplaced;
        }
    }
}

template <int kBytes, int kWidth, int kThreads>
void rollouts(uint32_t d) {
    if (d < 16u / kBytes) return;
    const uint32_t lengths[] = {1, 7, 31, 32, 33, 40, 64, 77, 96};
    for (uint32_t steps : lengths)
        for (int reverse = 0; reverse < 2; ++reverse)
            for (int64_t step : {(int64_t)d, (int64_t)d + 5})
                for (uint32_t at = 0; at < steps; at += pxr::C) {
                    const uint32_t n = steps - at < (uint32_t)pxr::C ? steps - at : (uint32_t)pxr::C;
                    chunk<kBytes, kWidth, kThreads>(pxr::first_step(reverse, steps, at, n), n, steps, d, step);
                    for (uint32_t one = at; one < at + n; one += 15)  // steps that are taken one by one
                        chunk<kBytes, kWidth, kThreads>(pxr::first_step(reverse, steps, one, 1), 1, steps, d, step);
                }
}

template <int kBytes, int kWidth, int kWaves>
void kernel() {
    ++kernels;
    for (uint32_t d = 1; d <= (uint32_t)kWidth; ++d) rollouts<kBytes, kWidth, kWaves * 64>(d);            // x and y
    for (uint32_t d = 1; d <= (uint32_t)kWaves * 32; ++d) rollouts<kBytes, kWaves * 32, kWaves * 64>(d);  // z
}

}  // namespace

int main() {
#define PXR_CHECK(A, W) \
    kernel<2, A, W>();  \
    kernel<4, A, W>();
    PXR_SCAN_SHAPES(PXR_CHECK)
    if (outside || misplaced) {
        std::printf("%llu requests of %llu outside, %llu misplaced\n", (unsigned long long)outside, (unsigned long long)requests, (unsigned long long)misplaced);
        return 1;
    }
    std::printf("ok %llu %llu\n", (unsigned long long)requests, (unsigned long long)kernels);
    return 0;
}
