// How the lanes of a workgroup are dealt the steps of a chunk (linear_attention.hip): which 16 bytes of memory each of a lane's
// requests is for, in a header of its own so that a CPU test can walk all of them.
//
// A chunk is n <= 32 steps, rows of d values that lie `step` values apart.  The lanes take the rows of a tile of kWidth >= d columns in
// vectors of 16 bytes, kPerRow lanes a row, kRowsEach rows together, kCount times.  A row that ends inside a vector has its last vector moved
// back to its end, and vectors past a row's end are that one too.  A lane whose row is none of the chunk's n asks for the
// first row's instead: there is nothing behind the last chunk's rows that may be read.  Rows of fewer values than a vector
// are not asked for in vectors.
#ifndef PXR_STEPS_H
#define PXR_STEPS_H

#include <cstdint>

#ifdef __HIPCC__
#define PXR_STEPS_BOTH __host__ __device__ __forceinline__
#else
#define PXR_STEPS_BOTH inline
#endif

namespace pxr {

constexpr int C = 32;  // steps of a chunk

// The scan kernels that there are, as X(padded width of x and y, wavefronts): a wavefront has 32 columns of z.
#define PXR_SCAN_SHAPES(X) X(32, 1) X(32, 2) X(32, 4) X(64, 1) X(64, 2) X(64, 4) X(128, 2) X(128, 4) X(256, 4)

// The first of a chunk's n steps in memory, which the scan takes from position `at` on (in reverse, position p is step n_steps - 1 - p).
PXR_STEPS_BOTH int64_t first_step(bool reverse, uint32_t n_steps, uint32_t at, uint32_t n) {
    return reverse ? (int64_t)(n_steps - at - n) : (int64_t)at;
}

template <int kBytes, int kWidth, int kThreads>
struct Dealt {
    static constexpr uint32_t N = 16 / kBytes, kPerRow = kWidth / N, kCount = (C * kPerRow + kThreads - 1) / kThreads;
    static constexpr uint32_t kRowsEach = kThreads / kPerRow;  // rows that the lanes take together
    static_assert(kThreads % kPerRow == 0);

    static PXR_STEPS_BOTH uint32_t row(uint32_t thread) { return thread / kPerRow; }
    static PXR_STEPS_BOTH uint32_t col(uint32_t thread) { return thread % kPerRow * N; }
    static PXR_STEPS_BOTH uint32_t place_in_row(uint32_t col, uint32_t d) { return d < N ? 0u : col < d - N ? col : d - N; }
    // Of a lane's first request, in values from the chunk's first one.
    static PXR_STEPS_BOTH int64_t offset(uint32_t row, uint32_t col, uint32_t d, int64_t step) { return (int64_t)row * step + place_in_row(col, d); }
    // Where its request i is, 1 <= n <= C.  `from` = the chunk's first value: a pointer, or a number that counts values.
    template <class At>
    static PXR_STEPS_BOTH At request(At from, uint32_t i, uint32_t n, uint32_t row, uint32_t col, uint32_t d, int64_t step, int64_t offset) {
        At p = from + (int64_t)(i * kRowsEach) * step + offset;
        // (a whole chunk has a row for every lane, unless the lanes take more rows together than a chunk has)
        if ((n < (uint32_t)C || kRowsEach * kCount > (uint32_t)C) && row + i * kRowsEach >= n) p = from + place_in_row(col, d);
        return p;
    }
};

}  // namespace pxr

#endif
