// A learner's update with its singular values pushed towards one (pxr_orthogonalise in include/pxr.h).  gfx950 only.
//
//   X_0 = x / (|x| + eps),  |x| the Frobenius norm;   X_{k+1} = a X_k + (b A + c A^2) X_k,  A = X_k X_k^T
//
// with X [s,l] the update or, where it has more rows than columns, its transpose: s <= l.  On a singular value t a step is the polynomial a t + b t^3 + c t^5.  Three products
// a step, the first two symmetric (half of their tiles):
//   A = X X^T,   B = a 1 + b A + c A A,   X <- B X
//
// All on the matrix cores, in fp16 operands and fp32 sums.  A value of X, A and B is held as two fp16 parts, the value rounded and what that left out, 22 bits and more
// together, and a product is three: hi hi + hi lo + lo hi; lo lo is 2^-22 of it and left out.  fp16 has the bits that bfloat16 has not (two parts of it are 16 bits: an
// update whose singular values lie far apart loses its small ones) and its range does not matter: a singular value of X_k, and so every value of X, A and B, has a
// bound that follows from the coefficients alone, and each of the three is held times a power of two that puts that bound just below fp16's largest.
//
// Large matrices are bound by the matrix cores, and those by the power that they may draw: 4096 x 4096 in 4.3 ms, 0.95 PFLOP/s of fp16 where a library's product of 8192 reaches 1.16 (an
// update's product 395 us, 60 % of its clocks in matrix instructions).  Below about 1000 x 1000 it is the chain of launches, 17 to 27 of 5 to 9 us each; matrices that fit LDS have one.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "pxr_internal.h"

namespace pxr {
namespace {

typedef _Float16 half;
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr uint32_t kThreads = 256;
constexpr uint32_t kPad = 128;       // rows and columns of the matrices in the workspace come in multiples of it, a large tile's side; what is behind the matrix is zeros
constexpr uint32_t kNormParts = 512; // of a matrix whose squares are summed, at most (1024 and 2048: within 1 % either way)
constexpr uint32_t kNormColumns = 1024;
// Values of the summed axis in one chain of sums; the chains' results are added up.  (Of one chain of all, 4096 x 4096 in fp32 are off by 3.2e-6 of their norm, by 1.2e-6 of these, and in plain fp32
// by 4.8e-6; in bfloat16 they take 4285 us instead of
// 4235.  Chains of 256: 1.0e-6, 4319 us.)
constexpr uint32_t kChain = 512;
constexpr uint32_t depth_of(int M) { return M == 2 ? 32u : 64u; }  // values of the summed axis that a stage in LDS has: 32 KB either way (32 of small tiles: 1024 x 1024 279 us, 64 245)

__host__ __device__ constexpr uint32_t padded(uint32_t n) { return (n + kPad - 1u) / kPad * kPad; }

// Two planes of fp16 parts of a batch of matrices in the workspace: [plane][matrix][rows][cols].
struct Planes {
    half* hi;
    size_t plane, matrix;
    uint32_t row;
    __host__ __device__ half* at(uint32_t p, uint32_t m) const { return hi + p * plane + m * matrix; }
};

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __bf16* p) { return (float)*p; }

struct Prepare {
    const void* x;
    int64_t x_matrix, x_row;
    uint32_t rows, cols, parts;
    double* sums;  // [matrices][parts]
    Planes to;
    float eps, scale;
};

// The power of two of a row's quads of values, at most a workgroup's threads; and units of 1024 values, or of rows side by side.
__host__ __device__ inline uint32_t quads_shift(uint32_t cols) {
    uint32_t shift = 0;
    while ((1u << shift) < kThreads && (4u << shift) < cols) ++shift;
    return shift;
}
__host__ __device__ inline uint64_t norm_units(uint32_t rows, uint32_t cols) {
    const uint32_t together = kThreads >> quads_shift(cols);
    return (uint64_t)((rows + together - 1u) / together) * ((cols + kNormColumns - 1u) / kNormColumns);
}

// Squares in 64 bits: those of fp32 values neither overflow nor vanish.
template <class T>
__global__ __launch_bounds__(kThreads) void square_sums_kernel(const Prepare a) {
    __shared__ double shared[kThreads / 64];
    const uint32_t part = blockIdx.x, matrix = blockIdx.y;
    const T* x = static_cast<const T*>(a.x) + (int64_t)matrix * a.x_matrix;
    // a workgroup has 1024 values of a row, or of as many rows as their quads of values (padded to a power of two) take; four such units together
    const uint32_t shift = quads_shift(a.cols), r_in = threadIdx.x >> shift, c_in = (threadIdx.x & ((1u << shift) - 1u)) * 4u;
    const uint32_t together = kThreads >> shift, per_row = (a.cols + kNormColumns - 1u) / kNormColumns;
    const uint64_t units = norm_units(a.rows, a.cols);
    double sum = 0.0;
    for (uint64_t first = part; first < units; first += 4ull * a.parts) {
        T v[4][4];
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n) {
            const uint64_t u = first + (uint64_t)n * a.parts;
            const uint32_t block = (uint32_t)(u / per_row), r = block * together + r_in, c = (uint32_t)(u - (uint64_t)block * per_row) * kNormColumns + c_in;
            const bool there = u < units && r < a.rows && c < a.cols;
            const T* p = x + (there ? (int64_t)r * a.x_row + c : 0);
            if (there && c + 4u <= a.cols) {
                __builtin_memcpy(v[n], p, sizeof(v[n]));  // (at the address of any value)
            } else {
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) v[n][e] = there && c + e < a.cols ? p[e] : (T)0.0f;
            }
        }
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n)
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) sum = __builtin_fma((double)load1(v[n] + e), (double)load1(v[n] + e), sum);
    }
#pragma unroll
    for (uint32_t m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m);
    if ((threadIdx.x & 63u) == 0) shared[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.sums[(size_t)matrix * a.parts + part] = shared[0] + shared[1] + shared[2] + shared[3];
}

__device__ __forceinline__ void split(float v, half& hi, half& lo) {
    hi = (half)v;  // round to nearest even
    lo = (half)(v - (float)hi);
}

// Divided by the norm and split, 64 x 64 values a workgroup, transposed where the update has more rows than columns.
template <class T>
__global__ __launch_bounds__(kThreads) void split_kernel(const Prepare a) {
    __shared__ float tile[64][65];
    __shared__ double total;
    const uint32_t matrix = blockIdx.z;
    double sum = 0.0;
    if (threadIdx.x < 64u) {
        for (uint32_t p = threadIdx.x; p < a.parts; p += 64u) sum += a.sums[(size_t)matrix * a.parts + p];
#pragma unroll
        for (uint32_t m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m);
        if (threadIdx.x == 0) total = sum;
    }
    // the tile of the update: rows r0.., columns c0..
    const bool tall = a.rows > a.cols;
    const uint32_t r0 = (tall ? blockIdx.x : blockIdx.y) * 64u, c0 = (tall ? blockIdx.y : blockIdx.x) * 64u;
    const T* x = static_cast<const T*>(a.x) + (int64_t)matrix * a.x_matrix;
    for (uint32_t i = threadIdx.x; i < 64u * 64u; i += kThreads) {
        const uint32_t r = i >> 6, c = i & 63u;
        const float v = r0 + r < a.rows && c0 + c < a.cols ? load1(x + (int64_t)(r0 + r) * a.x_row + (c0 + c)) : 0.0f;
        tile[tall ? c : r][tall ? r : c] = v;
    }
    __syncthreads();
    const double over = (double)a.scale / (sqrt(total) + (double)a.eps);
    half *hi = a.to.at(0, matrix), *lo = a.to.at(1, matrix);
    for (uint32_t i = threadIdx.x; i < 64u * 8u; i += kThreads) {
        const uint32_t r = i >> 3, c = (i & 7u) * 8u;
        f16x8 h, l;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            half p, q;
            split((float)((double)tile[r][c + e] * over), p, q);
            h[e] = p;
            l[e] = q;
        }
        const size_t at = (size_t)(blockIdx.y * 64u + r) * a.to.row + blockIdx.x * 64u + c;
        *reinterpret_cast<f16x8*>(hi + at) = h;
        *reinterpret_cast<f16x8*>(lo + at) = l;
    }
}

// ---- products

enum { kGram, kPoly, kUpdate, kLast };

struct Product {
    Planes a, b, to;     // kGram: X, X -> A;  kPoly: A, A -> B;  kUpdate: B, X -> X;  kLast: B, X -> out
    uint32_t depth;      // the summed axis, a multiple of 64
    uint32_t tiles_i, tiles_j;
    uint32_t whole, splits, steps_each;  // tiles from number `whole` on are cut along the summed axis: into `splits` parts of steps_each steps of depth_of(M)
    float* partial;      // [matrices][splits][tiles - whole][tile][tile]
    float scale;         // of the sums
    float c0, c1;        // kPoly: on the diagonal; times A's held values
    uint32_t s;          // rows with a diagonal
    void* out;
    int64_t out_matrix, out_row;
    uint32_t rows, cols, transposed, bf16;
};

// Tiles of a symmetric product: those of its lower triangle, row by row.
__device__ __forceinline__ void triangle(uint32_t t, uint32_t& i, uint32_t& j) {
    i = (uint32_t)((__builtin_sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while (i * (i + 1u) / 2u > t) --i;
    while ((i + 1u) * (i + 2u) / 2u <= t) ++i;
    j = t - i * (i + 1u) / 2u;
}

// The order in which tiles are taken: workgroups go to the eight dies in turn, so a die has a run of this order, and tiles that follow each other in it read the same
// rows and columns: bands of kBand rows of tiles, column by column.
constexpr uint32_t kDies = 8, kBand = 4;
__host__ __device__ constexpr uint32_t on_dies(uint32_t groups) { return (groups + kDies - 1u) / kDies * kDies; }
__device__ __forceinline__ uint32_t in_order(uint32_t group, uint32_t groups) { return group % kDies * (groups / kDies) + group / kDies; }
__device__ __forceinline__ void of_band(uint32_t t, uint32_t rows, uint32_t cols, uint32_t& i, uint32_t& j) {
    const uint32_t band = t / (kBand * cols), r = t - band * kBand * cols, high = min(kBand, rows - band * kBand);
    j = r / high;
    i = band * kBand + r - j * high;
}
// Of a symmetric product's lower triangle of tiles.  `whole` bands have 4 columns of tiles each for every band before them, and a triangle; rows behind the last whole band come one by
// one.
__device__ __forceinline__ void of_triangle(uint32_t t, uint32_t rows, uint32_t& i, uint32_t& j) {
    const auto before = [](uint32_t band) { return 8u * band * band + 2u * band; };
    const uint32_t whole = rows / kBand;
    if (t >= before(whole)) return triangle(t - before(whole) + whole * kBand * (whole * kBand + 1u) / 2u, i, j);
    uint32_t band = (uint32_t)__builtin_sqrtf((float)t * 0.125f);
    while (before(band) > t) --band;
    while (before(band + 1u) <= t) ++band;
    const uint32_t r = t - before(band), left = band * kBand;
    if (r < left * kBand) {
        j = r / kBand;
        i = left + r % kBand;
    } else {
        triangle(r - left * kBand, i, j);
        i += left;
        j += left;
    }
}

// A tile's operand in LDS, one plane, kDepth values deep.  Along: rows of 64 or 128 bytes, chunks of 8 values, chunk c of row r at place c ^ (r / 4 % 4) or c ^ (r / 2 % 8): the 16 rows whose chunks of
// one c are read together lie in the 64 banks once each.  Across (the summed axis is the rows'): rows of `kSide` values; the transposing read takes 32 values of four rows together, chunks of them at place
// c ^ 4 (k % 4), or where two rows are 256 bytes c ^ 4 (k / 2 % 2).  The requests that write LDS put a wavefront's lanes side by side, so it is the addresses that they ask for which are
// exchanged.  (Exchanged for 32 banks, half of the LDS' cycles were conflicts: 4096 x 4096 bfloat16 5250 us.)
template <int kSide, bool kAcross>
struct Operand {
    static constexpr uint32_t kDepth = depth_of(kSide / 64), kChunks = kSide * kDepth / 8;  // of 16 bytes, in a plane
    static __device__ __forceinline__ uint32_t turn(uint32_t row) {
        if (!kAcross) return kDepth == 32u ? row >> 2 & 3u : row >> 1 & 7u;
        return kSide == 128 ? (row & 3u) << 2 : (row >> 1 & 1u) << 2;
    }
    // Which value chunk number i of the plane is: row and column in the tile.
    static __device__ __forceinline__ void place(uint32_t i, uint32_t& row, uint32_t& col) {
        if (kAcross) {
            row = i / (kSide / 8);
            col = ((i % (kSide / 8)) ^ turn(row)) * 8u;
        } else {
            row = i / (kDepth / 8u);
            col = ((i % (kDepth / 8u)) ^ turn(row)) * 8u;
        }
    }
    // Eight values of the summed axis, 16 k + 8 h .. + 7, of line lane % 32 from `line` on, of both planes.
    static __device__ __forceinline__ void fragments(const half* planes, uint32_t line, uint32_t k, uint32_t lane, f16x8 (&f)[2]) {
        const uint32_t h = lane >> 5;
        if constexpr (kAcross) {
            // The transposing read: lane i of 16 gives the address of four columns of row i / 4 and gets four rows of column i.  Before its builtin the compiler waits for
            // every request that writes LDS, those of the stages ahead too, so it is written out, with a wait of its own.
            const uint32_t i = lane & 15u, row = 16u * k + 8u * h + (i >> 2), col = line + (lane & 16u) + 4u * (i & 3u);
            const half* p = planes + row * kSide + (((col >> 3) ^ turn(row)) << 3) + (col & 7u);  // (four rows on: turned alike)
            const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const half*)p;
            s16x4 q[4];
            asm volatile(
                "ds_read_b64_tr_b16 %0, %4\n\t"
                "ds_read_b64_tr_b16 %1, %4 offset:%5\n\t"
                "ds_read_b64_tr_b16 %2, %4 offset:%6\n\t"
                "ds_read_b64_tr_b16 %3, %4 offset:%7\n\t"
                "s_waitcnt lgkmcnt(0)"
                : "=&v"(q[0]), "=&v"(q[1]), "=&v"(q[2]), "=&v"(q[3])
                : "v"(at), "n"(4 * kSide * 2), "n"(kSide * kDepth * 2), "n"(kSide * kDepth * 2 + 4 * kSide * 2)
                : "memory");
            f[0] = __builtin_bit_cast(f16x8, __builtin_shufflevector(q[0], q[1], 0, 1, 2, 3, 4, 5, 6, 7));
            f[1] = __builtin_bit_cast(f16x8, __builtin_shufflevector(q[2], q[3], 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const uint32_t row = line + (lane & 31u);
#pragma unroll
            for (uint32_t plane = 0; plane < 2; ++plane)
                f[plane] = *reinterpret_cast<const f16x8*>(planes + plane * kSide * kDepth + row * kDepth + (((2u * k + h) ^ turn(row)) << 3));
        }
    }
};

// Four values of a row leave: to the planes, or as the update's own (row and column of X, which has rows of the update's shorter side).
template <bool kPolynomial>
__device__ __forceinline__ void put_planes(const Product& p, const half* ah, const half* al, half* th, half* tl, uint32_t row, uint32_t col, f32x4 v) {
    if constexpr (kPolynomial) {
        const f16x4 hi = *reinterpret_cast<const f16x4*>(ah + (size_t)row * p.a.row + col), lo = *reinterpret_cast<const f16x4*>(al + (size_t)row * p.a.row + col);
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) v[e] = __builtin_fmaf((float)hi[e] + (float)lo[e], p.c1, v[e]) + (row == col + e && row < p.s ? p.c0 : 0.0f);
    }
    f16x4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        half h, l;
        split(v[e], h, l);
        hi[e] = h;
        lo[e] = l;
    }
    *reinterpret_cast<f16x4*>(th + (size_t)row * p.to.row + col) = hi;
    *reinterpret_cast<f16x4*>(tl + (size_t)row * p.to.row + col) = lo;
}

template <class T>
__device__ __forceinline__ void put_values(T* to, f32x4 v, uint32_t n) {
    T w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (T)v[e];  // round to nearest even
    if (n >= 4u) {
        __builtin_memcpy(to, w, sizeof(w));  // (at the address of any value)
        return;
    }
#pragma unroll
    for (uint32_t e = 0; e < 3; ++e)
        if (e < n) to[e] = w[e];
}

// `row`, `col`: of the update itself.
__device__ __forceinline__ void put_out(const Product& p, uint32_t matrix, uint32_t row, uint32_t col, f32x4 v) {
    if (row >= p.rows || col >= p.cols) return;
    const int64_t at = (int64_t)matrix * p.out_matrix + (int64_t)row * p.out_row + col;
    if (p.bf16)
        put_values(static_cast<__bf16*>(p.out) + at, v, p.cols - col);
    else
        put_values(static_cast<float*>(p.out) + at, v, p.cols - col);
}

// A tile of 64 M x 64 M values by four wavefronts, 2 x 2, each 32 M x 32 M.  Two stages in LDS, one that is worked on and one on its way, 64 KB: two workgroups a compute unit, and one's matrix
// instructions run while the other waits.  (Three and four stages of large tiles, one workgroup: 4096 x 4096 4710 and 4740 us, with two 4260; of small ones 1000 x 4000 424 and 423, 383.)
// G groups of four wavefronts have the same tile and every Gth step of the summed axis each.
template <int kKind, int M, int G>
__global__ __launch_bounds__(kThreads * G) void product_kernel(const Product p) {
    constexpr int kSide = 64 * M;
    constexpr uint32_t kDepth = depth_of(M);
    constexpr bool kSym = kKind <= kPoly;
    typedef Operand<kSide, false> OpA;
    typedef Operand<kSide, !kSym> OpB;
    constexpr uint32_t kPlane = kSide * kDepth, kStage = 4 * kPlane;  // halves: A hi, A lo, B hi, B lo
    __shared__ __align__(16) half stages_of[G][2][kStage];
    const uint32_t lane = threadIdx.x & 63u, of_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = of_all & 3u, group = G == 1 ? 0u : of_all >> 2, matrix = blockIdx.z;
    half(&stage)[2][kStage] = stages_of[group];
    // (whole tiles and parts of tiles each in their own order: every die has as many of both)
    const uint32_t tiles = kSym ? p.tiles_i * (p.tiles_i + 1u) / 2u : p.tiles_i * p.tiles_j, cut = tiles - p.whole, of_whole = on_dies(p.whole);
    const bool partly = blockIdx.x >= of_whole;
    const uint32_t place = partly ? in_order(blockIdx.x - of_whole, gridDim.x - of_whole) : in_order(blockIdx.x, of_whole);
    if (place >= (partly ? cut * p.splits : p.whole)) return;
    const uint32_t part = partly ? place / cut : 0u, tile = partly ? p.whole + place - part * cut : place;
    uint32_t ti, tj;
    if (kSym)
        of_triangle(tile, p.tiles_i, ti, tj);
    else
        of_band(tile, p.tiles_i, p.tiles_j, ti, tj);
    const uint32_t i0 = ti * kSide, j0 = tj * kSide;
    // each wavefront asks for every fourth run of 64 chunks of each plane
    constexpr uint32_t kRuns = OpA::kChunks / 64 / 4;
    const half *a_from[kRuns], *b_from[kRuns];
    const uint32_t k_first = (part * p.steps_each + group) * kDepth;
#pragma unroll
    for (uint32_t n = 0; n < kRuns; ++n) {
        uint32_t row, col;
        OpA::place((n * 4u + wave) * 64u + lane, row, col);
        a_from[n] = p.a.at(0, matrix) + (size_t)(i0 + row) * p.a.row + k_first + col;
        OpB::place((n * 4u + wave) * 64u + lane, row, col);
        b_from[n] = p.b.at(0, matrix) + (kSym ? (size_t)(j0 + row) * p.b.row + k_first + col : (size_t)(k_first + row) * p.b.row + j0 + col);
    }
    const size_t b_step = kSym ? G * kDepth : (size_t)G * kDepth * p.b.row;
    const auto ask = [&](half* to) {
        typedef const __attribute__((address_space(1))) void* global;
        typedef __attribute__((address_space(3))) void* shared;
#pragma unroll
        for (uint32_t n = 0; n < kRuns; ++n)
#pragma unroll
            for (uint32_t plane = 0; plane < 2; ++plane) {
                __builtin_amdgcn_global_load_lds((global)(a_from[n] + plane * p.a.plane), (shared)(to + plane * kPlane + (n * 4u + wave) * 512u), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((global)(b_from[n] + plane * p.b.plane), (shared)(to + (2 + plane) * kPlane + (n * 4u + wave) * 512u), 16, 0, 0);
            }
#pragma unroll
        for (uint32_t n = 0; n < kRuns; ++n) {
            a_from[n] += G * kDepth;
            b_from[n] += b_step;
        }
    };
    f32x16 acc[M][M], whole[M][M];  // a chain's sums, and those of the chains before it
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < M; ++j) acc[i][j] = whole[i][j] = (f32x16)0.0f;
    const uint32_t row0 = (wave >> 1) * 32 * M, col0 = (wave & 1u) * 32 * M;
    const uint32_t left = p.depth / kDepth - part * p.steps_each, all_steps = partly ? min(p.steps_each, left) : left, steps = (all_steps + G - 1u - group) / G;
    if (steps) ask(stage[0]);
    constexpr uint32_t kTogether = kChain / kDepth;
    for (uint32_t first = 0; first < steps; first += kTogether) {
        const uint32_t last = min(steps, first + kTogether);
#pragma nounroll
        for (uint32_t k = first; k < last; ++k) {
            // this stage is there, and the values that were read of the other one have been used
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (k + 1u < steps) ask(stage[(k + 1u) & 1u]);
            const half* from = stage[k & 1u];
#pragma unroll
            for (uint32_t kk = 0; kk < kDepth / 16; ++kk) {
                f16x8 a[M][2], b[M][2];
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    OpA::fragments(from, row0 + 32 * i, kk, lane, a[i]);
                    OpB::fragments(from + 2 * kPlane, col0 + 32 * i, kk, lane, b[i]);
                }
#pragma unroll
                for (int i = 0; i < M; ++i)
#pragma unroll
                    for (int j = 0; j < M; ++j) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][1], b[j][0], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][0], b[j][1], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][0], b[j][0], acc[i][j], 0, 0, 0);
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < M; ++i)
#pragma unroll
            for (int j = 0; j < M; ++j) {
                whole[i][j] += acc[i][j];
                acc[i][j] = (f32x16)0.0f;
            }
    }
    // (A group that has a step less: the barrier of the others' last one.  Not a way out of the middle of the loop: behind such a one the compiler has left out the wait between a matrix instruction
    // and the first use of its result.)
    if (G > 1 && steps < (all_steps + G - 1u) / G) __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < M; ++j) acc[i][j] = whole[i][j];
    if constexpr (G > 1) {  // the groups' sums, in their order
        constexpr uint32_t kEach = M * M * 16;
        float* const sums = reinterpret_cast<float*>(&stages_of[0][0][0]) + wave * 64u + lane;
        __syncthreads();
        if (group)
#pragma unroll
            for (int i = 0; i < M; ++i)
#pragma unroll
                for (int j = 0; j < M; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) sums[((group - 1u) * kEach + (i * M + j) * 16u + r) * kThreads] = acc[i][j][r];
        __syncthreads();
        if (group == 0)
#pragma unroll
            for (uint32_t g = 0; g + 1u < G; ++g)
#pragma unroll
                for (int i = 0; i < M; ++i)
#pragma unroll
                    for (int j = 0; j < M; ++j)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[i][j][r] += sums[(g * kEach + (i * M + j) * 16u + r) * kThreads];
    }
    // a lane has column lane % 32 and rows 8 (r / 4) + 4 (lane / 32) + r % 4 of every 32 x 32
    const uint32_t down = 4u * (lane >> 5), across = lane & 31u;
    if (kSym && partly) {
        if (group) return;
        float* to = p.partial + (((size_t)matrix * p.splits + part) * cut + tile - p.whole) * (kSide * kSide);
#pragma unroll
        for (int i = 0; i < M; ++i)
#pragma unroll
            for (int j = 0; j < M; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    to[(row0 + 32 * i + 8 * (r >> 2) + down + (r & 3)) * kSide + col0 + 32 * j + across] = acc[i][j][r];
        return;
    }
    // Through LDS, 64 rows of the tile at a time, so that rows leave in whole lines; of a symmetric product the mirrored tile too.
    float* const pass = reinterpret_cast<float*>(&stages_of[0][0][0]);
    const half *ah = p.a.at(0, matrix), *al = p.a.at(1, matrix);
    half *th = p.to.at(0, matrix), *tl = p.to.at(1, matrix);
    const auto leave = [&](auto turned, uint32_t part64) {
        constexpr bool kTurned = decltype(turned)::value;
        constexpr uint32_t kRow = kTurned ? 64u + 4u : kSide + 4u, kRows = kTurned ? kSide : 64u, kQuads = (kTurned ? 64u : kSide) / 4u;
        __syncthreads();
        if (group == 0 && (M == 1 || wave >> 1 == part64)) {
            const uint32_t row_in = M == 1 ? row0 : 0u;
#pragma unroll
            for (int i = 0; i < M; ++i)
#pragma unroll
                for (int j = 0; j < M; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t row = row_in + 32 * i + 8 * q + down, col = col0 + 32 * j + across;
                        if constexpr (kTurned) {
                            *reinterpret_cast<f32x4*>(pass + col * kRow + row) = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                        } else {
#pragma unroll
                            for (int r = 0; r < 4; ++r) pass[(row + r) * kRow + col] = acc[i][j][4 * q + r];
                        }
                    }
        }
        __syncthreads();
        for (uint32_t n = threadIdx.x; n < kRows * kQuads; n += kThreads * G) {
            const uint32_t r = n / kQuads, c = n % kQuads * 4u;
            const f32x4 v = *reinterpret_cast<const f32x4*>(pass + r * kRow + c) * p.scale;
            const uint32_t row = kTurned ? j0 + r : i0 + part64 * 64u + r, col = kTurned ? i0 + part64 * 64u + c : j0 + c;
            if constexpr (kKind == kLast)
                put_out(p, matrix, row, col, v);
            else
                put_planes<kKind == kPoly>(p, ah, al, th, tl, row, col, v);
        }
    };
#pragma unroll
    for (uint32_t part64 = 0; part64 < M; ++part64) {
        if (kKind != kLast || !p.transposed) leave(std::false_type{}, part64);
        if (kKind == kLast ? p.transposed : kSym && ti != tj) leave(std::true_type{}, part64);
    }
}

// The tiles of a symmetric product whose summed axis was cut: the parts' sums in their order, 16 x 64 values of a tile a workgroup.
template <int kKind, int M>
__global__ __launch_bounds__(kThreads) void join_kernel(const Product p) {
    constexpr uint32_t kSide = 64 * M, kValues = kSide * kSide;
    __shared__ float turned[64][17];
    const uint32_t cut = p.tiles_i * (p.tiles_i + 1u) / 2u - p.whole, tile = blockIdx.x / (4u * M * M), place = blockIdx.x % (4u * M * M), matrix = blockIdx.z;
    uint32_t ti, tj;
    of_triangle(p.whole + tile, p.tiles_i, ti, tj);
    const uint32_t row_in = place / M * 16u, col_in = place % M * 64u, r = threadIdx.x >> 4, c = (threadIdx.x & 15u) * 4u;
    const float* from = p.partial + ((size_t)matrix * p.splits * cut + tile) * kValues + (row_in + r) * kSide + col_in + c;
    f32x4 v = (f32x4)0.0f;
#pragma unroll 8
    for (uint32_t s = 0; s < p.splits; ++s) v += *reinterpret_cast<const f32x4*>(from + (size_t)s * cut * kValues);
    v *= p.scale;
    const half *ah = p.a.at(0, matrix), *al = p.a.at(1, matrix);
    half *th = p.to.at(0, matrix), *tl = p.to.at(1, matrix);
    const uint32_t row0 = ti * kSide + row_in, col0 = tj * kSide + col_in;
    put_planes<kKind == kPoly>(p, ah, al, th, tl, row0 + r, col0 + c, v);
    if (ti == tj) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) turned[c + e][r] = v[e];
    __syncthreads();
    const uint32_t row = threadIdx.x >> 2, col = (threadIdx.x & 3u) * 4u;
    const f32x4 w{turned[row][col], turned[row][col + 1], turned[row][col + 2], turned[row][col + 3]};
    put_planes<kKind == kPoly>(p, ah, al, th, tl, col0 + row, row0 + col, w);
}

// ---- small matrices: one workgroup has one from its reading to the result, X, A and then B in LDS

struct Factors {
    float gram, poly, linear, diagonal, update;  // of the three products' sums, and of A and 1 in B
};

struct Small {
    const void* x;
    void* out;
    int64_t x_matrix, x_row, out_matrix, out_row;
    uint32_t rows, cols, s, l, sp, lp, n_steps;
    float eps, held;
    Factors steps[64];
};

constexpr uint32_t kSmallThreads = 512, kSmallWaves = kSmallThreads / 64;
constexpr uint32_t kLds = 160 * 1024;
constexpr uint32_t up64(uint32_t n) { return (n + 63u) / 64u * 64u; }
constexpr uint32_t up32(uint32_t n) { return (n + 31u) / 32u * 32u; }
// Rows lie 16 bytes apart from a multiple of 64, so that those of eight lanes lie in different banks.
constexpr uint32_t small_row(uint32_t n) { return n + 8u; }
constexpr uint32_t small_lds(uint32_t sp, uint32_t lp) { return 64u + 4u * sp * (small_row(lp) + small_row(sp)); }
bool is_small(uint32_t s, uint32_t l) {
    const uint32_t sp = up32(s), lp = up32(l);
    // (the tiles of the three products that a wavefront holds at once: see the kernel)
    return sp <= 128u && lp <= 2048u && small_lds(sp, lp) <= kLds && (sp / 32u) * (lp / 32u) <= 5u * kSmallWaves;
}

__device__ __forceinline__ f16x8 along(const half* plane, uint32_t row, uint32_t stride, uint32_t k, uint32_t lane) {
    return *reinterpret_cast<const f16x8*>(plane + (row + (lane & 31u)) * stride + k + 8u * (lane >> 5));
}
__device__ __forceinline__ f16x8 across(const half* plane, uint32_t k, uint32_t stride, uint32_t col, uint32_t lane) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const uint32_t i = lane & 15u;
    const half* p = plane + (k + 8u * (lane >> 5) + (i >> 2)) * stride + col + (lane & 16u) + 4u * (i & 3u);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * stride));
    return __builtin_bit_cast(f16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A number that is the same in all lanes, as one that the compiler does not know.
__device__ __forceinline__ uint32_t again(uint32_t v) {
    v = __builtin_amdgcn_readfirstlane(v);
    asm volatile("" : "+s"(v));
    return v;
}

// The sum over `depth` values (a multiple of 32) of a 32 x 32 tile.  Two chains of sums, and 32 values' operands asked for together, so that one instruction does not wait for the last
// one's result.  A lane has column lane % 32 of the tile and rows 8 (r / 4) + 4 (lane / 32) + r % 4.  kAcross: the rows are a's columns.
template <bool kAcross>
__device__ __forceinline__ f32x16 small_product(const half* a, uint32_t a_plane, uint32_t row, uint32_t a_stride, const half* b, uint32_t b_plane, uint32_t col, uint32_t b_stride, uint32_t depth,
                                                uint32_t lane) {
    f32x16 sum[2];
    const auto add = [&](uint32_t k, const f32x16& from0, const f32x16& from1) {
        f16x8 x[2][2], y[2][2];
#pragma unroll
        for (uint32_t n = 0; n < 2; ++n)
#pragma unroll
            for (uint32_t plane = 0; plane < 2; ++plane) {
                x[n][plane] = kAcross ? across(a + plane * a_plane, k + 16u * n, a_stride, row, lane) : along(a + plane * a_plane, row, a_stride, k + 16u * n, lane);
                y[n][plane] = along(b + plane * b_plane, col, b_stride, k + 16u * n, lane);
            }
        sum[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[0][0], y[0][1], from0, 0, 0, 0);
        sum[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[0][1], y[0][0], from1, 0, 0, 0);
        sum[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[0][0], y[0][0], sum[0], 0, 0, 0);
        sum[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[1][1], y[1][0], sum[1], 0, 0, 0);
        sum[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[1][0], y[1][1], sum[0], 0, 0, 0);
        sum[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[1][0], y[1][0], sum[1], 0, 0, 0);
    };
    add(0, (f32x16)0.0f, (f32x16)0.0f);
#pragma nounroll
    for (uint32_t k = 32; k < depth; k += 32u) add(k, sum[0], sum[1]);
    return sum[0] + sum[1];
}

// The tile's transpose, at row `col` and column `row` of a matrix in LDS: four values lie together.
__device__ __forceinline__ void small_put(half* to, uint32_t plane, uint32_t row, uint32_t stride, uint32_t col, const f32x16& v, uint32_t lane) {
    half* const at = to + (col + (lane & 31u)) * stride + row + 4 * (lane >> 5);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        f16x4 hi, lo;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            half h, l;
            split(v[4 * q + r], h, l);
            hi[r] = h;
            lo[r] = l;
        }
        *reinterpret_cast<f16x4*>(at + 8 * q) = hi;
        *reinterpret_cast<f16x4*>(at + plane + 8 * q) = lo;
    }
}

template <class T>
__global__ __launch_bounds__(kSmallThreads) void small_kernel(const Small a) {
    extern __shared__ __align__(16) unsigned char small_memory[];
    double* const sums = reinterpret_cast<double*>(small_memory);
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), matrix = blockIdx.x;
    uint32_t x_stride = small_row(a.lp), s_stride = small_row(a.sp);
    const uint32_t x_plane = a.sp * x_stride, s_plane = a.sp * s_stride;
    half* const X = reinterpret_cast<half*>(small_memory + 64);
    half* const S = X + 2 * x_plane;
    const bool tall = a.rows > a.cols;
    const T* x = static_cast<const T*>(a.x) + (int64_t)matrix * a.x_matrix;
    for (uint32_t i = threadIdx.x; i < (2 * x_plane) / 8u; i += kSmallThreads) reinterpret_cast<uint4*>(X)[i] = make_uint4(0, 0, 0, 0);
    // The update is read twice (the second time from the caches), four values of a row a lane.  One compute unit's instructions are what it costs: where a value took 40 of them, 64 x 448 values
    // took 25 us.
    const uint32_t per_row = (a.cols + 3u) / 4u, quads = a.rows * per_row, over_row = 0xFFFFFFFFu / per_row + 1u;  // (quads * per_row < 2^32: the quotient below is exact)
    const auto each = [&](auto&& use) {
        constexpr uint32_t kAhead = 4;
        for (uint32_t first = threadIdx.x; first < quads; first += kSmallThreads * kAhead) {
            T v[kAhead][4];
            uint32_t row[kAhead], col[kAhead];
#pragma unroll
            for (uint32_t n = 0; n < kAhead; ++n) {
                const uint32_t at = min(first + n * kSmallThreads, quads - 1u);
                row[n] = per_row == 1u ? at : __umulhi(at, over_row);
                col[n] = (at - row[n] * per_row) * 4u;
                const T* p = x + (int64_t)row[n] * a.x_row + col[n];
                if (col[n] + 4u <= a.cols) {
                    __builtin_memcpy(v[n], p, sizeof(v[n]));  // (at the address of any value)
                } else {
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e) v[n][e] = col[n] + e < a.cols ? p[e] : (T)0.0f;
                }
            }
#pragma unroll
            for (uint32_t n = 0; n < kAhead; ++n)
                if (first + n * kSmallThreads < quads) use(row[n], col[n], v[n]);
        }
    };
    double sum = 0.0;
    each([&](uint32_t, uint32_t, const T (&v)[4]) {
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) sum = __builtin_fma((double)load1(v + e), (double)load1(v + e), sum);
    });
#pragma unroll
    for (uint32_t m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (uint32_t w = 0; w < kSmallWaves; ++w) sum += sums[w];
    // what a value is multiplied with, as a power of two and a number in [1/2, 1): the first alone may lie outside of fp32
    const double over = (double)a.held / (sqrt(sum) + (double)a.eps);
    const int exponent = __builtin_amdgcn_frexp_exp(over);
    const float mantissa = (float)__builtin_amdgcn_frexp_mant(over);
    each([&](uint32_t r, uint32_t c, const T (&v)[4]) {
        f16x4 hi, lo;
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
            half h, l;
            split(__builtin_amdgcn_ldexpf(load1(v + e), exponent) * mantissa, h, l);
            hi[e] = h;
            lo[e] = l;
        }
        if (!tall) {  // (values behind the row's end are zeros)
            half* const at = X + r * x_stride + c;
            *reinterpret_cast<f16x4*>(at) = hi;
            *reinterpret_cast<f16x4*>(at + x_plane) = lo;
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
                if (c + e < a.cols) {
                    half* const at = X + (c + e) * x_stride + r;
                    at[0] = hi[e];
                    at[x_plane] = lo[e];
                }
        }
    });
    const uint32_t ti = a.sp / 32u, tj = a.lp / 32u;
    for (uint32_t step = 0; step < a.n_steps; ++step) {
        const Factors f = a.steps[step];
        // (the addresses of all tiles' values, formed in front of the loop over steps, would take more registers than there are)
        x_stride = again(x_stride);
        s_stride = again(s_stride);
        // A, whose tiles stay with their wavefronts
        constexpr int kSquare = 16 / kSmallWaves, kWide = 5;
        f32x16 of_a[kSquare];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kSquare; ++n) {
            const uint32_t t = again(wave + n * kSmallWaves), i = t / ti * 32u, j = t % ti * 32u;
            if (t >= ti * ti) continue;
            of_a[n] = small_product<false>(X, x_plane, i, x_stride, X, x_plane, j, x_stride, a.lp, lane) * f.gram;
            small_put(S, s_plane, i, s_stride, j, of_a[n], lane);
        }
        __syncthreads();
        // B in A's place
        f32x16 of_b[kSquare];
#pragma unroll
        for (int n = 0; n < kSquare; ++n) {
            const uint32_t t = again(wave + n * kSmallWaves), i = t / ti * 32u, j = t % ti * 32u;
            if (t >= ti * ti) continue;
            of_b[n] = small_product<false>(S, s_plane, i, s_stride, S, s_plane, j, s_stride, a.sp, lane);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t row = i + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3), col = j + (lane & 31u);
                of_b[n][r] = __builtin_fmaf(of_a[n][r], f.linear, of_b[n][r] * f.poly) + (row == col && row < a.s ? f.diagonal : 0.0f);
            }
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kSquare; ++n) {
            const uint32_t t = again(wave + n * kSmallWaves);
            if (t < ti * ti) small_put(S, s_plane, t / ti * 32u, s_stride, t % ti * 32u, of_b[n], lane);
        }
        __syncthreads();
        // X in its own place: tiles of its transpose
        f32x16 of_x[kWide];
#pragma unroll
        for (int n = 0; n < kWide; ++n) {
            const uint32_t t = again(wave + n * kSmallWaves);
            if (t < ti * tj) of_x[n] = small_product<true>(X, x_plane, t % tj * 32u, x_stride, S, s_plane, t / tj * 32u, s_stride, a.sp, lane) * f.update;
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kWide; ++n) {
            const uint32_t t = again(wave + n * kSmallWaves), i = t / tj * 32u, j = t % tj * 32u;
            if (t >= ti * tj) continue;
            if (step + 1u < a.n_steps) {
                small_put(X, x_plane, j, x_stride, i, of_x[n], lane);
                continue;
            }
            // the result, as it is, in the place of both planes
            float* const at = reinterpret_cast<float*>(X) + (i + (lane & 31u)) * x_stride + j + 4 * (lane >> 5);
#pragma unroll
            for (int q = 0; q < 4; ++q) *reinterpret_cast<f32x4*>(at + 8 * q) = f32x4{of_x[n][4 * q], of_x[n][4 * q + 1], of_x[n][4 * q + 2], of_x[n][4 * q + 3]};
        }
    }
    __syncthreads();
    T* const out = static_cast<T*>(a.out) + (int64_t)matrix * a.out_matrix;
    const float* const Y = reinterpret_cast<const float*>(X);
    for (uint32_t at = threadIdx.x; at < quads; at += kSmallThreads) {
        const uint32_t r = per_row == 1u ? at : __umulhi(at, over_row), c = (at - r * per_row) * 4u;
        f32x4 v;
        if (!tall) {
            v = *reinterpret_cast<const f32x4*>(Y + r * x_stride + c);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) v[e] = Y[min(c + e, a.sp - 1u) * x_stride + r];
        }
        put_values(out + (int64_t)r * a.out_row + c, v, a.cols - c);
    }
}

// ---- long matrices of at most 32 rows (or columns): X is read twice.  Every X_k is a product P_k X_0 with P_0 = 1, P_{k+1} = B_k P_k, and A_{k+1} = B_k A_k B_k: a sum over the long axis, steps on matrices
// of 32 x 32, and a product.  All in fp64, on its matrix cores: in fp32 this way loses the small singular values, whose squares A has from the beginning on.  |x|^2 is A's trace.  10 x 28196 in fp32: sums
// 7 us, steps 17, product 4; what is left is three launches and the chain of the steps.  32 x 200000: 32, 26 and 20, where 26 and 51 MB would take 5 and 10: the sums have a compute unit for each of 128 parts, half of
// them, because the steps' workgroup reads all of the parts' sums, 17 us of its 26 (five steps are 9).
//
// A that is carried along is off by its first roundings, 2^-53, times the square of what the steps multiply a small singular value with.  Where X has no such direction those roundings are all that A has of it; they
// may be negative, and then the steps' terms add up instead of cancelling (32 x 400 of rank 5 in fp32: off by 2e-3 after 14 steps, NaN after 20).  So the steps come in rounds, each of which forms A from X
// again: X = P X in fp64 in the workspace.  A round ends before the step in front of which its steps have multiplied by kNarrowGrowth: A is off by 2^-33 then.

constexpr uint32_t kNarrow = 32, kNarrowRow = kNarrow + 1;
constexpr uint32_t kNarrowParts = 128, kNarrowGroups = 2048;  // of a matrix, at most (32 x 200000: 256 of them 78 us, 128 76), and of all
constexpr uint32_t kNarrowAhead = 2;                          // requests of a wavefront, 16 values of the long axis each
constexpr double kNarrowGrowth = 1024.0;

typedef double f64x4 __attribute__((ext_vector_type(4)));

struct Narrow {
    const void* x;
    void* out;
    int64_t x_matrix, x_down, x_along, out_matrix, out_down, out_along;  // from one of the at most 32 rows to the next, and along them
    uint32_t s, l, parts, each, begin, end;  // each: values of the long axis of a part, a multiple of 64; begin, end: the round's steps
    double *sums, *products;  // [matrices][parts][32][32]; [matrices][32][32], of X as it is
    float eps;
    float coefficients[64][3];
};

__device__ __forceinline__ double load1(const double* p) { return *p; }
template <class O>
__device__ __forceinline__ O rounded(double v) {
    if constexpr (sizeof(O) == 8)
        return v;
    else
        return (O)(float)v;  // (to bfloat16 by way of fp32: 2^-24 more)
}

// A lane has row lane % 16 of a's 16 and column lane % 16 of b's, value lane / 16 of the summed axis' four; of the result column lane % 16 and rows 4 r + lane / 16.
__device__ __forceinline__ f64x4 product64(double a, double b, f64x4 sum) { return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, sum, 0, 0, 0); }

// A part's share of A = X X^T.  A wavefront takes 16 values of the long axis at a time, four of each row a lane.
template <class T>
__global__ __launch_bounds__(256) void narrow_sums_kernel(const Narrow a) {
    __shared__ double total[3][256][4];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), matrix = blockIdx.y, row = lane & 15u;
    const T* x = static_cast<const T*>(a.x) + (int64_t)matrix * a.x_matrix;
    const uint32_t begin = blockIdx.x * a.each, end = min(begin + a.each, a.l);
    f64x4 sum[3] = {(f64x4)0.0, (f64x4)0.0, (f64x4)0.0};
    for (uint32_t first = begin + 16u * wave; first < end; first += 64u * kNarrowAhead) {
        T v[kNarrowAhead][2][4];
        const bool whole = a.x_along == 1 && first + 64u * kNarrowAhead - 48u <= end;
#pragma unroll
        for (uint32_t n = 0; n < kNarrowAhead; ++n)
#pragma unroll
            for (uint32_t half = 0; half < 2; ++half) {
                // (of rows and places that are not there the last one's: requests without conditions do not wait for each other)
                const uint32_t r = min(row + 16u * half, a.s - 1u), p = first + 64u * n + 4u * (lane >> 4);
                const T* at = x + (int64_t)r * a.x_down;
                if (whole) {
                    __builtin_memcpy(v[n][half], at + p, sizeof(v[n][half]));  // (at the address of any value)
                } else {
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e) v[n][half][e] = at[(int64_t)min(p + e, end - 1u) * a.x_along];
                }
            }
#pragma unroll
        for (uint32_t n = 0; n < kNarrowAhead; ++n)
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
                const bool there = first + 64u * n + 4u * (lane >> 4) + e < end;
                const double lo = there && row < a.s ? (double)load1(&v[n][0][e]) : 0.0, hi = there && row + 16u < a.s ? (double)load1(&v[n][1][e]) : 0.0;
                sum[0] = product64(lo, lo, sum[0]);
                if (a.s > 16u) {
                    sum[1] = product64(hi, lo, sum[1]);
                    sum[2] = product64(hi, hi, sum[2]);
                }
            }
    }
    // the wavefronts' sums, in their order
    double* const to = a.sums + ((size_t)matrix * a.parts + blockIdx.x) * (kNarrow * kNarrow);
#pragma unroll
    for (uint32_t t = 0; t < 3; ++t)
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) total[t][threadIdx.x][r] = sum[t][r];
    __syncthreads();
    for (uint32_t n = threadIdx.x; n < 3u * 256u; n += 256u) {
        const uint32_t t = n >> 8, r = n >> 6 & 3u, from = n & 63u;
        const double v = total[t][from][r] + total[t][from + 64u][r] + total[t][from + 128u][r] + total[t][from + 192u][r];
        const uint32_t i = 4u * r + (from >> 4) + (t ? 16u : 0u), j = (from & 15u) + (t == 2u ? 16u : 0u);
        to[i * kNarrow + j] = v;
        if (t == 1u) to[j * kNarrow + i] = v;
    }
}

// The steps: a workgroup has a matrix' A, B and P in LDS.  All of its wavefronts add up the parts' sums, four of them have a tile of 16 x 16 each then.
__global__ __launch_bounds__(kNarrow * kNarrow) void narrow_steps_kernel(const Narrow a) {
    __shared__ double A[kNarrow][kNarrowRow], B[kNarrow][kNarrowRow], P[kNarrow][kNarrowRow], T[kNarrow][kNarrowRow];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), matrix = blockIdx.x, row0 = wave / 2u * 16u, col0 = wave % 2u * 16u;
    const uint32_t row = threadIdx.x / kNarrow, col = threadIdx.x % kNarrow;
    const double* from = a.sums + (size_t)matrix * a.parts * (kNarrow * kNarrow) + threadIdx.x;
    double v = 0.0;
    for (uint32_t first = 0; first < a.parts; first += 16u) {
        double some[16];
#pragma unroll
        for (uint32_t n = 0; n < 16; ++n) some[n] = first + n < a.parts ? from[(size_t)(first + n) * (kNarrow * kNarrow)] : 0.0;
#pragma unroll
        for (uint32_t n = 0; n < 16; ++n) v += some[n];
    }
    A[row][col] = v;
    __syncthreads();
    double trace = 0.0;
#pragma unroll
    for (uint32_t i = 0; i < kNarrow; ++i) trace += A[i][i];  // (zeros behind the last row)
    const double over = a.begin ? 1.0 : 1.0 / (sqrt(trace) + (double)a.eps);
    __syncthreads();
    A[row][col] = v * over * over;
    __syncthreads();
    const auto multiplied = [&](const double (&p)[kNarrow][kNarrowRow], const double (&q)[kNarrow][kNarrowRow]) {
        f64x4 sum[2] = {(f64x4)0.0, (f64x4)0.0};
#pragma unroll
        for (uint32_t k = 0; k < kNarrow; k += 4u) sum[k >> 2 & 1u] = product64(p[row0 + (lane & 15u)][k + (lane >> 4)], q[k + (lane >> 4)][col0 + (lane & 15u)], sum[k >> 2 & 1u]);
        return sum[0] + sum[1];
    };
    const auto put = [&](double (&to)[kNarrow][kNarrowRow], f64x4 tile) {
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) to[row0 + 4u * r + (lane >> 4)][col0 + (lane & 15u)] = tile[r];
    };
    const bool works = wave < 4u;
    for (uint32_t step = a.begin; step < a.end; ++step) {
        const double c0 = a.coefficients[step][0], c1 = a.coefficients[step][1], c2 = a.coefficients[step][2];
        f64x4 b = (f64x4)0.0, p = b, t = b;
        if (works) {
            b = multiplied(A, A);
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) {
                const uint32_t i = row0 + 4u * r + (lane >> 4), j = col0 + (lane & 15u);
                b[r] = c2 * b[r] + c1 * A[i][j] + (i == j ? c0 : 0.0);
            }
            put(B, b);
        }
        __syncthreads();
        if (works) {
            p = step > a.begin ? multiplied(B, P) : b;
            t = multiplied(A, B);
            put(T, t);
        }
        __syncthreads();
        if (works) {
            put(P, p);
            put(A, multiplied(T, B));
        }
        __syncthreads();
    }
    a.products[(size_t)matrix * (kNarrow * kNarrow) + threadIdx.x] = P[row][col] * over;
}

// P X: a workgroup has 64 places on the long axis, whose values each of its wavefronts reads before any of them writes its share of the rows.
template <class T, class O>
__global__ __launch_bounds__(256) void narrow_product_kernel(const Narrow a) {
    typedef const __attribute__((address_space(4))) double* Constant;  // (P's values are all lanes': scalar registers)
    const uint32_t matrix = blockIdx.y;
    const Constant P = (Constant)(a.products + (size_t)matrix * (kNarrow * kNarrow));
    const uint32_t at = blockIdx.x * 64u + (threadIdx.x & 63u), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), each = (a.s + 3u) / 4u;
    const bool there = at < a.l;
    const T* x = static_cast<const T*>(a.x) + ((int64_t)matrix * a.x_matrix + (there ? (int64_t)at * a.x_along : 0));
    O* out = static_cast<O*>(a.out) + ((int64_t)matrix * a.out_matrix + (int64_t)at * a.out_along);
    T raw[kNarrow];
#pragma unroll
    for (uint32_t k = 0; k < kNarrow; ++k) raw[k] = x[(int64_t)min(k, a.s - 1u) * a.x_down];
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (they have come, not only been asked for: out may be x)
    __syncthreads();
    if (!there) return;
#pragma unroll
    for (uint32_t k = 0; k < kNarrow; ++k) raw[k] = k < a.s ? raw[k] : (T)0.0f;
#pragma unroll 2
    for (uint32_t i = wave * each; i < min(a.s, (wave + 1u) * each); ++i) {
        double sum[4] = {};
#pragma unroll
        for (uint32_t k = 0; k < kNarrow; ++k) sum[k & 3u] = __builtin_fma(P[i * kNarrow + k], (double)load1(&raw[k]), sum[k & 3u]);
        out[(int64_t)i * a.out_down] = rounded<O>(sum[0] + sum[1] + (sum[2] + sum[3]));
    }
}

// (32 x 1200 by one workgroup in LDS 64 us, so 28; 32 x 300 26 and 27; 8 x 400 27 and 22.  10 x 28196 by the products of large matrices 139 us, so 30.)
bool is_narrow(uint32_t s, uint32_t l) { return s <= kNarrow && l > 320u; }
// Parts of 256 values, of 512 where those are more than 32: the steps' workgroup reads all of their sums.  (10 x 28196: of 256 35 us, of 512 30; 31 x 4000: 27 and 31.)
uint32_t narrow_parts(uint32_t l, uint32_t n_matrices) {
    return std::min({kNarrowParts, std::max(1u, kNarrowGroups / n_matrices), std::max(std::min((l + 255u) / 256u, 32u), (l + 511u) / 512u)});
}

// Where the rounds of steps end, and how many there are.
uint32_t narrow_rounds(const pxr_orthogonalise_desc& d, uint32_t (&ends)[64]) {
    uint32_t rounds = 0;
    double most = 1.0, grown = 1.0;
    for (uint32_t k = 0; k < d.n_steps; ++k) {
        if (grown > kNarrowGrowth) {
            ends[rounds++] = k;
            grown = 1.0;
        }
        const float* c = d.coefficients + 3 * k;
        const OrthogonaliseBounds next = orthogonalise_bounds(c[0], c[1], c[2], most);
        grown = std::max(grown, 1.0) * next.factor;  // (steps that make everything smaller make room for no more roundings)
        most = next.most;
    }
    ends[rounds++] = d.n_steps;
    return rounds;
}

float power_below(double v) { return (float)std::exp2(std::floor(std::log2(v))); }

// Bounds of the singular values, and the powers of two by which X, A and B are held: 2 less than half of fp16's largest number, so that no rounding reaches it.
constexpr double kMost = 30000.0, kLeast = 1e-9;

// How a symmetric product is cut.
struct Cut {
    int M;
    uint32_t whole, splits, steps_each;
};

struct Layout {
    uint32_t s, l, sp, lp, parts;
    Cut gram, poly;
    int update;  // M of its tiles
    size_t sums, partial, x[2], a, b, bytes;  // offsets
};

// Symmetric products take tiles of 128 x 128 from this many on, of one matrix or of several (whose last ones are not cut), unless a matrix has fewer than kLargeEach, whose tiles on the diagonal
// cost more than the larger tiles save.  Calls with 64 x 64 against 128 x 128: 4096 x 4096, 528 tiles, 4630 us, 4280; 3584, 406, 3336, 3273; 3328, 351, 2744, 2759; 2048, 136, 759, 796; eight of
// 2048, 1088, 5226, 4824; four, 544, 2527, 2635; 32 of 1024, 1152, 3143, 2999; 16, 576, 1497, 1593; 200 of 512, 10 tiles each, 3642, 3943.
constexpr uint64_t kLargeTiles = 400, kLargeBatch = 1000;
constexpr uint32_t kLargeEach = 32;
// A product of no more workgroups than compute units has two groups of wavefronts in each (at twice that many workgroups: 1300 x 1300 310 us, 290 without).
constexpr uint64_t kFewGroups = 256;
constexpr int kGroups = 2;
constexpr uint32_t kJoinSteps = 6;  // that take as long as a join_kernel (4 within 2 %; 9: 200 x 1000 127 us, 114 so)
constexpr uint64_t kPlaces = 512;  // workgroups that a device has room for at once, two on a compute unit

uint32_t tiles_of(uint32_t n, int M) { return (n + 64u * M - 1u) / (64u * M); }
uint32_t triangle_of(uint32_t s, int M) { return tiles_of(s, M) * (tiles_of(s, M) + 1u) / 2u; }

// The steps that a wavefront takes one after the other.
uint32_t in_turn(uint32_t steps, uint64_t workgroups) { return workgroups <= kFewGroups ? (steps + kGroups - 1u) / kGroups : steps; }

// Tiles that do not fill the places, and those that are left when the others have filled them some times (4096 x 4096: 16 of 528; as whole ones 5025 us, 4560 so), are cut along the summed axis, into
// parts of 256 values at least (of 512 or 1024: 200 x 5000 143 and 169 us, 133 so).  Tiles that fill no place twice are cut only where a part takes kJoinSteps steps less than the whole: 1024 x 1024
// in three parts 226 us, in one 198; 700 x 2000 in one 227, in seven 200; 200 x 1500 in one 151, in five 119.
Cut cut_of(uint32_t s, uint32_t depth, uint32_t n_matrices) {
    Cut c{};
    c.M = triangle_of(s, 2) >= kLargeEach && triangle_of(s, 2) * (uint64_t)n_matrices >= (n_matrices == 1u ? kLargeTiles : kLargeBatch) ? 2 : 1;
    const uint32_t tiles = triangle_of(s, c.M), steps = (depth + depth_of(c.M) - 1u) / depth_of(c.M);
    const uint64_t all = (uint64_t)tiles * n_matrices;
    c.whole = all < kPlaces ? 0u : n_matrices == 1u ? (uint32_t)(tiles / kPlaces * kPlaces) : tiles;
    const uint64_t left = (uint64_t)(tiles - c.whole) * n_matrices;
    c.splits = left ? (uint32_t)std::max<uint64_t>(1u, std::min<uint64_t>(steps / (256u / depth_of(c.M)), kPlaces / left)) : 1u;
    c.steps_each = (steps + c.splits - 1u) / c.splits;
    if (c.whole == 0u && in_turn(steps, left) < in_turn(c.steps_each, left * c.splits) + kJoinSteps) c.steps_each = steps;
    c.splits = (steps + c.steps_each - 1u) / c.steps_each;
    if (c.splits == 1u) c.whole = tiles;
    return c;
}

Layout layout_of(const pxr_orthogonalise_desc& d) {
    Layout y{};
    y.s = std::min(d.rows, d.cols);
    y.l = std::max(d.rows, d.cols);
    y.sp = padded(y.s);
    y.lp = padded(y.l);
    y.parts = (uint32_t)std::min<uint64_t>(kNormParts, norm_units(d.rows, d.cols));
    y.gram = cut_of(y.s, y.l, d.n_matrices);
    y.poly = cut_of(y.s, y.s, d.n_matrices);
    // (1300 x 1300, 121 of them, 338 us in tiles of 128 x 128, 293 of 64 x 64; 1500 x 1500, 144, 453 and 471; 2048 x 2048, 256, 728 and 780)
    y.update = (uint64_t)tiles_of(y.s, 2) * tiles_of(y.l, 2) * d.n_matrices >= 128u ? 2 : 1;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t from = at;
        at += (bytes + 255u) & ~(size_t)255u;
        return from;
    };
    const auto partial = [&](const Cut& c) { return (size_t)(triangle_of(y.s, c.M) - c.whole) * d.n_matrices * c.splits * (4096u * c.M * c.M) * sizeof(float); };
    y.sums = take((size_t)d.n_matrices * y.parts * sizeof(double));
    y.partial = take(std::max(partial(y.gram), partial(y.poly)));
    for (size_t& x : y.x) x = take((size_t)2 * d.n_matrices * y.sp * y.lp * sizeof(half));
    y.a = take((size_t)2 * d.n_matrices * y.sp * y.sp * sizeof(half));
    y.b = take((size_t)2 * d.n_matrices * y.sp * y.sp * sizeof(half));
    y.bytes = at;
    return y;
}

// What the steps' sums are multiplied with; the first value is what X_0 is held times.
float factors_of(const pxr_orthogonalise_desc& d, Factors* steps) {
    double most = 1.0;  // of the singular values
    const float first = power_below(kMost);
    float held = first;
    for (uint32_t k = 0; k < d.n_steps; ++k) {
        const double a = d.coefficients[3 * k], b = d.coefficients[3 * k + 1], c = d.coefficients[3 * k + 2];
        const OrthogonaliseBounds next = orthogonalise_bounds(a, b, c, most);
        most = std::max(most, kLeast);
        const float held_a = power_below(kMost / (most * most)), held_b = power_below(kMost / std::max(next.factor, kLeast));
        const float held_x = k + 1u < d.n_steps ? power_below(kMost / std::max(next.most, kLeast)) : 1.0f;
        steps[k] = {held_a / held / held, (float)(c * held_b / held_a / held_a), (float)(b * held_b / held_a), (float)(a * held_b), held_x / held_b / held};
        held = held_x;
        most = next.most;
    }
    return first;
}

template <int kKind>
hipError_t launch_product(const Product& p, int M, uint32_t n_matrices, hipStream_t st) {
    constexpr bool kSym = kKind <= kPoly;
    const uint32_t tiles = kSym ? p.tiles_i * (p.tiles_i + 1u) / 2u : p.tiles_i * p.tiles_j, cut = tiles - p.whole;
    const dim3 grid(on_dies(p.whole) + on_dies(cut * p.splits), 1, n_matrices), threads(kThreads), joined(cut * 4u * M * M, 1, n_matrices);
    const bool few = (uint64_t)(p.whole + cut * p.splits) * n_matrices <= kFewGroups;
    if (M == 2) {  // (a symmetric product takes tiles of this size where there are many)
        if (kSym || !few)
            hipLaunchKernelGGL((product_kernel<kKind, 2, 1>), grid, threads, 0, st, p);
        else if constexpr (!kSym)
            hipLaunchKernelGGL((product_kernel<kKind, 2, kGroups>), grid, dim3(kThreads * kGroups), 0, st, p);
    } else if (few)
        hipLaunchKernelGGL((product_kernel<kKind, 1, kGroups>), grid, dim3(kThreads * kGroups), 0, st, p);
    else
        hipLaunchKernelGGL((product_kernel<kKind, 1, 1>), grid, threads, 0, st, p);
    if constexpr (kSym)
        if (cut) {
            if (M == 2)
                hipLaunchKernelGGL((join_kernel<kKind, 2>), joined, threads, 0, st, p);
            else
                hipLaunchKernelGGL((join_kernel<kKind, 1>), joined, threads, 0, st, p);
        }
    return hipGetLastError();
}

// Small kernels' LDS is more than a kernel has by default: asked for by the first launch on a device.
template <class T>
hipError_t launch_small(const Small& a, uint32_t n_matrices, hipStream_t st) {
    static std::atomic<uint64_t> devices{0};
    int device = 0;
    if (const hipError_t rc = hipGetDevice(&device); rc != hipSuccess) return rc;
    const uint64_t bit = device < 64 ? 1ull << device : 0ull;
    if (!(devices.load(std::memory_order_relaxed) & bit)) {
        if (const hipError_t rc = hipFuncSetAttribute(reinterpret_cast<const void*>(&small_kernel<T>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds); rc != hipSuccess) return rc;
        devices.fetch_or(bit, std::memory_order_relaxed);
    }
    hipLaunchKernelGGL((small_kernel<T>), dim3(n_matrices), dim3(kSmallThreads), small_lds(a.sp, a.lp), st, a);
    return hipGetLastError();
}

// `a`: of all rounds at once, from the update to the result; `held`: X between rounds, [matrices][s][l].
template <class T>
hipError_t launch_narrow(const Narrow& a, const uint32_t* ends, uint32_t rounds, double* held, uint32_t n_matrices, hipStream_t st) {
    const dim3 threads(256), parts(a.parts, n_matrices), places((a.l + 63u) / 64u, n_matrices);
    Narrow n = a;
    for (uint32_t round = 0; round < rounds; ++round) {
        const bool first = round == 0u, last = round + 1u == rounds;
        n.begin = first ? 0u : ends[round - 1u];
        n.end = ends[round];
        if (!first) {
            n.x = held;
            n.x_matrix = (int64_t)a.s * a.l;
            n.x_down = a.l;
            n.x_along = 1;
        }
        n.out = last ? a.out : held;
        n.out_matrix = last ? a.out_matrix : (int64_t)a.s * a.l;
        n.out_down = last ? a.out_down : a.l;
        n.out_along = last ? a.out_along : 1;
        if (first)
            hipLaunchKernelGGL((narrow_sums_kernel<T>), parts, threads, 0, st, n);
        else
            hipLaunchKernelGGL((narrow_sums_kernel<double>), parts, threads, 0, st, n);
        hipLaunchKernelGGL(narrow_steps_kernel, dim3(n_matrices), dim3(kNarrow * kNarrow), 0, st, n);
        if (first && last)
            hipLaunchKernelGGL((narrow_product_kernel<T, T>), places, threads, 0, st, n);
        else if (first)
            hipLaunchKernelGGL((narrow_product_kernel<T, double>), places, threads, 0, st, n);
        else if (last)
            hipLaunchKernelGGL((narrow_product_kernel<double, T>), places, threads, 0, st, n);
        else
            hipLaunchKernelGGL((narrow_product_kernel<double, double>), places, threads, 0, st, n);
        if (const hipError_t rc = hipGetLastError(); rc != hipSuccess) return rc;
    }
    return hipSuccess;
}

int result(hipError_t rc, std::string& err) {
    if (rc == hipSuccess) return PXR_OK;
    err = std::string("kernel launch failed: ") + hipGetErrorString(rc);
    return PXR_ERR_DEVICE;
}

}  // namespace

size_t orthogonalise_workspace(const pxr_orthogonalise_desc& d) {
    const uint32_t shorter = std::min(d.rows, d.cols), longer = std::max(d.rows, d.cols);
    if (is_narrow(shorter, longer)) {
        uint32_t ends[64];
        const size_t held = narrow_rounds(d, ends) > 1u ? (size_t)shorter * longer : 0u;
        return (size_t)d.n_matrices * ((narrow_parts(longer, d.n_matrices) + 1u) * (kNarrow * kNarrow) + held) * sizeof(double);
    }
    return is_small(shorter, longer) ? 0 : layout_of(d).bytes;
}

int launch_orthogonalise(const pxr_orthogonalise_desc& d, const void* x, void* out, void* ws, void* stream, std::string& err) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint32_t shorter = std::min(d.rows, d.cols), longer = std::max(d.rows, d.cols);
    if (is_narrow(shorter, longer)) {
        const bool tall = d.rows > d.cols;
        Narrow a{x, out, d.x_matrix, tall ? 1 : d.x_row, tall ? d.x_row : 1, d.out_matrix, tall ? 1 : d.out_row, tall ? d.out_row : 1, shorter, longer, narrow_parts(longer, d.n_matrices), 0, 0, 0,
                 static_cast<double*>(ws), nullptr, d.eps, {}};
        a.products = a.sums + (size_t)d.n_matrices * a.parts * (kNarrow * kNarrow);
        double* const held = a.products + (size_t)d.n_matrices * (kNarrow * kNarrow);
        a.each = ((longer + a.parts - 1u) / a.parts + 63u) / 64u * 64u;
        a.parts = (longer + a.each - 1u) / a.each;
        std::copy_n(d.coefficients, 3 * d.n_steps, &a.coefficients[0][0]);
        uint32_t ends[64];
        const uint32_t rounds = narrow_rounds(d, ends);
        return result(d.dtype == PXR_F32 ? launch_narrow<float>(a, ends, rounds, held, d.n_matrices, st) : launch_narrow<__bf16>(a, ends, rounds, held, d.n_matrices, st), err);
    }
    if (is_small(shorter, longer)) {
        Small a{x, out, d.x_matrix, d.x_row, d.out_matrix, d.out_row, d.rows, d.cols, shorter, longer, up32(shorter), up32(longer), d.n_steps, d.eps, 0.0f, {}};
        a.held = factors_of(d, a.steps);
        return result(d.dtype == PXR_F32 ? launch_small<float>(a, d.n_matrices, st) : launch_small<__bf16>(a, d.n_matrices, st), err);
    }
    const Layout y = layout_of(d);
    char* const base = static_cast<char*>(ws);
    const auto planes = [&](size_t at, uint32_t cols) {
        const size_t matrix = (size_t)y.sp * cols;
        return Planes{reinterpret_cast<half*>(base + at), matrix * d.n_matrices, matrix, cols};
    };
    const Planes xs[2] = {planes(y.x[0], y.lp), planes(y.x[1], y.lp)}, as = planes(y.a, y.sp), bs = planes(y.b, y.sp);
    Factors steps[64];
    const float held = factors_of(d, steps);
    Prepare prep{x, d.x_matrix, d.x_row, d.rows, d.cols, y.parts, reinterpret_cast<double*>(base + y.sums), xs[0], d.eps, held};
    const dim3 threads(kThreads), sums(y.parts, d.n_matrices), tiles(y.lp / 64u, y.sp / 64u, d.n_matrices);
    if (d.dtype == PXR_F32) {
        hipLaunchKernelGGL((square_sums_kernel<float>), sums, threads, 0, st, prep);
        hipLaunchKernelGGL((split_kernel<float>), tiles, threads, 0, st, prep);
    } else {
        hipLaunchKernelGGL((square_sums_kernel<__bf16>), sums, threads, 0, st, prep);
        hipLaunchKernelGGL((split_kernel<__bf16>), tiles, threads, 0, st, prep);
    }
    hipError_t rc = hipGetLastError();
    const auto cut_as = [](Product& p, const Cut& c, uint32_t s) {
        p.tiles_i = p.tiles_j = tiles_of(s, c.M);
        p.whole = c.whole;
        p.splits = c.splits;
        p.steps_each = c.steps_each;
    };
    for (uint32_t k = 0; k < d.n_steps && rc == hipSuccess; ++k) {
        const Factors& f = steps[k];
        const Planes from = xs[k & 1u], to = xs[(k + 1u) & 1u];
        Product p{};
        // A
        p.a = p.b = from;
        p.to = as;
        p.depth = up64(y.l);
        cut_as(p, y.gram, y.s);
        p.partial = reinterpret_cast<float*>(base + y.partial);
        p.scale = f.gram;
        p.s = y.s;
        rc = launch_product<kGram>(p, y.gram.M, d.n_matrices, st);
        if (rc != hipSuccess) break;
        // B
        p.a = p.b = as;
        p.to = bs;
        p.depth = up64(y.s);
        cut_as(p, y.poly, y.s);
        p.scale = f.poly;
        p.c0 = f.diagonal;
        p.c1 = f.linear;
        rc = launch_product<kPoly>(p, y.poly.M, d.n_matrices, st);
        if (rc != hipSuccess) break;
        // X
        p.a = bs;
        p.b = from;
        p.to = to;
        p.tiles_i = tiles_of(y.s, y.update);
        p.tiles_j = tiles_of(y.l, y.update);
        p.whole = p.tiles_i * p.tiles_j;
        p.splits = 1u;
        p.scale = f.update;
        p.out = out;
        p.out_matrix = d.out_matrix;
        p.out_row = d.out_row;
        p.rows = d.rows;
        p.cols = d.cols;
        p.transposed = d.rows > d.cols;
        p.bf16 = d.dtype == PXR_BF16;
        rc = k + 1u == d.n_steps ? launch_product<kLast>(p, y.update, d.n_matrices, st)
                                 : launch_product<kUpdate>(p, y.update, d.n_matrices, st);
    }
    return result(rc, err);
}

}  // namespace pxr
