// Layer norm over rows, forward and backward (pxr_layer_norm_* in include/pxr.h).  gfx950 only.
//
//   mean = sum x / D,  rstd = 1 / sqrt(sum (x - mean)^2 / D + eps),  y = (x - mean) rstd w + b
//   dx = rstd (g - sum g / D - xh sum(g xh) / D),  g = w dy,  xh = (x - mean) rstd;  dw = sum_rows dy xh,  db = sum_rows dy
//
// Both directions are bound by HBM: a few operations for every byte.  So a row of ordinary width is read once and stays in registers, as it came,
// until it leaves: the deviations are squared after the mean is taken off (a row far from zero keeps its variance), from the
// registers.  All sums are fp32.
//
// A lane holds VPL vectors of 16 bytes of a row, lanes of a row next to each other.  Who takes a row goes by the number of its
// vectors:
//   up to 64      a part of a wavefront, 1 to 64 lanes: eight rows of 64 bfloat16 values in a wavefront
//   up to 256     a wavefront, two or four vectors a lane (backward: up to 128, two)
//   up to 16384   a workgroup of 256 to 1024 threads, two to sixteen vectors a lane: what a lane has in flight counts for more than lanes do
//                 (backward: up to 32768 values, one to eight vectors)
//                 (forward, 30000 x 7000 bfloat16: 256 threads 175 us, 512 of them 188; 9000 x 5000 fp32: 512 threads 59, 1024 of them 80; 4096 x 30752 bfloat16:
//                 two rows at a time 85, four 98)
//   more          a workgroup that reads the row again for each sum (from the caches, mostly): 800 x 50000 fp32 124 us, 70 from registers
// The backward pass of rows of more than 32768 values forms the sums over rows in a kernel of its own, which reads dy and x once; the one that forms dx reads them
// once more (bfloat16, up to 65536 values) or twice (800 x 50000 fp32 186 us, 94 at the rate of a copy).
// What leaves is not read again by the kernel and goes past the caches that it would push x out of (524288 x 64 bfloat16 31 -> 25 us, 4096 x 30752 146 -> 110;
// requests that go past them as well are slower where x lies in them).
//
// Workgroups are persistent and walk the rows, so that weights and biases are read once by a wavefront, or once for four rows by a workgroup:
// in 32 bits they are twice the bytes of a bfloat16 row, each.  The sums over rows of the backward pass stay in registers as well, and
// leave once for each workgroup; a second kernel adds the workgroups' sums in their order, so that equal inputs give equal bits.

#include <hip/hip_runtime.h>

#include <atomic>

#include "pxr_internal.h"

namespace pxr {
namespace {

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __bf16* p) { return (float)*p; }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__bf16* p, float v) { *p = (__bf16)v; }  // round to nearest even

typedef uint32_t any_u32x4 __attribute__((ext_vector_type(4), aligned(2)));  // at the address of any value

// 16 bytes of a row: 4 or 8 values, as they came.  Rows may begin at any element: the memory takes 16-byte requests at any address.
template <class T>
struct Vec {
    static constexpr int N = 16 / sizeof(T);
    uint32_t w[4];

    __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(w, p, 16); }
    // The first `count` of them alone (rows narrower than a vector).
    __device__ __forceinline__ void load_some(const T* p, int count) {
        T v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = e < count ? p[e] : (T)0.0f;
        __builtin_memcpy(w, v, 16);
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        return __uint_as_float((e & 1) ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    }
    // Zero in place of the values that are not in [from, to).
    __device__ __forceinline__ void keep(int from, int to) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < from || e >= to) {
                if constexpr (sizeof(T) == 4)
                    w[e] = 0u;
                else
                    w[e >> 1] &= (e & 1) ? 0x0000FFFFu : 0xFFFF0000u;
            }
    }
    // What follows takes the values from these registers again instead of keeping them all as floats in others.
    __device__ __forceinline__ void as_they_came() {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(w[i]));
    }
    static __device__ __forceinline__ void store(T* p, const float (&f)[N], int from, int to) {
        T v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)f[e];  // round to nearest even
        if (from == 0 && to >= N) {
            any_u32x4 w;
            __builtin_memcpy(&w, v, 16);
            __builtin_nontemporal_store(w, reinterpret_cast<any_u32x4*>(p));
            return;
        }
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e >= from && e < to) p[e] = v[e];
    }
};

// Where a lane's vector lies in the row and which of its values [from, to) are the lane's own.  A row that ends inside a vector has its last
// vector moved back to its end, so that it is one request like the others (the values it shares with the vector before it
// are that one's); lanes past the end have the last vector as well, and none of it is theirs.  kTiny: rows narrower than a vector.
template <int N, bool kTiny>
struct Place {
    uint32_t at;
    int from, to;
    __device__ __forceinline__ Place(uint32_t vector, uint32_t D) {
        const uint32_t want = vector * N;
        if (kTiny) {
            at = 0;
            from = 0;
            to = vector == 0 ? (int)D : 0;
        } else {
            at = min(want, D - N);
            from = (int)min(want - at, (uint32_t)N);
            to = N;
        }
    }
    __device__ __forceinline__ bool whole() const { return kTiny ? to == N : from == 0; }
    __device__ __forceinline__ bool any() const { return from < to; }
    __device__ __forceinline__ bool own(int e) const { return kTiny ? e < to : e >= from; }
};

// A lane's number where 1024 threads hold a row: the places of its vectors are worked out again where they are used, since the
// registers are full without them.
template <int NT>
__device__ __forceinline__ uint32_t again(uint32_t l) {
    if (NT == 1024) asm volatile("" : "+v"(l));
    return l;
}

// A sum is formed up to here: the compiler would otherwise put off what it is made of, and keep all of it, until the sum is read.
__device__ __forceinline__ void formed(float& v) { asm volatile("" : "+v"(v)); }

// The parameters of a vector, `def` where there is no array.
template <class P, int N, bool kTiny>
__device__ __forceinline__ void load_params(const P* p, float def, const Place<N, kTiny>& at, float (&f)[N]) {
    if (!p) {
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = def;
    } else if (kTiny) {
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = at.own(e) ? load1(p + e) : def;
    } else {
        P v[N];
        __builtin_memcpy(v, p + at.at, sizeof(v));
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = (float)v[e];
    }
}

// Sums of U values over a row's lanes, the same bits in each of them.  NT == 0: `lanes` (a power of two) next to each other in a
// wavefront; otherwise the NT threads of the workgroup, through `lds` [U][NT / 64], with one barrier (the caller does not write these words
// again before another barrier).
template <int NT, int U>
__device__ __forceinline__ void row_sums(float (&v)[U], uint32_t lanes, float* lds) {
    if constexpr (NT == 0) {
        for (uint32_t m = lanes >> 1; m >= 1; m >>= 1)
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] += __shfl_xor(v[u], m);
    } else {
        constexpr uint32_t W = NT / 64;
#pragma unroll
        for (uint32_t m = 32; m >= 1; m >>= 1)
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] += __shfl_xor(v[u], m);
        if ((threadIdx.x & 63u) == 0)
#pragma unroll
            for (int u = 0; u < U; ++u) lds[u * W + (threadIdx.x >> 6)] = v[u];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = lds[u * W + (threadIdx.x & (W - 1u))];
#pragma unroll
        for (uint32_t m = W >> 1; m >= 1; m >>= 1)
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] += __shfl_xor(v[u], m);
    }
}

constexpr uint32_t kSubThreads = 512;  // of a workgroup whose rows take a wavefront or less each
constexpr uint32_t kThreadsOf(int nt) { return nt ? (uint32_t)nt : kSubThreads; }

struct NormForward {
    const void *x, *weight, *bias;
    void* y;
    float *mean, *rstd;
    int64_t x_stride, y_stride;
    uint32_t n, D, lanes;
    float eps;
};

// U rows at a time: their requests are in flight together, and they share one read of weight and bias.  Where rows are shorter than a line of
// memory, a wavefront's groups of lanes have rows next to each other, so that a request is of whole lines (2 000 000 x 8 in fp32 54 -> 24 us); longer
// ones lie together for each group (524288 x 64 bfloat16 24.8 us, otherwise 26.6).
template <class T, class P, int NT, int VPL, int U, bool kTiny = false>
__global__ __launch_bounds__(kThreadsOf(NT)) void norm_forward_kernel(const NormForward a) {
    constexpr int N = Vec<T>::N;
    constexpr bool kKeep = NT == 0;  // parameters stay in registers
    typedef Place<N, kTiny> At;
    __shared__ float lds[2 * U * 16];
    const uint32_t lanes = NT ? NT : a.lanes, l = NT ? threadIdx.x : threadIdx.x & (lanes - 1u);
    const uint32_t group = NT ? 0u : threadIdx.x / lanes, groups = NT ? 1u : kThreadsOf(NT) / lanes;
    const uint32_t apart = NT || lanes >= 8u ? 1u : 64u / lanes, in_wave = group & (apart - 1u);  // rows from one of the U to the next
    const P *weight = static_cast<const P*>(a.weight), *bias = static_cast<const P*>(a.bias);
    float w[kKeep ? VPL : 1][N], b[kKeep ? VPL : 1][N];
    if (kKeep)
#pragma unroll
        for (int p = 0; p < VPL; ++p) {
            load_params(weight, 1.0f, At(l + p * lanes, a.D), w[kKeep ? p : 0]);
            load_params(bias, 0.0f, At(l + p * lanes, a.D), b[kKeep ? p : 0]);
        }
    const float width = (float)a.D;  // (divided by: a product with 1 / D would move the mean of equal values)
    for (uint64_t row0 = ((uint64_t)blockIdx.x * groups + (group - in_wave)) * U + in_wave; row0 < a.n; row0 += (uint64_t)gridDim.x * groups * U) {
        Vec<T> x[U][VPL];
        const T* first = static_cast<const T*>(a.x) + (int64_t)row0 * a.x_stride;
        T* to = static_cast<T*>(a.y) + (int64_t)row0 * a.y_stride;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const T* xr = first + (row0 + u * apart < a.n ? (int64_t)(u * apart) * a.x_stride : 0);
#pragma unroll
            for (int p = 0; p < VPL; ++p) {
                const At at(again<NT>(l) + p * lanes, a.D);
                if (kTiny)
                    x[u][p].load_some(xr, at.to);
                else
                    x[u][p].load(xr + at.at);
            }
        }
        float mean[U], rstd[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            mean[u] = 0.0f;
#pragma unroll
            for (int p = 0; p < VPL; ++p) {
                const At at(again<NT>(l) + p * lanes, a.D);
                float s = 0.0f;
#pragma unroll
                for (int e = 0; e < N; ++e) s += x[u][p].get(e);
                if (!at.whole()) {
                    s = 0.0f;
#pragma unroll
                    for (int e = 0; e < N; ++e) s += at.own(e) ? x[u][p].get(e) : 0.0f;
                }
                mean[u] += s;
                formed(mean[u]);
                x[u][p].as_they_came();
            }
        }
        row_sums<NT, U>(mean, lanes, lds);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            mean[u] /= width;
            rstd[u] = 0.0f;
#pragma unroll
            for (int p = 0; p < VPL; ++p) {
                const At at(again<NT>(l) + p * lanes, a.D);
                float s = 0.0f;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float c = x[u][p].get(e) - mean[u];
                    s = __builtin_fmaf(c, c, s);
                }
                if (!at.whole()) {
                    s = 0.0f;
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float c = at.own(e) ? x[u][p].get(e) - mean[u] : 0.0f;
                        s = __builtin_fmaf(c, c, s);
                    }
                }
                rstd[u] += s;
                formed(rstd[u]);
                x[u][p].as_they_came();
            }
        }
        row_sums<NT, U>(rstd, lanes, lds + U * 16);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            rstd[u] = 1.0f / sqrtf(rstd[u] / width + a.eps);
            if (l == 0 && row0 + u * apart < a.n) {
                if (a.mean) a.mean[row0 + u * apart] = mean[u];
                if (a.rstd) a.rstd[row0 + u * apart] = rstd[u];
            }
        }
#pragma unroll
        for (int p = 0; p < VPL; ++p) {
            const At at(again<NT>(l) + p * lanes, a.D);
            if (!kKeep) {
                load_params(weight, 1.0f, at, w[0]);
                load_params(bias, 0.0f, at, b[0]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (row0 + u * apart >= a.n || !at.any()) continue;
                float y[N];
#pragma unroll
                for (int e = 0; e < N; ++e) y[e] = __builtin_fmaf((x[u][p].get(e) - mean[u]) * rstd[u], w[kKeep ? p : 0][e], b[kKeep ? p : 0][e]);
                Vec<T>::store(to + ((int64_t)(u * apart) * a.y_stride + at.at), y, at.from, at.to);
            }
        }
    }
}

// Rows of any width, read again for each sum.
template <class T, class P>
__global__ __launch_bounds__(1024) void norm_forward_wide_kernel(const NormForward a) {
    constexpr int N = Vec<T>::N;
    typedef Place<N, false> At;
    __shared__ float lds[32];
    const T* xr = static_cast<const T*>(a.x) + (int64_t)blockIdx.x * a.x_stride;
    T* yr = static_cast<T*>(a.y) + (int64_t)blockIdx.x * a.y_stride;
    const uint32_t vectors = (a.D + N - 1u) / N;
    const float width = (float)a.D;
    float mean[1] = {0.0f}, rstd[1] = {0.0f};
    for (uint32_t i = threadIdx.x; i < vectors; i += 1024u) {
        const At at(i, a.D);
        Vec<T> x;
        x.load(xr + at.at);
#pragma unroll
        for (int e = 0; e < N; ++e) mean[0] += at.own(e) ? x.get(e) : 0.0f;
    }
    row_sums<1024, 1>(mean, 0, lds);
    mean[0] /= width;
    for (uint32_t i = threadIdx.x; i < vectors; i += 1024u) {
        const At at(i, a.D);
        Vec<T> x;
        x.load(xr + at.at);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float c = at.own(e) ? x.get(e) - mean[0] : 0.0f;
            rstd[0] = __builtin_fmaf(c, c, rstd[0]);
        }
    }
    row_sums<1024, 1>(rstd, 0, lds + 16);
    rstd[0] = 1.0f / sqrtf(rstd[0] / width + a.eps);
    for (uint32_t i = threadIdx.x; i < vectors; i += 1024u) {
        const At at(i, a.D);
        Vec<T> x;
        x.load(xr + at.at);
        float w[N], b[N], y[N];
        load_params(static_cast<const P*>(a.weight), 1.0f, at, w);
        load_params(static_cast<const P*>(a.bias), 0.0f, at, b);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = __builtin_fmaf((x.get(e) - mean[0]) * rstd[0], w[e], b[e]);
        Vec<T>::store(yr + at.at, y, at.from, at.to);
    }
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[blockIdx.x] = mean[0];
        if (a.rstd) a.rstd[blockIdx.x] = rstd[0];
    }
}

struct NormBackward {
    const void *dy, *x;
    const float *mean, *rstd;
    const void* weight;
    void* dx;
    float* sums;    // [workgroups][2][D]: dw, db of a workgroup's rows; null = not wanted
    void *dw, *db;  // where one workgroup has all rows: the results themselves; null = not wanted
    int64_t dy_stride, x_stride, dx_stride;
    uint32_t n, D, lanes;
};

// kSums: the sums over rows are formed here as well.  Workgroups of 1024 threads hold those of db in LDS, each lane its own words: beside dw and a
// row they do not fit the registers.  Where the weights stay in registers a workgroup asks for its next rows before it works on the present ones
// (a request for weights behind them would have to wait for them: the memory answers in order).
template <class T, class P, int NT, int VPL, int U, bool kSums, bool kTiny = false>
__global__ __launch_bounds__(kThreadsOf(NT)) void norm_backward_kernel(const NormBackward a) {
    constexpr int N = Vec<T>::N;
    constexpr bool kKeep = VPL * N <= 16, kAhead = NT != 0 && VPL <= 2, kLds = kSums && NT == 1024;
    static_assert(kKeep || !kAhead);
    typedef Place<N, kTiny> At;
    extern __shared__ __align__(16) float lds[];  // 2 x 2 U x 16 floats and db, or (NT == 0) the sums of a wavefront's lanes
    float* const db_lds = lds + 2 * (2 * U * 16);  // [VPL N][1024]
    const uint32_t lanes = NT ? NT : a.lanes, l = NT ? threadIdx.x : threadIdx.x & (lanes - 1u);
    const uint32_t group = NT ? 0u : threadIdx.x / lanes, groups = NT ? 1u : kThreadsOf(NT) / lanes;
    const uint32_t apart = NT || lanes >= 8u ? 1u : 64u / lanes, in_wave = group & (apart - 1u);  // rows from one of the U to the next
    const P* weight = static_cast<const P*>(a.weight);
    float w[kKeep ? VPL : 1][N];
    if (kKeep)
#pragma unroll
        for (int p = 0; p < VPL; ++p) load_params(weight, 1.0f, At(l + p * lanes, a.D), w[kKeep ? p : 0]);
    float dw[kSums ? VPL : 1][N] = {}, db[kSums && !kLds ? VPL : 1][N] = {};
    if (kLds)
#pragma unroll
        for (int i = 0; i < VPL * N; ++i) db_lds[i * 1024 + l] = 0.0f;
    const float per = 1.0f / (float)a.D;
    struct Rows {
        Vec<T> g[U][VPL], x[U][VPL];
        float mean[U], rstd[U];
    };
    const auto ask = [&](Rows& r, uint64_t row0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint64_t row = min(row0 + u * apart, (uint64_t)a.n - 1u);
            const T *gr = static_cast<const T*>(a.dy) + (int64_t)row * a.dy_stride, *xr = static_cast<const T*>(a.x) + (int64_t)row * a.x_stride;
#pragma unroll
            for (int p = 0; p < VPL; ++p) {
                const At at(again<NT>(l) + p * lanes, a.D);
                if (kTiny) {
                    r.g[u][p].load_some(gr, at.to);
                    r.x[u][p].load_some(xr, at.to);
                } else {
                    r.g[u][p].load(gr + at.at);
                    r.x[u][p].load(xr + at.at);
                }
            }
            r.mean[u] = a.mean[row];
            r.rstd[u] = a.rstd[row];
        }
    };
    uint32_t turn = 0;
    uint64_t row0 = ((uint64_t)blockIdx.x * groups + (group - in_wave)) * U + in_wave;
    const uint64_t stride = (uint64_t)gridDim.x * groups * U;
    Rows r, ahead;
    if (kAhead && row0 < a.n) ask(ahead, row0);
    for (; row0 < a.n; row0 += stride) {
        if (kAhead) {
            r = ahead;
            if (row0 + stride < a.n) ask(ahead, row0 + stride);
        } else {
            ask(r, row0);
        }
        float s[2 * U];
#pragma unroll
        for (int u = 0; u < U; ++u) s[2 * u] = s[2 * u + 1] = 0.0f;
#pragma unroll
        for (int p = 0; p < VPL; ++p) {
            const At at(again<NT>(l) + p * lanes, a.D);
            // (one vector's weights and floats after the other: all of them at once do not fit the registers of 1024 threads)
            if (NT == 1024) __builtin_amdgcn_sched_barrier(0);
            if (!kKeep) load_params(weight, 1.0f, at, w[0]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                // What is not the lane's own is nothing: its gradient is zero here, and so is what it adds to a sum.  (x beside it is of the same
                // row: where it is no number, the row's gradient is none either.  A row past the last must not reach the sums over rows.)
                if (!at.whole()) r.g[u][p].keep(at.from, at.to);
                if (row0 + u * apart >= a.n) {
                    r.g[u][p].keep(0, 0);
                    r.x[u][p].keep(0, 0);
                    r.mean[u] = r.rstd[u] = 0.0f;
                }
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float d = r.g[u][p].get(e), xh = (r.x[u][p].get(e) - r.mean[u]) * r.rstd[u];
                    const float wd = d * w[kKeep ? p : 0][e];
                    s[2 * u] += wd;
                    s[2 * u + 1] = __builtin_fmaf(wd, xh, s[2 * u + 1]);
                    if (kSums) dw[kSums ? p : 0][e] = __builtin_fmaf(d, xh, dw[kSums ? p : 0][e]);
                    if (kLds) formed(dw[kSums ? p : 0][e]);
                    if (kLds)
                        db_lds[(p * N + e) * 1024 + again<NT>(l)] += d;
                    else if (kSums)
                        db[kSums && !kLds ? p : 0][e] += d;
                }
                formed(s[2 * u]);
                formed(s[2 * u + 1]);
                r.g[u][p].as_they_came();
                r.x[u][p].as_they_came();
            }
        }
        row_sums<NT, 2 * U>(s, lanes, lds + (turn & 1u) * (2 * U * 16));
        ++turn;
#pragma unroll
        for (int p = 0; p < VPL; ++p) {
            const At at(again<NT>(l) + p * lanes, a.D);
            if (NT == 1024) __builtin_amdgcn_sched_barrier(0);
            if (!kKeep) load_params(weight, 1.0f, at, w[0]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (row0 + u * apart >= a.n || !at.any()) continue;
                float dx[N];
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float xh = (r.x[u][p].get(e) - r.mean[u]) * r.rstd[u];
                    dx[e] = r.rstd[u] * __builtin_fmaf(-xh, s[2 * u + 1] * per, __builtin_fmaf(r.g[u][p].get(e), w[kKeep ? p : 0][e], -s[2 * u] * per));
                }
                Vec<T>::store(static_cast<T*>(a.dx) + ((int64_t)(row0 + u * apart) * a.dx_stride + at.at), dx, at.from, at.to);
            }
        }
    }
    if (!kSums || !(a.sums || a.dw || a.db)) return;
    const auto put = [&](uint32_t i, float w_sum, float b_sum) {
        if (a.sums) {
            float* out = a.sums + (size_t)blockIdx.x * 2u * a.D;
            out[i] = w_sum;
            out[a.D + i] = b_sum;
        } else {
            if (a.dw) store1(static_cast<P*>(a.dw) + i, w_sum);
            if (a.db) store1(static_cast<P*>(a.db) + i, b_sum);
        }
    };
    if constexpr (NT == 0) {
        // the rows' groups of a wavefront, then the wavefronts one after the other
        for (uint32_t m = lanes; m < 64u; m <<= 1)
#pragma unroll
            for (int p = 0; p < VPL; ++p)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    dw[kSums ? p : 0][e] += __shfl_xor(dw[kSums ? p : 0][e], m);
                    db[kSums && !kLds ? p : 0][e] += __shfl_xor(db[kSums && !kLds ? p : 0][e], m);
                }
        const uint32_t span = lanes * VPL * N;
        for (uint32_t wave = 0; wave < kSubThreads / 64u; ++wave) {
            __syncthreads();
            if (threadIdx.x >> 6 == wave && (threadIdx.x & 63u) < lanes)
#pragma unroll
                for (int p = 0; p < VPL; ++p)
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        float* q = lds + (p * N + e) * lanes + l;
                        q[0] = (wave ? q[0] : 0.0f) + dw[kSums ? p : 0][e];
                        q[span] = (wave ? q[span] : 0.0f) + db[kSums && !kLds ? p : 0][e];
                    }
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < a.D; i += kSubThreads) {
            const uint32_t v = i / N, e = i - At(v, a.D).at, at = (v / lanes * N + e) * lanes + (v & (lanes - 1u));
            put(i, lds[at], lds[span + at]);
        }
    } else {
#pragma unroll
        for (int p = 0; p < VPL; ++p) {
            const At at(again<NT>(l) + p * lanes, a.D);
            if (!at.any()) continue;
            float b[N];
#pragma unroll
            for (int e = 0; e < N; ++e) b[e] = kLds ? db_lds[(p * N + e) * 1024 + l] : db[kSums && !kLds ? p : 0][e];
            if (at.whole()) {  // (whole vectors: value by value 4096 x 30752 bfloat16 took 229 us, 204 so)
                if (a.sums) {
                    float* out = a.sums + (size_t)blockIdx.x * 2u * a.D + at.at;
                    __builtin_memcpy(out, dw[kSums ? p : 0], sizeof(b));
                    __builtin_memcpy(out + a.D, b, sizeof(b));
                } else {
                    P wp[N], bp[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        store1(wp + e, dw[kSums ? p : 0][e]);
                        store1(bp + e, b[e]);
                    }
                    if (a.dw) __builtin_memcpy(static_cast<P*>(a.dw) + at.at, wp, sizeof(wp));
                    if (a.db) __builtin_memcpy(static_cast<P*>(a.db) + at.at, bp, sizeof(bp));
                }
                continue;
            }
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (at.own(e)) put(at.at + e, dw[kSums ? p : 0][e], b[e]);
        }
    }
}

// dx alone, rows of any width.
template <class T, class P>
__global__ __launch_bounds__(1024) void norm_dx_wide_kernel(const NormBackward a) {
    constexpr int N = Vec<T>::N;
    typedef Place<N, false> At;
    __shared__ float lds[32];
    const T* dyr = static_cast<const T*>(a.dy) + (int64_t)blockIdx.x * a.dy_stride;
    const T* xr = static_cast<const T*>(a.x) + (int64_t)blockIdx.x * a.x_stride;
    T* dxr = static_cast<T*>(a.dx) + (int64_t)blockIdx.x * a.dx_stride;
    const P* weight = static_cast<const P*>(a.weight);
    const uint32_t vectors = (a.D + N - 1u) / N;
    const float m = a.mean[blockIdx.x], r = a.rstd[blockIdx.x];
    float s[2] = {0.0f, 0.0f};
    for (uint32_t i = threadIdx.x; i < vectors; i += 1024u) {
        const At at(i, a.D);
        Vec<T> dy, x;
        dy.load(dyr + at.at);
        x.load(xr + at.at);
        float w[N];
        load_params(weight, 1.0f, at, w);
        if (!at.whole()) dy.keep(at.from, at.to);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float g = dy.get(e) * w[e];
            s[0] += g;
            s[1] = __builtin_fmaf(g, (x.get(e) - m) * r, s[1]);
        }
    }
    row_sums<1024, 2>(s, 0, lds);
    const float per = 1.0f / (float)a.D;
    for (uint32_t i = threadIdx.x; i < vectors; i += 1024u) {
        const At at(i, a.D);
        Vec<T> dy, x;
        dy.load(dyr + at.at);
        x.load(xr + at.at);
        float w[N], dx[N];
        load_params(weight, 1.0f, at, w);
#pragma unroll
        for (int e = 0; e < N; ++e) dx[e] = r * __builtin_fmaf(-(x.get(e) - m) * r, s[1] * per, __builtin_fmaf(dy.get(e), w[e], -s[0] * per));
        Vec<T>::store(dxr + at.at, dx, at.from, at.to);
    }
}

// The sums over rows alone, for rows whose sums a workgroup cannot hold: a wavefront takes 64 vectors of columns and every fourth row of its
// workgroup's.
template <class T>
__global__ __launch_bounds__(256) void norm_sums_kernel(const NormBackward a, uint32_t rows) {
    constexpr int N = Vec<T>::N;
    __shared__ float lds[2 * N * 64];
    const uint32_t l = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const Place<N, false> at(blockIdx.x * 64u + l, a.D);
    const size_t col = at.at;
    float dw[N] = {}, db[N] = {};
    const uint64_t first = (uint64_t)blockIdx.y * rows, last = min(first + rows, (uint64_t)a.n);
    if (at.any())
#pragma unroll 2
        for (uint64_t row = first + wave; row < last; row += 4) {
            Vec<T> g, x;
            g.load(static_cast<const T*>(a.dy) + (int64_t)row * a.dy_stride + col);
            x.load(static_cast<const T*>(a.x) + (int64_t)row * a.x_stride + col);
            const float m = a.mean[row], r = a.rstd[row];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                dw[e] = __builtin_fmaf(g.get(e), (x.get(e) - m) * r, dw[e]);
                db[e] += g.get(e);
            }
        }
    for (uint32_t k = 0; k < 4; ++k) {
        if (wave == k)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                dw[e] += k ? lds[e * 64 + l] : 0.0f;
                db[e] += k ? lds[(N + e) * 64 + l] : 0.0f;
                lds[e * 64 + l] = dw[e];
                lds[(N + e) * 64 + l] = db[e];
            }
        __syncthreads();
    }
    float* out = a.sums + (size_t)blockIdx.y * 2u * a.D;
    if (wave != 3) return;
    if (at.whole()) {
        __builtin_memcpy(out + col, dw, sizeof(dw));
        __builtin_memcpy(out + a.D + col, db, sizeof(db));
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (at.own(e)) {
            out[col + e] = dw[e];
            out[a.D + col + e] = db[e];
        }
}

// The workgroups' sums in their order: 64 columns a workgroup, their sums dealt to 16 wavefronts.  A launch counts its threads in 32 bits, and what is
// more is dropped without an error: rows of more than 2^27 - 32 values take several layers of kFinishAcross workgroups.
constexpr uint32_t kFinishAcross = (1u << 22) - 1u;
template <class P>
__global__ __launch_bounds__(1024) void norm_finish_kernel(const float* sums, uint32_t parts, uint32_t D, P* dw, P* db) {
    __shared__ float lds[16][64];
    const uint32_t l = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const size_t i = ((size_t)blockIdx.y * kFinishAcross + blockIdx.x) * 64u + l;
    float s = 0.0f;
    if (i < 2u * (size_t)D)
#pragma unroll 8
        for (uint32_t k = wave; k < parts; k += 16u) s += sums[(size_t)k * 2u * D + i];
    lds[wave][l] = s;
    __syncthreads();
    if (wave) return;
    for (uint32_t k = 1; k < 16u; ++k) s += lds[k][l];
    if (i < D) {
        if (dw) store1(dw + i, s);
    } else if (i < 2u * (size_t)D) {
        if (db) store1(db + (i - D), s);
    }
}

// How a description is laid out on the device.
struct Plan {
    uint32_t vectors, lanes, groups;  // of a row; lanes of a row (0 = a workgroup); rows that a workgroup takes in one go
    bool sums_inside;                 // the backward kernel forms the sums over rows
    uint32_t parts, rows;             // workgroups' sums, and rows for each where a kernel of their own forms them
};

constexpr uint32_t kCus = 256;  // compute units of the device this library is for

Plan plan_of(const pxr_layer_norm_desc& d, uint32_t widest) {
    const uint32_t N = d.dtype == PXR_F32 ? 4u : 8u;
    Plan p{};
    p.vectors = (d.width + N - 1u) / N;
    p.lanes = 0;
    p.groups = 1;
    if (p.vectors <= widest) {  // (the widest row that a wavefront takes)
        p.lanes = 64;
        while (p.lanes > 1u && p.lanes / 2u >= p.vectors) p.lanes /= 2u;
        p.groups = kSubThreads / p.lanes;
    }
    p.sums_inside = p.vectors * N <= 32768u;  // 32 values a lane of 1024: what its registers hold of dw and LDS of db
    if (p.sums_inside) {
        // two workgroups of up to 512 threads, or one of 1024, for each compute unit
        const uint64_t need = (d.n_rows + p.groups - 1u) / p.groups, most = p.vectors <= 1024u ? 2u * kCus : kCus;
        // Few rows are one workgroup's, whose sums are the results: no second kernel and no workspace (a call from Python, fp32: 16 x 256 12.2 us, otherwise 16.5;
        // 2 x 5000 12.7 / 17.0; but 4 x 30000 43 / 26).
        const bool few = need == 1u || (need <= 4u && need * p.vectors <= 4096u);
        p.parts = few && need ? 1u : (uint32_t)(need < most ? need : most);
    } else {
        const uint32_t across = (p.vectors + 63u) / 64u;
        uint64_t parts = (4u * kCus + across - 1u) / across;
        if (parts > (d.n_rows + 15u) / 16u) parts = (d.n_rows + 15u) / 16u;
        if (parts == 0) parts = 1;
        p.rows = (uint32_t)((d.n_rows + parts - 1u) / parts);
        p.parts = p.rows ? (uint32_t)((d.n_rows + p.rows - 1u) / p.rows) : 0u;
    }
    return p;
}
constexpr uint32_t kWidestForward = 256u, kWidestBackward = 128u;

template <class T, class P>
void forward_as(const pxr_layer_norm_desc& d, NormForward a, hipStream_t st) {
    const Plan p = plan_of(d, kWidestForward);
    const auto grid = [&](uint32_t rows_each, uint32_t most) {
        const uint64_t need = (d.n_rows + rows_each - 1u) / rows_each;
        return dim3((uint32_t)(need < most ? need : most));
    };
    a.lanes = p.lanes;
#define PXR_NORM(NT, VPL, U, GROUPS, MOST) \
    hipLaunchKernelGGL((norm_forward_kernel<T, P, NT, VPL, U>), grid(GROUPS * U, MOST), dim3(kThreadsOf(NT)), 0, st, a)
    // Rows that do not fill the device go one by one; many go two or four at a time (fp32: 300 x 1500 4.8 us, several at a time 6.2; 3000 x 12345 49.8, one at a
    // time 52.1).
    const bool many = d.n_rows >= 4u * kCus;
    if (d.width < (uint32_t)Vec<T>::N)
        hipLaunchKernelGGL((norm_forward_kernel<T, P, 0, 1, 4, true>), grid(4u * p.groups, 4u * kCus), dim3(kSubThreads), 0, st, a);
    else if (p.vectors <= 64u)
        PXR_NORM(0, 1, 4, p.groups, 4u * kCus);
    else if (p.vectors <= 128u)
        PXR_NORM(0, 2, 2, p.groups, 4u * kCus);
    else if (p.vectors <= 256u)
        PXR_NORM(0, 4, 1, p.groups, 4u * kCus);
    else if (p.vectors <= 512u) {
        if (many)
            PXR_NORM(256, 2, 4, 1u, 4u * kCus);
        else
            PXR_NORM(256, 2, 1, 1u, 4u * kCus);
    } else if (p.vectors <= 1024u) {
        if (many)
            PXR_NORM(256, 4, 2, 1u, 4u * kCus);
        else
            PXR_NORM(256, 4, 1, 1u, 4u * kCus);
    } else if (p.vectors <= 2048u) {
        if (many)
            PXR_NORM(512, 4, 2, 1u, 2u * kCus);
        else
            PXR_NORM(512, 4, 1, 1u, 4u * kCus);
    } else if (p.vectors <= 4096u) {
        if (many)
            PXR_NORM(1024, 4, 2, 1u, 2u * kCus);
        else
            PXR_NORM(1024, 4, 1, 1u, 2u * kCus);
    } else if (p.vectors <= 8192u)
        PXR_NORM(1024, 8, 1, 1u, 2u * kCus);
    else if (p.vectors <= 16384u)
        PXR_NORM(1024, 16, 1, 1u, kCus);
    else
        hipLaunchKernelGGL((norm_forward_wide_kernel<T, P>), dim3((uint32_t)d.n_rows), dim3(1024), 0, st, a);
#undef PXR_NORM
}

// Launches of more LDS than the 64 KB that a kernel has by default: asked for by a kernel's first such launch on a device.
template <auto kKernel>
hipError_t allow_lds(uint32_t bytes) {
    static std::atomic<uint64_t> devices{0};
    int device = 0;
    if (bytes <= 64u * 1024u) return hipSuccess;
    if (const hipError_t rc = hipGetDevice(&device); rc != hipSuccess) return rc;
    const uint64_t bit = device < 64 ? 1ull << device : 0ull;
    if (devices.load(std::memory_order_relaxed) & bit) return hipSuccess;
    const hipError_t rc = hipFuncSetAttribute(reinterpret_cast<const void*>(kKernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (rc == hipSuccess) devices.fetch_or(bit, std::memory_order_relaxed);
    return rc;
}

template <class T, class P>
hipError_t backward_as(const pxr_layer_norm_desc& d, NormBackward a, float* sums, void* dw, void* db, hipStream_t st) {
    constexpr uint32_t N = Vec<T>::N;
    const Plan p = plan_of(d, kWidestBackward);
    a.lanes = p.lanes;
    const bool alone = p.sums_inside && p.parts == 1u;
    if (alone)
        a.dw = dw, a.db = db;
    else if (dw || db)
        a.sums = sums;
    const auto lds_of = [&](uint32_t vpl, uint32_t u, bool in_lds) {
        const uint32_t sums = p.lanes * vpl * N * 2u * 4u, turns = 2u * 2u * u * 16u * 4u;
        return p.lanes ? sums : turns + (in_lds ? vpl * N * 1024u * 4u : 0u);
    };
    const dim3 parts(p.parts);
#define PXR_NORM(NT, VPL, U, SUMS, GRID)                                                                                                      \
    do {                                                                                                                                      \
        const uint32_t lds = lds_of(VPL, U, SUMS && NT == 1024);                                                                              \
        if (const hipError_t rc = allow_lds<&norm_backward_kernel<T, P, NT, VPL, U, SUMS>>(lds); rc != hipSuccess) return rc;                 \
        hipLaunchKernelGGL((norm_backward_kernel<T, P, NT, VPL, U, SUMS>), GRID, dim3(kThreadsOf(NT)), lds, st, a);                           \
    } while (0)
    if (p.sums_inside) {
        if (d.n_rows) {
            if (d.width < N)
                hipLaunchKernelGGL((norm_backward_kernel<T, P, 0, 1, 2, true, true>), parts, dim3(kSubThreads), lds_of(1, 2, false), st, a);
            else if (p.vectors <= 64u)
                PXR_NORM(0, 1, 2, true, parts);
            else if (p.vectors <= 128u)
                PXR_NORM(0, 2, 1, true, parts);
            else if (p.vectors <= 256u)
                PXR_NORM(256, 1, 2, true, parts);
            else if (p.vectors <= 512u)
                PXR_NORM(512, 1, 2, true, parts);
            else if (p.vectors <= 1024u)
                PXR_NORM(512, 2, 1, true, parts);
            else if (p.vectors <= 2048u)
                PXR_NORM(1024, 2, 1, true, parts);
            else if (N == 8u || p.vectors <= 4096u)
                PXR_NORM(1024, 4, 1, true, parts);
            else if constexpr (N == 4u)
                PXR_NORM(1024, 8, 1, true, parts);
        }
    } else {
        // (the sums first: dx may be dy or x itself)
        if (a.sums && d.n_rows)
            hipLaunchKernelGGL((norm_sums_kernel<T>), dim3((p.vectors + 63u) / 64u, p.parts), dim3(256), 0, st, a, p.rows);
        if (d.n_rows) {
            bool done = false;
            if constexpr (N == 8u)
                if (p.vectors <= 8192u) {
                    PXR_NORM(1024, 8, 1, false, dim3((uint32_t)(d.n_rows < 2u * kCus ? d.n_rows : 2u * kCus)));
                    done = true;
                }
            if (!done) hipLaunchKernelGGL((norm_dx_wide_kernel<T, P>), dim3((uint32_t)d.n_rows), dim3(1024), 0, st, a);
        }
    }
#undef PXR_NORM
    if ((dw || db) && !alone) {
        const uint32_t need = (uint32_t)((2ull * d.width + 63u) / 64u), layers = (need + kFinishAcross - 1u) / kFinishAcross;
        hipLaunchKernelGGL((norm_finish_kernel<P>), dim3(layers > 1u ? kFinishAcross : need, layers), dim3(1024), 0, st, a.sums, p.parts, d.width,
                           static_cast<P*>(dw), static_cast<P*>(db));
    }
    return hipSuccess;
}

int launched(std::string& err, hipError_t rc = hipSuccess) {
    if (rc == hipSuccess) rc = hipGetLastError();
    if (rc == hipSuccess) return PXR_OK;
    err = std::string("kernel launch failed: ") + hipGetErrorString(rc);
    return PXR_ERR_DEVICE;
}

}  // namespace

size_t layer_norm_workspace(const pxr_layer_norm_desc& d) {
    const Plan p = plan_of(d, kWidestBackward);
    return p.sums_inside && p.parts == 1u ? 0 : (size_t)p.parts * 2u * d.width * sizeof(float);
}

int launch_layer_norm_forward(const pxr_layer_norm_desc& d, const void* x, const void* w, const void* b, void* y, float* mean, float* rstd,
                              void* stream, std::string& err) {
    if (d.n_rows == 0) return PXR_OK;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const NormForward a{x, w, b, y, mean, rstd, d.x_stride, d.y_stride, (uint32_t)d.n_rows, d.width, 0u, d.eps};
    if (d.dtype == PXR_F32)
        forward_as<float, float>(d, a, st);
    else if (d.param_dtype == PXR_F32)
        forward_as<__bf16, float>(d, a, st);
    else
        forward_as<__bf16, __bf16>(d, a, st);
    return launched(err);
}

int launch_layer_norm_backward(const pxr_layer_norm_desc& d, const void* dy, const void* x, const float* mean, const float* rstd,
                               const void* w, void* dx, void* dw, void* db, void* ws, void* stream, std::string& err) {
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const NormBackward a{dy, x, mean, rstd, w, dx, nullptr, nullptr, nullptr, d.y_stride, d.x_stride, d.dx_stride, (uint32_t)d.n_rows, d.width, 0u};
    float* sums = static_cast<float*>(ws);
    if (d.dtype == PXR_F32) return launched(err, backward_as<float, float>(d, a, sums, dw, db, st));
    if (d.param_dtype == PXR_F32) return launched(err, backward_as<__bf16, float>(d, a, sums, dw, db, st));
    return launched(err, backward_as<__bf16, __bf16>(d, a, sums, dw, db, st));
}

}  // namespace pxr
