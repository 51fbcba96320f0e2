// Norms of queries and keys for each head, and their rotation by the step's position, in one pass (pxr_head_norm_* in include/pxr.h).  gfx950 only.
//
//   y = x rstd w,  rstd = 1 / sqrt(sum x^2 / d + eps);  of the first r values the pairs (y_i, y_{i + r/2}) are turned by p f_i:  (u, v) -> (u cos - v sin, v cos + u sin)
//   backward, g = dy turned back:  dx = rstd (w g - xh sum(w g xh) / d),  dw = sum over tokens and heads of g xh,  xh = x rstd
//
// A head's values are dealt in slots of two: the pairs that are turned, and the values behind them, the first half of those with the second, turned by nothing.  A
// lane has V slots next to each other, two requests of V values; 1 to 64 lanes have a head.  They keep the sines of one token for all of its heads.
//
// The angle is formed in whole numbers: f / 2 pi as a fraction of 2^64, times the position, modulo 2^64 is the angle in turns modulo one, exact but for the fraction's
// own rounding: positions of 2^31 are off by 2^-22 turns, where a product in fp32 has lost them all.
//
// Bound by HBM: 256 x 128 steps of 8 + 8 heads of 64 bfloat16 29 us, 134 MB at 4.6 TB/s; gradients of 512 x 256 of 16 + 4 heads 206 us, 1.01 GB at 4.9.  (Stores past the caches: no faster, since what
// follows finds the heads there.)

#include <hip/hip_runtime.h>

#include <algorithm>

#include "pxr_internal.h"

namespace pxr {
namespace {

// One tensor of heads: x, what leaves (y or dx), dy, its weight and the sums for it.
struct HeadsOf {
    const void *x, *dy, *weight;
    void* out;
    int64_t x_env, x_step, x_head, dy_env, dy_step, dy_head, out_env, out_step, out_head;
    uint32_t heads, parts;  // parts of U heads
};

struct HeadNormArgs {
    HeadsOf q, k;
    const uint64_t* turns;  // [r/2] turns per position, in fractions of 2^64
    const void* positions;
    int64_t positions_env, positions_step, first;
    uint64_t items;  // tokens * split
    uint32_t n_steps, d, half, rest, lanes, split, wide;  // half = r / 2; rest: slots behind them; wide: positions of 64 bits
    float eps, width;
    float* sums;  // [workgroups][2][d]
};

constexpr uint32_t kThreads = 256;
constexpr uint32_t kMostGroups = 1024;  // workgroups of a launch, which walk the tokens (gradients of 512 x 256 tokens as below: 2048 of them 219 us, 1024 214)

template <class T, int N>
__device__ __forceinline__ void load(const T* p, T (&v)[N]) { __builtin_memcpy(v, p, sizeof(v)); }  // (at the address of any value)

template <class T, int N>
__device__ __forceinline__ void store(T* p, const T (&v)[N]) { __builtin_memcpy(p, v, sizeof(v)); }

// sin and cos of an angle in fractions of 2^32 of a turn: of the angle to the nearest quarter by their series (the first terms left out are below 2^-28), then
// the quarters.
__device__ __forceinline__ void sine(uint32_t turn, float& s, float& c) {
    const uint32_t quarter = (turn + 0x20000000u) >> 30;
    // 2 pi / 2^32 times 30 bits, both in two parts: rounded once (a sixth of the root mean square of the sines' errors)
    constexpr double kTurn = 1.46291807926715968e-9;
    constexpr float kFirst = (float)kTurn, kRest = (float)(kTurn - (double)kFirst);
    const int whole = (int)(turn - (quarter << 30));
    const float first = (float)whole, rest = (float)(whole - (int)first);
    const float x = __builtin_fmaf(first, kFirst, __builtin_fmaf(first, kRest, rest * kFirst));
    const float z = x * x;
    float p = __builtin_fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
    p = __builtin_fmaf(z, p, 8.33333333e-3f);
    p = __builtin_fmaf(z, p, -1.66666667e-1f);
    const float near = __builtin_fmaf(x * z, p, x);
    float q = __builtin_fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
    q = __builtin_fmaf(z, q, -1.38888889e-3f);
    q = __builtin_fmaf(z, q, 4.16666667e-2f);
    q = __builtin_fmaf(z, q, -0.5f);
    const float far = __builtin_fmaf(z, q, 1.0f);
    const float a = quarter & 1u ? far : near, b = quarter & 1u ? near : far;
    s = quarter & 2u ? -a : a;
    c = (quarter + 1u) & 2u ? -b : b;
}

// 1 / sqrt(v), the last digit of the two roundings given back (a tenth of the root mean square of all errors of a turned value).
__device__ __forceinline__ float reciprocal_root(float v) {
    const float r = 1.0f / sqrtf(v), h = v * r;
    const float off = __builtin_fmaf(-h, r, 1.0f) - __builtin_fmaf(v, r, -h) * r;  // 1 - v r^2
    return v > 0.0f && v < __builtin_inff() ? __builtin_fmaf(0.5f * r, off, r) : r;
}

// Where the slots of vector number `vector` lie in a head, V of them next to each other, and which of their second values there are.
// kMoved: vectors end where the turned values, or those behind them, do: the last ones are moved back, over values that the vectors before them have too (both write the same bits; in sums they
// are the latter's, own_lo and own_hi say from which value on they are this one's).  Fewer than 2 V values behind the turned ones have no second half, and where their vector reaches into those it writes only what is its own.
template <int V, bool kMoved>
struct Slots {
    uint32_t lo, hi, slot, own_lo, own_hi;
    bool any, second, whole;
    __device__ __forceinline__ Slots(const HeadNormArgs& a, uint32_t vector) {
        slot = vector * V;
        own_lo = own_hi = 0;
        whole = true;
        if constexpr (kMoved) {
            const uint32_t turned = (a.half + V - 1u) / V, behind = a.d - 2u * a.half;
            if (vector < turned) {
                lo = min(slot, a.half - V);
                own_lo = own_hi = slot - lo;
                slot = lo;
                hi = lo + a.half;
                any = second = true;
            } else {
                const uint32_t s = slot - turned * V, seconds = behind >= 2u * V ? behind / 2u : 0u, firsts = behind - seconds;
                any = s < firsts;
                second = s < seconds;
                const int at = min((int)s, (int)firsts - V);
                lo = any ? (uint32_t)((int)(2u * a.half) + at) : 0u;
                own_lo = s - (uint32_t)at;
                whole = at >= 0;
                const uint32_t at_hi = second ? min(s, seconds - V) : 0u;
                hi = second ? 2u * a.half + firsts + at_hi : lo;
                own_hi = s - at_hi;
                slot = a.half;
            }
        } else {
            const bool turned = slot < a.half;
            any = slot < a.half + a.rest;
            lo = any ? (turned ? slot : a.half + slot) : 0u;
            hi = turned ? slot + a.half : a.half + a.rest + slot;
            second = any && hi + V <= a.d;
            if (!second) hi = lo;
        }
    }
    // Whether value v of the first ones, or of the second ones, is there and is this vector's.
    __device__ __forceinline__ bool has_lo(int v) const { return any && (!kMoved || (uint32_t)v >= own_lo); }
    __device__ __forceinline__ bool has_hi(int v) const { return second && (!kMoved || (uint32_t)v >= own_hi); }
};

// Sums over the lanes of a head, the same bits in each of them.
template <int U>
__device__ __forceinline__ void head_sums(float (&v)[U], uint32_t lanes) {
    for (uint32_t m = lanes >> 1; m >= 1; m >>= 1)
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] += __shfl_xor(v[u], m);
}

// K vectors of V slots a lane, U heads at a time.
template <class T, class P, int V, int K, int U, bool kMoved, bool kBack>
__global__ __launch_bounds__(kThreads) void head_norm_kernel(const HeadNormArgs a) {
    __shared__ float shared[kBack ? kThreads / 64 * 2 * 256 : 1];
    const uint32_t lanes = a.lanes, l = threadIdx.x & (lanes - 1u), group = threadIdx.x / lanes, groups = kThreads / lanes;
    float weight[2][K][2][V], dw[kBack ? 2 : 1][K][2][V];
    uint64_t turns[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const Slots<V, kMoved> at(a, l + k * lanes);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            turns[k][v] = at.slot + v < a.half ? a.turns[at.slot + v] : 0u;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const P* p = static_cast<const P*>(w ? a.k.weight : a.q.weight);
                weight[w][k][0][v] = !at.any ? 0.0f : p ? (float)p[at.lo + v] : 1.0f;
                weight[w][k][1][v] = !at.second ? 0.0f : p ? (float)p[at.hi + v] : 1.0f;
                if constexpr (kBack) dw[w][k][0][v] = dw[w][k][1][v] = 0.0f;
            }
        }
    }
    for (uint64_t item = (uint64_t)blockIdx.x * groups + group; item < a.items; item += (uint64_t)gridDim.x * groups) {
        const uint32_t token = (uint32_t)(item / a.split), first = (uint32_t)(item - (uint64_t)token * a.split);
        const uint32_t env = token / a.n_steps, step = token - env * a.n_steps;
        int64_t position = a.first + (int64_t)step;
        if (a.positions) {
            const int64_t i = (int64_t)env * a.positions_env + (int64_t)step * a.positions_step;
            position = a.wide ? static_cast<const int64_t*>(a.positions)[i] : (int64_t)static_cast<const int32_t*>(a.positions)[i];
        }
        float sin[K][V], cos[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v) sine((uint32_t)(((uint64_t)position * turns[k][v]) >> 32), sin[k][v], cos[k][v]);

        const auto part = [&](const HeadsOf& t, const float (&w)[K][2][V], float (&sum)[K][2][V], uint32_t head0) {
            const T* x = static_cast<const T*>(t.x) + ((int64_t)env * t.x_env + (int64_t)step * t.x_step);
            const T* dy = static_cast<const T*>(t.dy) + (kBack ? (int64_t)env * t.dy_env + (int64_t)step * t.dy_step : 0);
            T* out = static_cast<T*>(t.out) + ((int64_t)env * t.out_env + (int64_t)step * t.out_step);
            T xs[U][K][2][V], ds[kBack ? U : 1][K][2][V];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t head = min(head0 + u, t.heads - 1u);  // (past the last one: the last one again)
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const Slots<V, kMoved> at(a, l + k * lanes);
                    load(x + head * t.x_head + at.lo, xs[u][k][0]);
                    load(x + head * t.x_head + at.hi, xs[u][k][1]);
                    if constexpr (kBack) {
                        load(dy + head * t.dy_head + at.lo, ds[u][k][0]);
                        load(dy + head * t.dy_head + at.hi, ds[u][k][1]);
                    }
                }
            }
            float both[kBack ? 2 * U : U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float s = 0.0f, along = 0.0f;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const Slots<V, kMoved> at(a, l + k * lanes);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const float lo = at.has_lo(v) ? (float)xs[u][k][0][v] : 0.0f, hi = at.has_hi(v) ? (float)xs[u][k][1][v] : 0.0f;
                        s = __builtin_fmaf(lo, lo, s);
                        s = __builtin_fmaf(hi, hi, s);
                        if constexpr (kBack) {
                            const float dlo = at.any ? (float)ds[u][k][0][v] : 0.0f, dhi = at.second ? (float)ds[u][k][1][v] : 0.0f;
                            const float glo = __builtin_fmaf(dlo, cos[k][v], dhi * sin[k][v]), ghi = __builtin_fmaf(dhi, cos[k][v], -(dlo * sin[k][v]));
                            along = __builtin_fmaf(w[k][0][v] * glo, lo, along);
                            along = __builtin_fmaf(w[k][1][v] * ghi, hi, along);
                        }
                    }
                }
                both[u] = s;
                if constexpr (kBack) both[U + u] = along;
            }
            head_sums(both, lanes);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (head0 + u >= t.heads) continue;
                const float rstd = reciprocal_root(both[u] / a.width + a.eps);
                float back = 0.0f;
                if constexpr (kBack) back = both[U + u] * rstd / a.width * rstd;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const Slots<V, kMoved> at(a, l + k * lanes);
                    T lo[V], hi[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const float xlo = (float)xs[u][k][0][v] , xhi = (float)xs[u][k][1][v];
                        if constexpr (kBack) {
                            const float dlo = (float)ds[u][k][0][v], dhi = at.second ? (float)ds[u][k][1][v] : 0.0f;
                            const float glo = __builtin_fmaf(dlo, cos[k][v], dhi * sin[k][v]), ghi = __builtin_fmaf(dhi, cos[k][v], -(dlo * sin[k][v]));
                            lo[v] = (T)(rstd * __builtin_fmaf(w[k][0][v], glo, -(xlo * back)));
                            hi[v] = (T)(rstd * __builtin_fmaf(w[k][1][v], ghi, -(xhi * back)));
                            sum[k][0][v] = __builtin_fmaf(glo, xlo * rstd, sum[k][0][v]);
                            sum[k][1][v] = __builtin_fmaf(ghi, xhi * rstd, sum[k][1][v]);
                        } else {
                            const float ylo = xlo * rstd * w[k][0][v], yhi = xhi * rstd * w[k][1][v];
                            lo[v] = (T)__builtin_fmaf(ylo, cos[k][v], -(yhi * sin[k][v]));
                            hi[v] = (T)__builtin_fmaf(yhi, cos[k][v], ylo * sin[k][v]);
                        }
                    }
                    T* to = out + (int64_t)(head0 + u) * t.out_head;
                    if (at.any && at.whole) store(to + at.lo, lo);
                    if (at.second) store(to + at.hi, hi);
                    if constexpr (kMoved)
                        if (at.any && !at.whole)
#pragma unroll
                            for (int v = 0; v < V; ++v)
                                if (at.has_lo(v)) to[at.lo + v] = lo[v];
                }
            }
        };
        for (uint32_t p = first; p < a.q.parts; p += a.split) part(a.q, weight[0], dw[0], p * U);
        // (the keys' parts come behind the queries': the first of them that is this group's)
        uint32_t p = first;
        if (p < a.q.parts) p += (a.q.parts - p + a.split - 1u) / a.split * a.split;
        for (; p < a.q.parts + a.k.parts; p += a.split) part(a.k, weight[1], dw[kBack ? 1 : 0], (p - a.q.parts) * U);
    }
    if constexpr (kBack) {
        if (!a.sums) return;
        const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const Slots<V, kMoved> at(a, l + k * lanes);
#pragma unroll
                for (int side = 0; side < 2; ++side)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        float s = dw[t][k][side][v];
                        for (uint32_t m = lanes; m < 64u; m <<= 1) s += __shfl_xor(s, m);
                        if (lane < lanes && (side ? at.has_hi(v) : at.has_lo(v))) shared[(wave * 2 + t) * 256 + (side ? at.hi : at.lo) + v] = s;
                    }
            }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < 2 * a.d; i += kThreads) {
            const uint32_t t = i / a.d, c = i - t * a.d;
            float s = 0.0f;
            for (uint32_t w = 0; w < kThreads / 64; ++w) s += shared[(w * 2 + t) * 256 + c];
            a.sums[(size_t)blockIdx.x * 2 * a.d + i] = s;
        }
    }
}

// The workgroups' sums, in their order: 16 columns and 16 runs of rows a workgroup.
template <class P>
__global__ __launch_bounds__(256) void head_norm_sums_kernel(const float* sums, uint32_t rows, uint32_t d, P* dq_weight, P* dk_weight) {
    __shared__ float shared[16][17];
    const uint32_t c = threadIdx.x & 15u, run = threadIdx.x >> 4, column = blockIdx.x * 16u + c;
    float s = 0.0f;
    if (column < 2 * d)
#pragma unroll 8
        for (uint32_t r = run; r < rows; r += 16u) s += sums[(size_t)r * 2 * d + column];
    shared[run][c] = s;
    __syncthreads();
    if (run || column >= 2 * d) return;
    for (uint32_t r = 1; r < 16u; ++r) s += shared[r][c];
    P* to = column < d ? dq_weight : dk_weight;
    if (to) to[column < d ? column : column - d] = (P)s;
}

struct HeadNormShape {
    uint32_t V, K, lanes, split, groups;  // groups: workgroups
    bool moved;
};

// Heads that a group of lanes has in flight, and the values of one of its requests: more are more registers and fewer wavefronts.  (Gradients of 512 x 256 tokens of 16 + 4 heads of 64 bfloat16: 4 heads in
// requests of 16 bytes 358 us, 2 of them 237, 2 in requests of 8 bytes 216; forward, 256 x 128 tokens of 8 + 8 heads: 31, 32.7 and 33.)
constexpr uint32_t kMovedValues = 4;  // of a vector that is moved back
constexpr uint32_t together(bool backward) { return backward ? 2u : 4u; }
constexpr uint32_t most_values(uint32_t dtype, bool backward) { return dtype == PXR_F32 || backward ? 4u : 8u; }

HeadNormShape shape_of(const HeadNormConsts& c, uint32_t dtype, uint64_t tokens, uint32_t n_heads, uint32_t n_key_heads, bool backward) {
    HeadNormShape s{};
    const uint32_t half = c.r / 2u, behind = c.d - c.r, slots = half + (behind + 1u) / 2u;
    s.V = most_values(dtype, backward);
    while (s.V > 1u && (half % s.V || behind % (2u * s.V))) s.V /= 2u;
    uint32_t vectors = slots / s.V;
    // Where whole vectors are short, they are of kMovedValues and the last ones moved back.  (256 x 128 steps of 8 + 8 heads of bfloat16, 100 values, 50 of them turned: one by one 100 us, so 59, gradients 154
    // and 107; 20 of 100 turned: by twos 62, so 54, but gradients 100 and 102 and, in fp32, 36 of 64 turned 51 and 53.)
    if ((s.V == 1u || (s.V == 2u && 2u * kMovedValues == most_values(dtype, backward))) && (half == 0u || half >= kMovedValues) && c.d >= kMovedValues) {
        s.V = kMovedValues;
        s.moved = true;
        vectors = (half + s.V - 1u) / s.V + ((behind >= 2u * s.V ? (behind + 1u) / 2u : behind) + s.V - 1u) / s.V;
    }
    s.lanes = 1u;
    while (s.lanes < 64u && s.lanes < vectors) s.lanes *= 2u;
    s.K = s.lanes < vectors ? 2u : 1u;
    const uint32_t U = together(backward), parts = (n_heads + U - 1u) / U + (n_key_heads + U - 1u) / U;
    // a token's heads are shared out where the tokens alone are too few wavefronts (512 and 4096 of them: 16 x 100 steps of 8 + 2 heads 14.1 and 14.4 us, 13.4 so)
    const uint64_t waves = (tokens * s.lanes + 63u) / 64u;
    s.split = (uint32_t)std::min<uint64_t>(std::max(parts, 1u), waves ? (2048u + waves - 1u) / waves : 1u);
    const uint32_t per_group = kThreads / s.lanes;
    s.groups = (uint32_t)std::min<uint64_t>(kMostGroups, (tokens * s.split + per_group - 1u) / per_group);
    return s;
}

template <class T, class P, bool kBack>
hipError_t launch(const HeadNormShape& s, const HeadNormArgs& a, hipStream_t st) {
    constexpr int U = (int)together(kBack);
    const dim3 grid(s.groups), threads(kThreads);
    if (s.moved)
        hipLaunchKernelGGL((head_norm_kernel<T, P, kMovedValues, 1, U, true, kBack>), grid, threads, 0, st, a);
    else if (s.K == 2u)
        hipLaunchKernelGGL((head_norm_kernel<T, P, 1, 2, U, false, kBack>), grid, threads, 0, st, a);
    else if (s.V == 1u)
        hipLaunchKernelGGL((head_norm_kernel<T, P, 1, 1, U, false, kBack>), grid, threads, 0, st, a);
    else if (s.V == 2u)
        hipLaunchKernelGGL((head_norm_kernel<T, P, 2, 1, U, false, kBack>), grid, threads, 0, st, a);
    else if (s.V == 4u)
        hipLaunchKernelGGL((head_norm_kernel<T, P, 4, 1, U, false, kBack>), grid, threads, 0, st, a);
    else if constexpr (sizeof(T) == 2 && !kBack)
        hipLaunchKernelGGL((head_norm_kernel<T, P, 8, 1, U, false, kBack>), grid, threads, 0, st, a);
    return hipGetLastError();
}

template <bool kBack>
hipError_t launch_typed(const pxr_heads& r, const HeadNormShape& s, const HeadNormArgs& a, hipStream_t st) {
    if (r.dtype == PXR_F32) return launch<float, float, kBack>(s, a, st);
    return r.param_dtype == PXR_F32 ? launch<__bf16, float, kBack>(s, a, st) : launch<__bf16, __bf16, kBack>(s, a, st);
}

HeadNormArgs arguments(const HeadNormConsts& c, const pxr_heads& r, const HeadNormShape& s, const pxr_tokens* q_out, const pxr_tokens* k_out,
                       const pxr_tokens* dq, const pxr_tokens* dk) {
    HeadNormArgs a{};
    const uint32_t U = together(dq || dk);
    const auto fill = [U](HeadsOf& t, const pxr_tokens& x, const void* weight, uint32_t heads, const pxr_tokens* out, const pxr_tokens* dy) {
        t.heads = heads;
        t.parts = (heads + U - 1u) / U;
        if (!heads) return;
        t.x = x.data;
        t.x_env = x.env;
        t.x_step = x.step;
        t.x_head = x.head;
        t.weight = weight;
        t.out = out->data;
        t.out_env = out->env;
        t.out_step = out->step;
        t.out_head = out->head;
        if (!dy) return;
        t.dy = dy->data;
        t.dy_env = dy->env;
        t.dy_step = dy->step;
        t.dy_head = dy->head;
    };
    fill(a.q, r.q, r.d_q_weight, r.n_heads, q_out, dq);
    fill(a.k, r.k, r.d_k_weight, r.n_key_heads, k_out, dk);
    a.turns = c.turns;
    a.positions = r.d_positions;
    a.positions_env = r.positions_env;
    a.positions_step = r.positions_step;
    a.wide = r.position_bits == 64u;
    a.first = r.first;
    a.items = (uint64_t)r.n_envs * r.n_steps * s.split;
    a.n_steps = r.n_steps;
    a.d = c.d;
    a.half = c.r / 2u;
    a.rest = (c.d - c.r + 1u) / 2u;
    a.lanes = s.lanes;
    a.split = s.split;
    a.eps = c.eps;
    a.width = (float)c.d;
    return a;
}

int result(hipError_t rc, std::string& err) {
    if (rc == hipSuccess) return PXR_OK;
    err = std::string("kernel launch failed: ") + hipGetErrorString(rc);
    return PXR_ERR_DEVICE;
}

}  // namespace

size_t head_norm_workspace(const HeadNormConsts& c, const pxr_heads& r) {
    return (size_t)shape_of(c, r.dtype, (uint64_t)r.n_envs * r.n_steps, r.n_heads, r.n_key_heads, true).groups * 2 * c.d * sizeof(float);
}

int launch_head_norm_forward(const HeadNormConsts& c, const pxr_heads& r, const pxr_tokens* q_out, const pxr_tokens* k_out, void* stream, std::string& err) {
    const HeadNormShape s = shape_of(c, r.dtype, (uint64_t)r.n_envs * r.n_steps, r.n_heads, r.n_key_heads, false);
    if (!s.groups || r.n_heads + r.n_key_heads == 0) return PXR_OK;
    return result(launch_typed<false>(r, s, arguments(c, r, s, q_out, k_out, nullptr, nullptr), static_cast<hipStream_t>(stream)), err);
}

int launch_head_norm_backward(const HeadNormConsts& c, const pxr_heads& r, const pxr_tokens* dq_out, const pxr_tokens* dk_out, const pxr_tokens* dq,
                              const pxr_tokens* dk, void* dq_weight, void* dk_weight, void* ws, void* stream, std::string& err) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const HeadNormShape s = shape_of(c, r.dtype, (uint64_t)r.n_envs * r.n_steps, r.n_heads, r.n_key_heads, true);
    HeadNormArgs a = arguments(c, r, s, dq, dk, dq_out, dk_out);
    const bool sums = dq_weight || dk_weight;
    a.sums = sums ? static_cast<float*>(ws) : nullptr;
    hipError_t rc = s.groups ? launch_typed<true>(r, s, a, st) : hipSuccess;
    if (rc == hipSuccess && sums) {
        const dim3 grid((2 * c.d + 15u) / 16u), threads(256);
        if (r.param_dtype == PXR_F32)
            hipLaunchKernelGGL((head_norm_sums_kernel<float>), grid, threads, 0, st, a.sums, s.groups, c.d, static_cast<float*>(dq_weight), static_cast<float*>(dk_weight));
        else
            hipLaunchKernelGGL((head_norm_sums_kernel<__bf16>), grid, threads, 0, st, a.sums, s.groups, c.d, static_cast<__bf16*>(dq_weight), static_cast<__bf16*>(dk_weight));
        rc = hipGetLastError();
    }
    return result(rc, err);
}

}  // namespace pxr
