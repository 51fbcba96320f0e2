// A gated linear recurrence (pxr_gated_recurrence_* in include/pxr.h).  gfx950 only.
//
//   h_t = k_t h_{t-1} + b_t,   a_t = 1 / (1 + exp(-gate_t)),   k_t = (t begins an episode ? 0 : a_t),   b_t = (coupled ? 1 - a_t : 1) x_t
//
// With r_t the gradient that step t hands to the state before it and dout_t that of its output:
//   L_t = dout_t + r_{t+1},   r_t = k_t L_t,   dx_t = (coupled ? 1 - a_t : 1) L_t,   dgate_t = a_t (1 - a_t) L_t (h'_{t-1} - (coupled ? x_t : 0))
// where h'_{t-1} is what step t saw of the state: 0 where it begins an episode.  r before the first step is the gradient of the state.
//
// Steps in a row are one step: with A their product of k, h = A h_before + H and r = A r_after + R, H and R from zero.  A wavefront has C steps of its channels in
// registers; the wavefronts of a workgroup have steps that follow each other and tell each other (A, H, R) through LDS, so that everything is read once.  A
// product A of 0 passes nothing on, whatever the state holds: what is not finite stays on its side of an episode's beginning.
//
// Bound by HBM.

#include <hip/hip_runtime.h>

#include <algorithm>

#include "pxr_internal.h"

namespace pxr {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// V values of a row as they came.
template <class T, int V>
struct Raw;
template <int V>
struct Raw<float, V> {
    float w[V];
    __device__ __forceinline__ float get(int i) const { return w[i]; }
};
template <>
struct Raw<__bf16, 2> {
    uint32_t w;
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i ? w & 0xFFFF0000u : w << 16); }
};
template <>
struct Raw<__bf16, 1> {
    uint16_t w;
    __device__ __forceinline__ float get(int) const { return __uint_as_float((uint32_t)w << 16); }
};

template <class T, int V>
__device__ __forceinline__ Raw<T, V> load(const T* p) {
    Raw<T, V> r;
    __builtin_memcpy(&r, p, sizeof(T) * V);  // (rows may begin at any element: the memory takes requests at any address)
    return r;
}

// Values [from, V) of a vector leave (rounded to nearest even), past the caches: nothing here reads them again.
template <class T, int V>
__device__ __forceinline__ void store(T* p, const float (&f)[V], int from) {
    T v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (T)f[i];
    if (from == 0) {
        typedef T some __attribute__((ext_vector_type(V), aligned(sizeof(T))));
        some s;
        __builtin_memcpy(&s, v, sizeof(v));
        __builtin_nontemporal_store(s, reinterpret_cast<some*>(p));
        return;
    }
#pragma unroll
    for (int i = 1; i < V; ++i)
        if (i >= from) p[i] = v[i];
}

// A gate as one number: a where it is the smaller of a and 1 - a, otherwise -(1 - a).  Each of the two is 1 less the other where that loses nothing.
template <class T>
__device__ __forceinline__ float gate_of(float g) {
    const float m = fabsf(g) > 100.0f ? 100.0f : fabsf(g);  // (a NaN stays one)
    const float t = m * -1.44269504f;
    float e = __builtin_amdgcn_exp2f(t);  // exp(-|g|)
    // (what t has lost in 24 bits is |g| of their last one: of 32 bits' results as well)
    if (sizeof(T) == 4) e = __builtin_fmaf(e, __builtin_fmaf(m, -1.44269504f, -t) * 0.69314718f - m * 1.3346e-8f, e);
    return copysignf(e * __builtin_amdgcn_rcpf(1.0f + e), -g);
}
__device__ __forceinline__ bool mostly(float s) { return (int)__float_as_uint(s) < 0; }  // a >= 1/2
__device__ __forceinline__ float taken(float s) { return mostly(s) ? -s : 1.0f - s; }    // 1 - a
// a v + b.  Where a is all but 1 it is v less a little: a itself, rounded, would be off in the same direction in every step of a gate that stays where it is (200
// steps of gates around 10: a state off by 3e-6, 3e-7 so).
__device__ __forceinline__ float kept(float s, float v, float b) { return __builtin_fmaf(s, v, mostly(s) ? v + b : b); }
__device__ __forceinline__ float kept(float s, float v) { return __builtin_fmaf(s, v, mostly(s) ? v : 0.0f); }

// Products in which 0 wins, over what is not a number as well.
__device__ __forceinline__ float times(float A, float B) { return A == 0.0f || B == 0.0f ? 0.0f : A * B; }
// What steps in a row (product A, own result H) make of a state.
__device__ __forceinline__ float through(float A, float H, float state) { return A != 0.0f ? __builtin_fmaf(A, state, H) : H; }

struct Recurrence {
    const void *x, *gate, *dout;
    void *out, *dgate;  // out: dx in the backward pass
    int64_t x_env, x_step, gate_env, gate_step, dout_env, dout_step, out_env, out_step, dgate_env, dgate_step;
    const uint8_t* resets;
    int64_t resets_env, resets_step;
    const float *state_in, *after;  // before the first step; the gradient of the state after the last one (null = zeros)
    float *state_out, *dstate;      // null = not wanted
    float* joined;                  // [segments][2 or 3 planes][n_envs * width]: A, H (, R) of the segments; of H and R, later, what comes in
    uint32_t n_envs, n_steps, width, lanes, strips, segments, seg_steps, coupled;
};

enum { kForward, kForwardSums, kBackward, kBackwardSums };
constexpr uint32_t kMostWaves = 8;

// Where a lane's channels are.  A row that ends inside a vector has its last vector moved back to its end, lanes behind the row have that one as well: values
// before `from` are another lane's.
template <int V>
struct Lane {
    uint32_t env, at;
    int from;
    __device__ __forceinline__ Lane(const Recurrence& a, uint32_t rows, uint32_t strip) {
        const uint32_t lane = threadIdx.x & 63u, in_row = lane & (a.lanes - 1u);
        const uint32_t e = rows * (64u / a.lanes) + lane / a.lanes, c = (strip * a.lanes + in_row) * V;
        env = min(e, a.n_envs - 1u);
        at = min(c, a.width - V);
        from = e < a.n_envs ? (int)min(c - at, (uint32_t)V) : V;
    }
};

// C steps of V channels a lane; kWhat: see the enum.  One workgroup: seg_steps steps (backward: at most what its wavefronts hold) of a strip of channels of
// 64 / lanes environments.
template <class T, int V, int C, int kWhat>
__global__ __launch_bounds__(kMostWaves * 64) void recurrence_kernel(const Recurrence a) {
    constexpr bool kBack = kWhat >= kBackward, kSums = kWhat == kForwardSums || kWhat == kBackwardSums;
    constexpr int kPlanes = kBack ? 3 : 2;
    __shared__ float shared[kBack ? 1 : 2][kMostWaves][kPlanes][V][64];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const uint32_t strip = blockIdx.x % a.strips, rest = blockIdx.x / a.strips, seg = rest % a.segments, rows = rest / a.segments;
    const Lane<V> at(a, rows, strip);
    const T* x = static_cast<const T*>(a.x) + (int64_t)at.env * a.x_env + at.at;
    const T* gate = static_cast<const T*>(a.gate) + (int64_t)at.env * a.gate_env + at.at;
    const T* dout = kBack ? static_cast<const T*>(a.dout) + (int64_t)at.env * a.dout_env + at.at : nullptr;
    const size_t cell = (size_t)at.env * a.width + at.at, cells = (size_t)a.n_envs * a.width;
    const uint32_t begin = seg * a.seg_steps, end = min(begin + a.seg_steps, a.n_steps);

    // what comes in
    float state[V], later[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        state[i] = later[i] = 0.0f;
        if (kSums) continue;
        const float* plane = a.joined + (size_t)seg * kPlanes * cells;
        state[i] = a.segments > 1u ? plane[cells + cell + i] : a.state_in ? a.state_in[cell + i] : 0.0f;
        if (kBack) later[i] = a.segments > 1u ? plane[2 * cells + cell + i] : a.after ? a.after[cell + i] : 0.0f;
    }
    float whole[V];  // the product over the segment (sums)
#pragma unroll
    for (int i = 0; i < V; ++i) whole[i] = 1.0f;

    uint32_t turn = 0;
    for (uint32_t block = begin; block < end; block += waves * C, turn ^= 1u) {
        const uint32_t first = block + wave * C;
        const int n = first < end ? (int)min(end - first, (uint32_t)C) : 0;  // this wavefront's steps
        Raw<T, V> xs[C], gs[C], ds[kBack ? C : 1];
        uint32_t cuts = 0;
        if (n) {
            // (steps past the last one are the last one again)
            const T *g = gate + (int64_t)first * a.gate_step, *v = x + (int64_t)first * a.x_step, *d = kBack ? dout + (int64_t)first * a.dout_step : nullptr;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                gs[j] = load<T, V>(g);
                xs[j] = load<T, V>(v);
                if (kBack) ds[j] = load<T, V>(d);
                g += j + 1 < n ? a.gate_step : 0;
                v += j + 1 < n ? a.x_step : 0;
                if (kBack) d += j + 1 < n ? a.dout_step : 0;
            }
            if (a.resets) {  // the first C of an environment's lanes ask for one of its steps each
                const uint32_t in_row = lane & (a.lanes - 1u);
                const bool mark = in_row < (uint32_t)n && a.resets[(int64_t)at.env * a.resets_env + (int64_t)(first + in_row) * a.resets_step];
                const uint64_t marks = __ballot(mark) >> (lane - in_row);
                cuts = (uint32_t)marks & (C == 32 ? 0xFFFFFFFFu : (1u << (C & 31)) - 1u);
            }
        }
        // each wavefront's steps by themselves
        float A[V], H[V], R[V];
        float h[C][V], s[C][V];  // forward: results from zero, and the products up to them; backward: the states that came in, and the gates
#pragma unroll
        for (int i = 0; i < V; ++i) {
            A[i] = 1.0f;
            H[i] = R[i] = 0.0f;
        }
        if (n) {
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const bool cut = cuts >> j & 1u;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float g = gate_of<T>(gs[j].get(i)), b = a.coupled ? taken(g) * xs[j].get(i) : xs[j].get(i);
                    if (j < n) {
                        A[i] = cut || A[i] == 0.0f ? 0.0f : kept(g, A[i]);
                        H[i] = cut ? b : kept(g, H[i], b);
                    }
                    h[j][i] = H[i];
                    s[j][i] = kBack ? g : A[i];
                }
            }
            if (kBack)
#pragma unroll
                for (int j = C - 1; j >= 0; --j)
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (j < n) R[i] = cuts >> j & 1u ? 0.0f : kept(s[j][i], ds[j].get(i) + R[i]);
        }
        float(&told)[kMostWaves][kPlanes][V][64] = shared[kBack ? 0 : turn];  // (the block after the next one writes here again)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            told[wave][0][i][lane] = A[i];
            told[wave][1][i][lane] = H[i];
            if constexpr (kBack) told[wave][2][i][lane] = R[i];
        }
        __syncthreads();
        float mine[V], mine_later[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            mine[i] = state[i];
            mine_later[i] = later[i];
            for (uint32_t w = 0; w < waves; ++w) {
                if (w == wave) mine[i] = state[i];
                const float p = told[w][0][i][lane];
                state[i] = through(p, told[w][1][i][lane], state[i]);
                if (kSums) whole[i] = times(whole[i], p);
            }
            if constexpr (kBack) {
                for (uint32_t w = waves; w-- > 0;) {
                    if (w == wave) mine_later[i] = later[i];
                    later[i] = through(told[w][0][i][lane], told[w][2][i][lane], later[i]);
                }
            }
        }
        if (kSums || !n) continue;
        if constexpr (kWhat == kForward) {
            T* out = static_cast<T*>(a.out) + ((int64_t)at.env * a.out_env + at.at + (int64_t)first * a.out_step);
#pragma unroll
            for (int j = 0; j < C; ++j) {
                float y[V];
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = through(s[j][i], h[j][i], mine[i]);
                if (j < n && at.from < V) store<T, V>(out, y, at.from);
                out += a.out_step;
            }
        } else if constexpr (kWhat == kBackward) {
            // the states again, now from what came in
#pragma unroll
            for (int j = 0; j < C; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float b = a.coupled ? taken(s[j][i]) * xs[j].get(i) : xs[j].get(i);
                    h[j][i] = cuts >> j & 1u ? 0.0f : mine[i];
                    mine[i] = cuts >> j & 1u ? b : kept(s[j][i], mine[i], b);
                }
            T* dx = static_cast<T*>(a.out) + ((int64_t)at.env * a.out_env + at.at + (int64_t)(first + n - 1) * a.out_step);
            T* dgate = static_cast<T*>(a.dgate) + ((int64_t)at.env * a.dgate_env + at.at + (int64_t)(first + n - 1) * a.dgate_step);
#pragma unroll
            for (int j = C - 1; j >= 0; --j) {
                if (j >= n) continue;
                float to_x[V], to_gate[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float take = taken(s[j][i]), L = ds[j].get(i) + mine_later[i];
                    to_x[i] = a.coupled ? take * L : L;
                    const float kept_L = kept(s[j][i], L);
                    to_gate[i] = take * kept_L * (a.coupled ? h[j][i] - xs[j].get(i) : h[j][i]);
                    mine_later[i] = cuts >> j & 1u ? 0.0f : kept_L;
                }
                if (at.from < V) {
                    store<T, V>(dx, to_x, at.from);
                    store<T, V>(dgate, to_gate, at.from);
                }
                dx -= a.out_step;
                dgate -= a.dgate_step;
            }
        }
    }
    if (wave == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (i < at.from) continue;
            if (kSums) {
                float* plane = a.joined + (size_t)seg * kPlanes * cells + cell + i;
                plane[0] = whole[i];
                plane[cells] = state[i];
                if (kBack) plane[2 * cells] = later[i];
            } else if (kWhat == kForward) {
                if (a.state_out && seg + 1u == a.segments) a.state_out[cell + i] = state[i];
            } else {
                if (a.dstate && seg == 0) a.dstate[cell + i] = later[i];
            }
        }
    }
}

// Of every segment's own results: what comes into it.  A workgroup has 64 channels, its wavefronts segments that follow each other.
constexpr uint32_t kJoinWaves = 16;
template <bool kBack>
__global__ __launch_bounds__(kJoinWaves * 64) void recurrence_join_kernel(const Recurrence a) {
    constexpr uint32_t kPlanes = kBack ? 3 : 2;
    __shared__ float told[kJoinWaves][kPlanes][64];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const size_t cells = (size_t)a.n_envs * a.width, own = (size_t)blockIdx.x * 64u + lane, cell = own < cells ? own : cells - 1u;
    const uint32_t each = (a.segments + kJoinWaves - 1u) / kJoinWaves, begin = min(wave * each, a.segments), end = min(begin + each, a.segments);
    float* const first = a.joined + cell;
    const size_t step = kPlanes * cells;
    float A = 1.0f, H = 0.0f, R = 0.0f;
#pragma unroll 8
    for (uint32_t s = begin; s < end; ++s) {
        const float* p = first + s * step;
        if (kBack) R = through(A, R, p[2 * cells]);
        H = through(p[0], p[cells], H);
        A = times(A, p[0]);
    }
    told[wave][0][lane] = A;
    told[wave][1][lane] = H;
    if constexpr (kBack) told[wave][2][lane] = R;
    __syncthreads();
    float state = a.state_in ? a.state_in[cell] : 0.0f, later = kBack && a.after ? a.after[cell] : 0.0f;
    for (uint32_t w = 0; w < wave; ++w) state = through(told[w][0][lane], told[w][1][lane], state);
    if constexpr (kBack)
        for (uint32_t w = kJoinWaves; --w > wave;) later = through(told[w][0][lane], told[w][2][lane], later);
    if (own >= cells) return;
#pragma unroll 8
    for (uint32_t s = begin; s < end; ++s) {
        float* p = first + s * step;
        const float came = state;
        state = through(p[0], p[cells], state);
        p[cells] = came;
    }
    if (kBack)
#pragma unroll 8
        for (uint32_t s = end; s-- > begin;) {
            float* p = first + s * step;
            const float came = later;
            later = through(p[0], p[2 * cells], later);
            p[2 * cells] = came;
        }
}

// One step: a lane has V channels of an environment, the state in place.
template <class T, int V>
__global__ __launch_bounds__(256) void recurrence_step_kernel(const Recurrence a) {
    const uint32_t per_row = (a.width + V - 1u) / V;
    const uint64_t item = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    if (item >= (uint64_t)a.n_envs * per_row) return;
    const uint32_t env = (uint32_t)(item / per_row), c = ((uint32_t)item - env * per_row) * V;
    const int n = (int)min(a.width - c, (uint32_t)V);
    const T* x = static_cast<const T*>(a.x) + (int64_t)env * a.x_env + c;
    const T* gate = static_cast<const T*>(a.gate) + (int64_t)env * a.gate_env + c;
    T* out = static_cast<T*>(a.out) + (int64_t)env * a.out_env + c;
    float* state = a.state_out + (size_t)env * a.width + c;
    const bool cut = a.resets && a.resets[(int64_t)env * a.resets_env];
    T xs[V], gs[V], y[V];
    float s[V];
    if (n == V) {
        __builtin_memcpy(xs, x, sizeof(xs));
        __builtin_memcpy(gs, gate, sizeof(gs));
        __builtin_memcpy(s, state, sizeof(s));
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            xs[i] = i < n ? x[i] : (T)0.0f;
            gs[i] = i < n ? gate[i] : (T)0.0f;
            s[i] = i < n ? state[i] : 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float g = gate_of<T>((float)gs[i]), b = a.coupled ? taken(g) * (float)xs[i] : (float)xs[i];
        s[i] = cut ? b : kept(g, s[i], b);
        y[i] = (T)s[i];
    }
    if (n == V) {
        __builtin_memcpy(state, s, sizeof(s));
        __builtin_memcpy(out, y, sizeof(y));
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) {
                state[i] = s[i];
                out[i] = y[i];
            }
    }
}

// No steps: the state (or its gradient) passes on.
__global__ __launch_bounds__(256) void recurrence_pass_kernel(const float* from, float* to, uint64_t n) {
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    if (i < n) to[i] = from ? from[i] : 0.0f;
}

struct Shape {
    uint32_t V, C, lanes, rows, strips, waves, segments, seg_steps;
};

// How a call is cut.
Shape shape_of(uint32_t n_envs, uint32_t n_steps, uint32_t width, bool backward) {
    Shape s{};
    s.V = width >= 2u ? 2u : 1u;
    s.C = 16u;
    if (backward && n_steps > kMostWaves * 16u) {
        s.V = 1u;
        s.C = 32u;
    }
    s.lanes = s.C;
    while (s.lanes < 64u && s.lanes * s.V < width) s.lanes *= 2u;
    s.rows = (n_envs + 64u / s.lanes - 1u) / (64u / s.lanes);
    s.strips = (width + s.lanes * s.V - 1u) / (s.lanes * s.V);
    const uint32_t chunks = (n_steps + s.C - 1u) / s.C, blocks = (chunks + kMostWaves - 1u) / kMostWaves;
    if (backward) {
        s.segments = blocks;
        s.waves = (chunks + blocks - 1u) / blocks;
        s.seg_steps = s.waves * s.C;
    } else {
        const uint64_t groups = (uint64_t)s.rows * s.strips;
        const uint32_t cut = (uint32_t)std::min<uint64_t>(blocks, groups >= 1024u ? 1u : (1024u + groups - 1u) / groups);
        const uint32_t each = (blocks + cut - 1u) / cut;  // blocks of a segment
        s.segments = (blocks + each - 1u) / each;
        s.waves = std::min(chunks, kMostWaves);
        s.seg_steps = each * s.waves * s.C;
    }
    s.segments = (n_steps + s.seg_steps - 1u) / s.seg_steps;
    return s;
}

template <class T, int kWhat>
hipError_t launch_part(const Shape& s, const Recurrence& a, hipStream_t st) {
    const dim3 grid(s.rows * s.strips * s.segments), threads(s.waves * 64u);
    constexpr bool kBack = kWhat >= kBackward;
    if (s.V == 2u)
        hipLaunchKernelGGL((recurrence_kernel<T, 2, 16, kWhat>), grid, threads, 0, st, a);
    else if (s.C == 16u)
        hipLaunchKernelGGL((recurrence_kernel<T, 1, 16, kWhat>), grid, threads, 0, st, a);
    else if constexpr (kBack)
        hipLaunchKernelGGL((recurrence_kernel<T, 1, 32, kWhat>), grid, threads, 0, st, a);
    return hipGetLastError();
}

template <class T, bool kBack>
hipError_t launch_all(const Shape& s, const Recurrence& a, hipStream_t st) {
    hipError_t rc = hipSuccess;
    if (s.segments > 1u) {
        rc = launch_part<T, kBack ? kBackwardSums : kForwardSums>(s, a, st);
        if (rc == hipSuccess) {
            const uint64_t cells = (uint64_t)a.n_envs * a.width;
            hipLaunchKernelGGL((recurrence_join_kernel<kBack>), dim3((uint32_t)((cells + 63u) / 64u)), dim3(kJoinWaves * 64u), 0, st, a);
            rc = hipGetLastError();
        }
    }
    return rc == hipSuccess ? launch_part<T, kBack ? kBackward : kForward>(s, a, st) : rc;
}

Recurrence arguments(const pxr_gated_rollout& r, const Shape& s, void* ws) {
    Recurrence a{};
    a.x = r.x.data;
    a.x_env = r.x.env;
    a.x_step = r.x.step;
    a.gate = r.gate.data;
    a.gate_env = r.gate.env;
    a.gate_step = r.gate.step;
    a.resets = r.d_resets;
    a.resets_env = r.resets_env;
    a.resets_step = r.resets_step;
    a.state_in = r.d_state;
    a.joined = static_cast<float*>(ws);
    a.n_envs = r.n_envs;
    a.n_steps = r.n_steps;
    a.width = r.width;
    a.lanes = s.lanes;
    a.strips = s.strips;
    a.segments = s.segments;
    a.seg_steps = s.seg_steps;
    a.coupled = r.coupled;
    return a;
}

int result(hipError_t rc, std::string& err) {
    if (rc == hipSuccess) return PXR_OK;
    err = std::string("kernel launch failed: ") + hipGetErrorString(rc);
    return PXR_ERR_DEVICE;
}

hipError_t pass_on(const float* from, float* to, const pxr_gated_rollout& r, hipStream_t st) {
    if (!to) return hipSuccess;
    const uint64_t n = (uint64_t)r.n_envs * r.width;
    hipLaunchKernelGGL(recurrence_pass_kernel, dim3((uint32_t)((n + 255u) / 256u)), dim3(256), 0, st, from, to, n);
    return hipGetLastError();
}

}  // namespace

size_t gated_recurrence_workspace(uint32_t n_envs, uint32_t n_steps, uint32_t width, bool backward) {
    if (n_steps == 0) return 0;
    const Shape s = shape_of(n_envs, n_steps, width, backward);
    return s.segments > 1u ? (size_t)s.segments * (backward ? 3 : 2) * n_envs * width * sizeof(float) : 0;
}

int launch_gated_recurrence_forward(const pxr_gated_rollout& r, const pxr_steps& out, float* state_out, void* ws, void* stream, std::string& err) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (r.n_steps == 0) return result(pass_on(r.d_state, state_out, r, st), err);
    const Shape s = shape_of(r.n_envs, r.n_steps, r.width, false);
    Recurrence a = arguments(r, s, ws);
    a.out = out.data;
    a.out_env = out.env;
    a.out_step = out.step;
    a.state_out = state_out;
    return result(r.dtype == PXR_F32 ? launch_all<float, false>(s, a, st) : launch_all<__bf16, false>(s, a, st), err);
}

int launch_gated_recurrence_backward(const pxr_gated_rollout& r, const pxr_steps& dout, const float* dstate_out, const pxr_steps& dx,
                                     const pxr_steps& dgate, float* dstate, void* ws, void* stream, std::string& err) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (r.n_steps == 0) return result(pass_on(dstate_out, dstate, r, st), err);
    const Shape s = shape_of(r.n_envs, r.n_steps, r.width, true);
    Recurrence a = arguments(r, s, ws);
    a.dout = dout.data;
    a.dout_env = dout.env;
    a.dout_step = dout.step;
    a.after = dstate_out;
    a.out = dx.data;
    a.out_env = dx.env;
    a.out_step = dx.step;
    a.dgate = dgate.data;
    a.dgate_env = dgate.env;
    a.dgate_step = dgate.step;
    a.dstate = dstate;
    return result(r.dtype == PXR_F32 ? launch_all<float, true>(s, a, st) : launch_all<__bf16, true>(s, a, st), err);
}

int launch_gated_recurrence_step(const pxr_gated_rollout& r, float* state, const pxr_steps& out, void* stream, std::string& err) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    Recurrence a = arguments(r, Shape{}, nullptr);
    a.out = out.data;
    a.out_env = out.env;
    a.state_out = state;
    const uint64_t items = (uint64_t)r.n_envs * ((r.width + 3u) / 4u);
    const dim3 grid((uint32_t)((items + 255u) / 256u));
    if (r.dtype == PXR_F32)
        hipLaunchKernelGGL((recurrence_step_kernel<float, 4>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((recurrence_step_kernel<__bf16, 4>), grid, dim3(256), 0, st, a);
    return result(hipGetLastError(), err);
}

}  // namespace pxr
