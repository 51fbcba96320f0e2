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
// product A of +0 is that of steps among which an episode begins and passes nothing on, whatever the state holds: what is not finite stays on its side of the beginning.
// One that is merely too small for fp32 is -0, which a state that is not finite does pass.
//
// Bound by HBM: 256 environments of 128 steps of 1024 channels of bfloat16 take 44 us, 203 MB at 4.6 TB/s; gradients of 512 x 256 x 1024 314 us, 1.34 GB at 4.3 (79 % of the cycles issue vector
// instructions); a step of 16384 x 1024 43 us, 235 MB at 5.5.  Few long rollouts are cut into segments: the segments' (A, H, R), what comes into each, outputs.  1 x 50000 x 512 take 58 us, of which
// the sums are 23, the join 9.  Gradients of more than 256 steps are cut so whatever their number, and read everything twice: 256 x 512 x 1024 523 us, 512 x 1024 x 256 503, for 267.
// (Two figures beside a rule below compare its two sides at the time when it was made; what a call takes now stands here.)

#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>

#include "pxr_internal.h"

namespace pxr {
namespace {

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

// Of a step that is not there: a gate that keeps everything, zeros.
template <class T, int V>
__device__ __forceinline__ Raw<T, V> absent(bool gate) {
    Raw<T, V> r;
    if constexpr (sizeof(T) == 4)
        r.w[0] = gate ? __builtin_inff() : 0.0f;
    else
        r.w = gate ? (V == 2 ? 0x7F807F80u : 0x7F80u) : 0u;
    return r;
}

// What follows takes a value from its register, whatever is known of it.
__device__ __forceinline__ void as_it_is(uint32_t& v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void as_it_is(float& v) { asm volatile("" : "+v"(v)); }
template <class T, int V>
__device__ __forceinline__ void as_it_is(Raw<T, V>& v) {
    if constexpr (sizeof(T) == 4)
        asm volatile("" : "+v"(v.w[0]));
    else
        asm volatile("" : "+v"(v.w));
}

// A lane's values of a row: the row's address is the same for all lanes, and a lane's place in it a number of 32 bits, so that an address takes no vector registers.
template <class T, int V>
__device__ __forceinline__ Raw<T, V> load(const T* row, uint32_t place) {
    Raw<T, V> r;
    __builtin_memcpy(&r, reinterpret_cast<const char*>(row) + place, sizeof(T) * V);  // (rows may begin at any element: the memory takes requests at any address)
    return r;
}

// Rounded to nearest even, past the caches: nothing here reads them again.
template <class T, int V>
__device__ __forceinline__ void store(T* row, uint32_t place, const float (&f)[V]) {
    typedef T some __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    some v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (T)f[i];
    __builtin_nontemporal_store(v, reinterpret_cast<some*>(reinterpret_cast<char*>(row) + place));
}

// What stands behind this is not begun before it: otherwise inputs of all steps are formed at once, in registers that there are not.
__device__ __forceinline__ void in_turn() { __builtin_amdgcn_sched_barrier(0); }

// A gate as one number: 1 - a where that is the smaller of a and 1 - a, otherwise -a.  Each of the two is 1 less the other where that loses nothing.
template <class T>
__device__ __forceinline__ float gate_of(float g) {
    float m = fabsf(g);
    if (sizeof(T) == 4 && m > 100.0f) m = 100.0f;  // (a NaN stays one)
    const float t = m * -1.44269504f;
    float e = __builtin_amdgcn_exp2f(t);  // exp(-|g|)
    // (what t has lost in 24 bits is |g| of their last one: of 32 bits' results as well)
    if (sizeof(T) == 4) e = __builtin_fmaf(e, __builtin_fmaf(m, -1.44269504f, -t) * 0.69314718f - m * 1.3346e-8f, e);
    return copysignf(e * __builtin_amdgcn_rcpf(1.0f + e), g);
}
__device__ __forceinline__ bool mostly(float s) { return (int)__float_as_uint(s) >= 0; }  // a >= 1/2
__device__ __forceinline__ float taken(float s) { return s + (mostly(s) ? 0.0f : 1.0f); }  // 1 - a
// a v + b.  Where a is all but 1 it is v less a little: a itself, rounded, would be off in the same direction in every step of a gate that stays where it is (200
// steps of gates around 10: a state off by 3e-6, 3e-7 so).
__device__ __forceinline__ float kept(float s, float v, float b) { return __builtin_fmaf(-s, v, (mostly(s) ? v : 0.0f) + b); }
__device__ __forceinline__ float kept(float s, float v) { return __builtin_fmaf(-s, v, mostly(s) ? v : 0.0f); }

// Products of steps in a row (+0: an episode begins among them; -0: too small), and what such steps (product A, own result H) make of a state.
__device__ __forceinline__ bool begins(float A) { return __float_as_uint(A) == 0u; }
__device__ __forceinline__ float too_small(float A) { return A == 0.0f ? -0.0f : A; }
__device__ __forceinline__ float times(float A, float B) { return begins(A) || begins(B) ? 0.0f : too_small(A * B); }
__device__ __forceinline__ float through(float A, float H, float state) { return begins(A) ? H : __builtin_fmaf(A, state, H); }

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
// Steps of a wavefront: as many as its registers have room for (8: 256 x 128 x 1024 50 us, 46 so; gradients of 512 x 256 x 1024, then in two segments, 625, 313), and few for rollouts that are shorter
// than kFewSteps (16000 x 4 x 256: 16 of them 52 us, 4 of them 24; 16000 x 8 x 256 62 and 44, gradients 87 and 69; of 16 steps 75 and 87).
constexpr int kSteps = 16, kStepsOfFew = 4;
constexpr uint32_t kFewSteps = 8;
constexpr uint32_t kMostWaves = 16;    // of a workgroup

// Where a lane's channels are: of environment `env`, from channel `at` on.  A row that ends inside a vector has its last vector moved back to its end: the values that
// it shares with the vector before it are computed in both lanes, by the same operations, and written by both, the same bits.  Lanes behind the row's end, and
// those of environments that are not there (`any` is false), take the last one's and write nothing.
template <class T, int V>
struct Lane {
    uint32_t env0, env, at;
    bool any;
    __device__ __forceinline__ Lane(const Recurrence& a, uint32_t rows, uint32_t strip) {
        const uint32_t lane = threadIdx.x & 63u, in_row = lane & (a.lanes - 1u);
        env0 = rows * (64u / a.lanes);
        const uint32_t e = env0 + lane / a.lanes, c = (strip * a.lanes + in_row) * V;
        env = min(e, a.n_envs - 1u);
        at = min(c, a.width - V);
        any = e < a.n_envs && c < a.width;
    }
    // In bytes from the first environment's row.  (The launch sees to it that these fit 32 bits.)
    __device__ __forceinline__ uint32_t place(int64_t env_stride) const { return ((env - env0) * (uint32_t)env_stride + at) * (uint32_t)sizeof(T); }
};

// A value, or 0 where a mask says so, whatever the value is.
__device__ __forceinline__ float masked(float v, uint32_t m) { return __uint_as_float(__float_as_uint(v) & m); }

// A wavefront's steps, C of V channels a lane.  `cuts`: a bit for each step that begins an episode.  Steps that are not there keep everything and add nothing (absent()).
template <class T, int V, int kWhat, bool kCoupled, int C>
struct Chunk {
    static constexpr bool kBack = kWhat >= kBackward;
    typedef Raw<T, V> Raws[C];

    // All bits where step j goes on with what was before it.
    static __device__ __forceinline__ uint32_t goes_on(uint32_t cuts, int j) { return (cuts >> j & 1u) - 1u; }
    static __device__ __forceinline__ float input(float s, float x) { return kCoupled ? taken(s) * x : x; }

    // By themselves: product, result from zero, and what they hand back of zero.  h, s: forward, the results and the products up to them; backward, the gates in s.
    static __device__ __forceinline__ void alone(const Raws& xs, const Raws& gs, const Raw<T, V>* ds, uint32_t cuts, float (&A)[V], float (&H)[V], float (&R)[V], float (&h)[C][V], float (&s)[C][V]) {
        uint32_t none = ~0u;  // that has begun an episode so far: products stay 0 after one that has, over gates that are no numbers
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const uint32_t on = goes_on(cuts, j);
            none &= on;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                // (where inputs are taken as they are, a step that begins an episode has no use for its gate, whatever that is)
                const float gate = gate_of<T>(gs[j].get(i)), g = kCoupled ? gate : masked(gate, on);
                A[i] = masked(kept(g, A[i]), none);
                H[i] = kept(g, masked(H[i], on), input(g, xs[j].get(i)));
                if (kWhat == kForward) h[j][i] = H[i];
                s[j][i] = kBack ? g : A[i];
            }
            in_turn();
        }
#pragma unroll
        for (int i = 0; i < V; ++i) A[i] = masked(too_small(A[i]), none);
        if constexpr (kBack) {
#pragma unroll
            for (int j = C - 1; j >= 0; --j)
#pragma unroll
                for (int i = 0; i < V; ++i) R[i] = masked(kept(s[j][i], ds[j].get(i) + R[i]), goes_on(cuts, j));
        }
    }

    static __device__ __forceinline__ void outputs(const float (&h)[C][V], const float (&s)[C][V], int n, uint32_t cuts, const float (&state)[V], T* out, int64_t step, uint32_t place) {
        uint32_t none = ~0u;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            none &= goes_on(cuts, j);
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = __builtin_fmaf(s[j][i], masked(state[i], none), h[j][i]);
            if (j < n) store<T, V>(out, place, y);
            out += step;
        }
    }

    // dx, dgate: of the last of the C steps.
    static __device__ __forceinline__ void gradients(Raws& xs, const Raw<T, V>* ds, float (&s)[C][V], int n, uint32_t cuts, float (&state)[V], float (&later)[V], T* dx, int64_t dx_step,
                                                     uint32_t dx_place, T* dgate, int64_t dgate_step, uint32_t dgate_place) {
        float h[C][V];  // what a step sees of the state
#pragma unroll
        for (int j = 0; j < C; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                h[j][i] = masked(state[i], goes_on(cuts, j));
                state[i] = kept(s[j][i], h[j][i], input(s[j][i], xs[j].get(i)));
                as_it_is(s[j][i]);  // (what it was made into, here and in front of the barrier, is made again below: there are no registers to keep it in)
            }
            as_it_is(xs[j]);
            in_turn();
        }
#pragma unroll
        for (int j = C - 1; j >= 0; --j) {
            float to_x[V], to_gate[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float take = taken(s[j][i]), L = ds[j].get(i) + later[i], kept_L = kept(s[j][i], L);
                to_x[i] = kCoupled ? take * L : L;
                to_gate[i] = take * kept_L * (kCoupled ? h[j][i] - xs[j].get(i) : h[j][i]);
                later[i] = masked(kept_L, goes_on(cuts, j));
            }
            if (j < n) {
                store<T, V>(dx, dx_place, to_x);
                store<T, V>(dgate, dgate_place, to_gate);
            }
            dx -= dx_step;
            dgate -= dgate_step;
            in_turn();
        }
    }
};

// One workgroup: seg_steps steps (backward: at most what its wavefronts hold) of a strip of channels of 64 / lanes environments.
template <class T, int V, int kWhat, bool kCoupled, int C>
__global__ __launch_bounds__(kMostWaves * 64) void recurrence_kernel(const Recurrence a) {
    constexpr bool kBack = kWhat >= kBackward, kSums = kWhat == kForwardSums || kWhat == kBackwardSums;
    constexpr int kPlanes = kBack ? 3 : 2;
    typedef Chunk<T, V, kWhat, kCoupled, C> Steps;
    typedef float Told[kPlanes][V][64];
    extern __shared__ float recurrence_memory[];  // of as many wavefronts as there are, twice where there are several blocks
    Told* const shared = reinterpret_cast<Told*>(recurrence_memory);
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const uint32_t strip = blockIdx.x % a.strips, rest = blockIdx.x / a.strips, seg = rest % a.segments, rows = rest / a.segments;
    const Lane<T, V> at(a, rows, strip);
    const T* x = static_cast<const T*>(a.x) + (int64_t)at.env0 * a.x_env;
    const T* gate = static_cast<const T*>(a.gate) + (int64_t)at.env0 * a.gate_env;
    const T* dout = kBack ? static_cast<const T*>(a.dout) + (int64_t)at.env0 * a.dout_env : nullptr;
    const uint32_t places[3] = {at.place(a.x_env), at.place(a.gate_env), at.place(a.dout_env)};
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
    float product[V];  // over the segment (sums)
#pragma unroll
    for (int i = 0; i < V; ++i) product[i] = 1.0f;

    uint32_t turn = 0, block = begin;
    do {  // (backward: once)
        uint32_t x_place = places[0], gate_place = places[1], dout_place = places[2];
        as_it_is(x_place);  // (otherwise an address of the whole, in vector registers, outside of the loop)
        as_it_is(gate_place);
        as_it_is(dout_place);
        const uint32_t first = block + wave * C;
        const int n = first < end ? (int)min(end - first, (uint32_t)C) : 0;  // this wavefront's steps
        Raw<T, V> xs[C], gs[C], ds[kBack ? C : 1];
        uint32_t cuts = 0;
        if (n) {
            // (steps past the last one are the last one again)
            const T *g = gate + (int64_t)first * a.gate_step, *v = x + (int64_t)first * a.x_step, *d = kBack ? dout + (int64_t)first * a.dout_step : nullptr;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                gs[j] = load<T, V>(g, gate_place);
                xs[j] = load<T, V>(v, x_place);
                if (kBack) ds[j] = load<T, V>(d, dout_place);
                g += j + 1 < n ? a.gate_step : 0;
                v += j + 1 < n ? a.x_step : 0;
                if (kBack) d += j + 1 < n ? a.dout_step : 0;
            }
            if (n < C)
#pragma unroll
                for (int j = 1; j < C; ++j)
                    if (j >= n) {
                        gs[j] = absent<T, V>(true);
                        xs[j] = absent<T, V>(false);
                        if (kBack) ds[j] = absent<T, V>(false);
                    }
            if (a.resets) {  // the first C of an environment's lanes ask for one of its steps each
                const uint32_t in_row = lane & (a.lanes - 1u);
                const bool mark = in_row < (uint32_t)n && a.resets[(int64_t)at.env * a.resets_env + (int64_t)(first + in_row) * a.resets_step];
                cuts = (uint32_t)(__ballot(mark) >> (lane - in_row)) & ((1u << C) - 1u);
            }
        }
        // each wavefront's steps by themselves
        float A[V], H[V], R[V], h[C][V], s[C][V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            A[i] = 1.0f;
            H[i] = R[i] = 0.0f;
        }
        if (n) Steps::alone(xs, gs, ds, cuts, A, H, R, h, s);
        if (kWhat == kBackward)
#pragma unroll
            for (int j = 0; j < C; ++j) {
                as_it_is(xs[j]);
                as_it_is(ds[j]);
#pragma unroll
                for (int i = 0; i < V; ++i) as_it_is(s[j][i]);
            }
        Told* const told = shared + (kBack ? 0u : turn * waves);  // (the block after the next one writes here again)
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
                if (kSums) product[i] = times(product[i], p);
            }
            if constexpr (kBack) {
                for (uint32_t w = waves; w-- > 0;) {
                    if (w == wave) mine_later[i] = later[i];
                    later[i] = through(told[w][0][i][lane], told[w][2][i][lane], later[i]);
                }
            }
        }
        if (kSums || !n || !at.any) continue;
        if constexpr (kWhat == kForward) {
            T* out = static_cast<T*>(a.out) + ((int64_t)at.env0 * a.out_env + (int64_t)first * a.out_step);
            uint32_t place = at.place(a.out_env);
            as_it_is(place);
            Steps::outputs(h, s, n, cuts, mine, out, a.out_step, place);
        } else if constexpr (kWhat == kBackward) {
            T* dx = static_cast<T*>(a.out) + ((int64_t)at.env0 * a.out_env + (int64_t)(first + C - 1) * a.out_step);
            T* dgate = static_cast<T*>(a.dgate) + ((int64_t)at.env0 * a.dgate_env + (int64_t)(first + C - 1) * a.dgate_step);
            uint32_t dx_place = at.place(a.out_env), dgate_place = at.place(a.dgate_env);
            as_it_is(dx_place);
            as_it_is(dgate_place);
            Steps::gradients(xs, ds, s, n, cuts, mine, mine_later, dx, a.out_step, dx_place, dgate, a.dgate_step, dgate_place);
        }
    } while (!kBack && (turn ^= 1u, block += waves * C) < end);
    if (wave == 0 && at.any) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (kSums) {
                float* plane = a.joined + (size_t)seg * kPlanes * cells + cell + i;
                plane[0] = product[i];
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

// A workgroup takes 4.7 us for a block of its steps, one after the other, and 128 of them side by side as many bytes a second as segments do, which read everything twice: forward passes are cut into
// segments only below that many, and from the number of blocks on that takes longer than three launches.  (100 x 600 x 1024, 800 groups: in two segments 157 us, whole 98; 24 x 1000 x 1024, 192: 57,
// 51; 64 x 1000 x 128, 64 groups of 8 blocks: 26, 41; of 3 blocks 20, 17.)
constexpr uint32_t kFewBlocks = 4, kFewGroups = 128;
// Workgroups of a forward pass have half of the wavefronts that they may have, unless there is at most one for a compute unit (200 x 1000 x 128: 8 wavefronts 52 us, 16 45; 300 x 1000 x 128: 72, 82;
// segments of 1 x 50000 x 512: 61, 78).
constexpr uint32_t kHalfWaves = kMostWaves / 2, kUnits = 256;
constexpr uint32_t kManyGroups = 2048;  // that segments make (1 x 50000 x 512: 1024 of them 67 us, 2048 62)

// How a call is cut (lanes, rows, strips: by its strides as well, in narrowed()).
Shape shape_of(uint32_t V, uint32_t n_envs, uint32_t n_steps, uint32_t width, bool backward) {
    Shape s{};
    s.V = V;
    s.C = n_steps <= kFewSteps ? kStepsOfFew : kSteps;
    s.lanes = s.C;
    while (s.lanes < 64u && s.lanes * s.V < width) s.lanes *= 2u;
    s.rows = (n_envs + 64u / s.lanes - 1u) / (64u / s.lanes);
    s.strips = (width + s.lanes * s.V - 1u) / (s.lanes * s.V);
    const uint32_t chunks = (n_steps + s.C - 1u) / s.C;
    const auto blocks_of = [&](uint32_t waves) { return (chunks + waves - 1u) / waves; };
    const uint64_t groups = (uint64_t)n_envs * ((width + 127u) / 128u);  // (by the sizes alone, like the workspace)
    if (backward || blocks_of(kHalfWaves) <= kFewBlocks || groups >= kFewGroups) {
        const uint32_t blocks = blocks_of(backward || (uint64_t)s.rows * s.strips <= kUnits ? kMostWaves : kHalfWaves);
        s.waves = (chunks + blocks - 1u) / blocks;
        s.seg_steps = (backward ? 1u : blocks) * s.waves * s.C;
    } else {
        const uint32_t blocks = blocks_of(kHalfWaves), cut = (uint32_t)std::min<uint64_t>(blocks, (kManyGroups + groups - 1u) / groups);
        s.waves = kHalfWaves;
        s.seg_steps = (blocks + cut - 1u) / cut * s.waves * s.C;
    }
    s.segments = (n_steps + s.seg_steps - 1u) / s.seg_steps;
    return s;
}

// Values of a lane: 4 bytes of them.  (Of bfloat16 one: 256 x 128 x 1024 55 us, 46 so; gradients of 512 x 256 x 1024 348, 316.)
uint32_t values_of(const pxr_gated_rollout& r) { return r.dtype == PXR_BF16 && r.width >= 2u ? 2u : 1u; }

// Environments that share a wavefront are numbers of 32 bits apart, in bytes; where they lie further, or backwards, each has one to itself.
Shape narrowed(Shape s, uint32_t n_envs, uint32_t width, std::initializer_list<int64_t> env_strides) {
    for (const int64_t e : env_strides)
        if (s.lanes < 64u && (e < 0 || e > (1ll << 26))) {
            s.lanes = 64u;
            s.rows = n_envs;
            s.strips = (width + 64u * s.V - 1u) / (64u * s.V);
        }
    return s;
}

template <class T, int kWhat, int C>
hipError_t launch_part(const Shape& s, const Recurrence& a, hipStream_t st) {
    const dim3 grid(s.rows * s.strips * s.segments), threads(s.waves * 64u);
    constexpr bool kBack = kWhat >= kBackward;
    const uint32_t lds = (!kBack && s.seg_steps > s.waves * C ? 2u : 1u) * s.waves * (kBack ? 3u : 2u) * s.V * 64u * (uint32_t)sizeof(float);
    if (sizeof(T) == 2 && s.V == 2u) {
        constexpr int V = sizeof(T) == 2 ? 2 : 1;
        if (a.coupled)
            hipLaunchKernelGGL((recurrence_kernel<T, V, kWhat, true, C>), grid, threads, lds, st, a);
        else
            hipLaunchKernelGGL((recurrence_kernel<T, V, kWhat, false, C>), grid, threads, lds, st, a);
    } else {
        if (a.coupled)
            hipLaunchKernelGGL((recurrence_kernel<T, 1, kWhat, true, C>), grid, threads, lds, st, a);
        else
            hipLaunchKernelGGL((recurrence_kernel<T, 1, kWhat, false, C>), grid, threads, lds, st, a);
    }
    return hipGetLastError();
}

template <class T, bool kBack>
hipError_t launch_all(const Shape& s, const Recurrence& a, hipStream_t st) {
    if (s.C == kStepsOfFew) return launch_part<T, kBack ? kBackward : kForward, kStepsOfFew>(s, a, st);  // (one segment)
    hipError_t rc = hipSuccess;
    if (s.segments > 1u) {
        rc = launch_part<T, kBack ? kBackwardSums : kForwardSums, kSteps>(s, a, st);
        if (rc == hipSuccess) {
            const uint64_t cells = (uint64_t)a.n_envs * a.width;
            hipLaunchKernelGGL((recurrence_join_kernel<kBack>), dim3((uint32_t)((cells + 63u) / 64u)), dim3(kJoinWaves * 64u), 0, st, a);
            rc = hipGetLastError();
        }
    }
    return rc == hipSuccess ? launch_part<T, kBack ? kBackward : kForward, kSteps>(s, a, st) : rc;
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
    const Shape s = shape_of(1, n_envs, n_steps, width, backward);
    return s.segments > 1u ? (size_t)s.segments * (backward ? 3 : 2) * n_envs * width * sizeof(float) : 0;
}

int launch_gated_recurrence_forward(const pxr_gated_rollout& r, const pxr_steps& out, float* state_out, void* ws, void* stream, std::string& err) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (r.n_steps == 0) return result(pass_on(r.d_state, state_out, r, st), err);
    const Shape s = narrowed(shape_of(values_of(r), r.n_envs, r.n_steps, r.width, false), r.n_envs, r.width, {r.x.env, r.gate.env, out.env});
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
    const Shape s = narrowed(shape_of(values_of(r), r.n_envs, r.n_steps, r.width, true), r.n_envs, r.width, {r.x.env, r.gate.env, dout.env, dx.env, dgate.env});
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
