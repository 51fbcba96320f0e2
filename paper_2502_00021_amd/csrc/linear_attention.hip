// Linear attention with a decay for each head (pxr_linear_attention_* in include/pxr.h).  gfx950 only.
//
//   S_t = (t begins an episode ? 0 : g S_{t-1}) + k_t v_t^T,   o_t = scale S_t^T q_t,   g = exp(log_decay_h)
//
// Every pass over a rollout is one form, a scan: out_i = out_scale sum_{j <= i} g^(i-j) key_scale (x_i . y_j) z_j + what the
// state before the scan adds.  The forward pass is the scan of (q, k, v).  With do the gradient of the outputs,
//   dq is the scan of (do, v, k): dq_t = scale S_t do_t, and the states are the forward pass' transposed;
//   dk and dv are scans from the last step to the first, of (v, do, q) and of (k, q, do): their state
//     R_t = scale q_t do_t^T + (t + 1 begins an episode ? 0 : g R_{t+1}) gives dk_t = R_t v_t, dv_t = R_t^T k_t.

#include <hip/hip_runtime.h>

#include "pxr_internal.h"

namespace pxr {
namespace {

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __bf16* p) { return (float)*p; }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__bf16* p, float v) { *p = (__bf16)v; }  // round to nearest even

// One scan: x, y [.., a], z [.., b] -> out [.., b]; state [a][b] per (environment, head), with strides of its own.
struct Scan {
    pxr_tokens x, y, z, out;
    uint32_t a, b;
    const float* state_in;  // null = zeros
    float* state_out;       // null = not wanted
    uint32_t state_row, state_col;
    float out_scale, key_scale;
    uint32_t reverse;
};

template <class T>
__device__ __forceinline__ T* head_of(const pxr_tokens& t, uint32_t e, uint32_t h) {
    return static_cast<T*>(t.data) + ((int64_t)e * t.env + (int64_t)h * t.head);
}

// One lane per column of the state, which lies in LDS; one step after the other.
template <class T>
__global__ __launch_bounds__(64) void scan_kernel(const Scan s, const LinearAttentionHead* heads, uint32_t n_heads, uint32_t n_steps,
                                                  const uint8_t* resets, int64_t resets_env, int64_t resets_step) {
    extern __shared__ float state[];  // [a][64]
    const uint32_t e = blockIdx.x / n_heads, h = blockIdx.x - e * n_heads, lane = threadIdx.x, col = blockIdx.y * 64u + lane;
    const bool on = col < s.b;
    const float decay = heads[h].decay, decay_rest = heads[h].decay_rest;
    const size_t base = (size_t)blockIdx.x * s.a * s.b;
    for (uint32_t d = 0; d < s.a; ++d)
        state[d * 64u + lane] = on && s.state_in ? s.state_in[base + (size_t)d * s.state_row + (size_t)col * s.state_col] : 0.0f;
    const T *x = head_of<const T>(s.x, e, h), *y = head_of<const T>(s.y, e, h), *z = head_of<const T>(s.z, e, h);
    T* out = head_of<T>(s.out, e, h);
    for (uint32_t k = 0; k < n_steps; ++k) {
        const int64_t t = s.reverse ? n_steps - 1u - k : k;
        // forward: the state decays before a step is added, and not at all into a step that begins an episode; in reverse it
        // decays after, on its way to the step before
        const bool cut = resets && resets[e * resets_env + t * resets_step];
        const float zc = on ? load1(z + t * s.z.step + col) * s.key_scale : 0.0f;
        float sum = 0.0f;
        for (uint32_t d = 0; d < s.a; ++d) {
            float v = state[d * 64u + lane];
            if (!s.reverse) v = cut ? 0.0f : __builtin_fmaf(v, decay, v * decay_rest);
            v = __builtin_fmaf(load1(y + t * s.y.step + d), zc, v);
            sum = __builtin_fmaf(load1(x + t * s.x.step + d), v, sum);
            if (s.reverse) v = cut ? 0.0f : __builtin_fmaf(v, decay, v * decay_rest);
            state[d * 64u + lane] = v;
        }
        if (on) store1(out + t * s.out.step + col, sum * s.out_scale);
    }
    if (on && s.state_out)
        for (uint32_t d = 0; d < s.a; ++d) s.state_out[base + (size_t)d * s.state_row + (size_t)col * s.state_col] = state[d * 64u + lane];
}

// One step of every environment: four wavefronts per (environment, head) and 64 columns, rows dealt to the wavefronts.
template <class T>
__global__ __launch_bounds__(256) void step_kernel(pxr_tokens q, pxr_tokens k, pxr_tokens v, pxr_tokens out, uint32_t dk, uint32_t dv,
                                                   float scale, const LinearAttentionHead* heads, uint32_t n_heads, const uint8_t* resets,
                                                   int64_t resets_env, float* state) {
    __shared__ float part[4][64];
    const uint32_t e = blockIdx.x / n_heads, h = blockIdx.x - e * n_heads, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t col = blockIdx.y * 64u + lane;
    const bool on = col < dv, cut = resets && resets[e * resets_env];
    const float decay = heads[h].decay, decay_rest = heads[h].decay_rest;
    const T *qh = head_of<const T>(q, e, h), *kh = head_of<const T>(k, e, h);
    const float vc = on ? load1(head_of<const T>(v, e, h) + col) : 0.0f;
    float sum = 0.0f;
    if (on)
        for (uint32_t d = wave; d < dk; d += 4) {
            float* p = state + ((size_t)blockIdx.x * dk + d) * dv + col;
            float s = cut ? 0.0f : *p;
            s = __builtin_fmaf(s, decay, s * decay_rest);
            s = __builtin_fmaf(load1(kh + d), vc, s);
            *p = s;
            sum = __builtin_fmaf(load1(qh + d), s, sum);
        }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && on)
        store1(head_of<T>(out, e, h) + col, ((part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane])) * scale);
}

int launched(std::string& err) {
    const hipError_t rc = hipGetLastError();
    if (rc == hipSuccess) return PXR_OK;
    err = std::string("kernel launch failed: ") + hipGetErrorString(rc);
    return PXR_ERR_DEVICE;
}

void enqueue(const LinearAttentionConsts& c, const pxr_rollout& r, const Scan& s, hipStream_t st) {
    const dim3 grid(r.n_envs * c.n_heads, (s.b + 63u) / 64u);
    const size_t lds = (size_t)s.a * 64u * 4u;
    if (r.dtype == PXR_F32)
        hipLaunchKernelGGL((scan_kernel<float>), grid, dim3(64), lds, st, s, c.heads, c.n_heads, r.n_steps, r.d_resets, r.resets_env, r.resets_step);
    else
        hipLaunchKernelGGL((scan_kernel<__bf16>), grid, dim3(64), lds, st, s, c.heads, c.n_heads, r.n_steps, r.d_resets, r.resets_env, r.resets_step);
}

}  // namespace

size_t linear_attention_workspace(const LinearAttentionConsts&, uint32_t, uint32_t, uint32_t, bool) { return 0; }

int launch_linear_attention_forward(const LinearAttentionConsts& c, const pxr_rollout& r, const pxr_tokens& out, float* state_out, void*,
                                    void* stream, std::string& err) {
    enqueue(c, r, Scan{r.q, r.k, r.v, out, c.dk, c.dv, r.d_state, state_out, c.dv, 1u, c.scale, 1.0f, 0u}, reinterpret_cast<hipStream_t>(stream));
    return launched(err);
}

int launch_linear_attention_backward(const LinearAttentionConsts& c, const pxr_rollout& r, const pxr_tokens& dout, const float* dstate_out,
                                     const pxr_tokens& dq, const pxr_tokens& dk, const pxr_tokens& dv, float* dstate, void*,
                                     void* stream, std::string& err) {
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    enqueue(c, r, Scan{dout, r.v, r.k, dq, c.dv, c.dk, r.d_state, nullptr, 1u, c.dv, c.scale, 1.0f, 0u}, st);
    enqueue(c, r, Scan{r.v, dout, r.q, dk, c.dv, c.dk, dstate_out, nullptr, 1u, c.dv, 1.0f, c.scale, 1u}, st);
    enqueue(c, r, Scan{r.k, r.q, dout, dv, c.dk, c.dv, dstate_out, dstate, c.dv, 1u, 1.0f, c.scale, 1u}, st);
    return launched(err);
}

int launch_linear_attention_step(const LinearAttentionConsts& c, const pxr_rollout& r, float* state, const pxr_tokens& out, void* stream,
                                 std::string& err) {
    const dim3 grid(r.n_envs * c.n_heads, (c.dv + 63u) / 64u);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (r.dtype == PXR_F32)
        hipLaunchKernelGGL((step_kernel<float>), grid, dim3(256), 0, st, r.q, r.k, r.v, out, c.dk, c.dv, c.scale, c.heads, c.n_heads, r.d_resets, r.resets_env, state);
    else
        hipLaunchKernelGGL((step_kernel<__bf16>), grid, dim3(256), 0, st, r.q, r.k, r.v, out, c.dk, c.dv, c.scale, c.heads, c.n_heads, r.d_resets, r.resets_env, state);
    return launched(err);
}

}  // namespace pxr
