// C ABI of a policy's memory (pxr_layer_norm_*, pxr_linear_attention_*, pxr_gated_recurrence_*, pxr_head_norm_* in include/pxr.h):
// validation, the layers' constants, launch.

#include <hip/hip_runtime.h>

#include <cmath>
#include <initializer_list>
#include <new>

#include "pxr_internal.h"
#include "views.h"

struct pxr_linear_attention {
    pxr::LinearAttentionConsts c{};
};

struct pxr_head_norm {
    pxr::HeadNormConsts c{};
};

namespace {

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
size_t element(uint32_t dtype) { return dtype == PXR_F32 ? 4u : 2u; }

// What all three calls ask of a description; empty = nothing is wrong.
const char* wrong_norm(const pxr_layer_norm_desc* d, bool backward) {
    if (!d) return "null argument";
    if (d->dtype > PXR_BF16 || (d->param_dtype != PXR_F32 && d->param_dtype != d->dtype)) return "dtype must be fp32 or bfloat16, param_dtype fp32 or dtype";
    if (d->width == 0 || d->width > (1u << 30)) return "width must lie in [1, 2^30]";
    if (d->n_rows > 0x7FFFFFFFull) return "n_rows must be below 2^31";
    if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return "eps must be finite and not negative";
    if (d->n_rows > 1 && (d->x_stride < (int64_t)d->width || d->y_stride < (int64_t)d->width || (backward && d->dx_stride < (int64_t)d->width)))
        return "a row stride is smaller than the width";
    return nullptr;
}

// A rollout's own arguments.
const char* wrong_rollout(const pxr_linear_attention* a, const pxr_rollout* r, bool step) {
    if (!a || !r) return "null argument";
    if (r->dtype > PXR_BF16) return "dtype must be fp32 or bfloat16";
    // (a launch counts its threads in 32 bits: 2^21 rows are 3 gradients x 2 tiles x 256 threads of them)
    if (r->n_envs == 0 || (uint64_t)r->n_envs * a->c.n_heads > (1u << 21)) return "n_envs must be positive and n_envs * n_heads at most 2^21";
    if (r->n_steps > 0x7FFFFFFFu) return "n_steps must be below 2^31";
    if (step && r->n_steps != 1) return "n_steps must be 1";
    if (!aligned(r->d_state, 4)) return "the state must be 4-byte aligned";
    return nullptr;
}

bool wrong_view(const pxr_tokens* t, uint32_t dtype, uint32_t n_steps) { return !t || (n_steps && !t->data) || !aligned(t->data, element(dtype)); }

bool overlap(const float* a, const float* b, size_t n) { return a && b && a < b + n && b < a + n; }

// Sizes of a gated recurrence.
const char* wrong_gated_sizes(uint32_t n_envs, uint32_t n_steps, uint32_t width) {
    if (n_envs == 0 || width == 0) return "n_envs and width must be positive";
    if (n_steps > 0x7FFFFFFFu) return "n_steps must be below 2^31";
    // (a launch counts its threads in 32 bits, and the parts of a rollout are at least this large; the factors are checked one by one, none of the products wraps)
    const uint64_t wide = (uint64_t)n_envs * ((width + 63ull) / 64ull), parts = (n_steps + 127ull) / 128ull;
    if (wide > (1ull << 22) || wide * (parts ? parts : 1u) > (1ull << 22)) return "n_envs * ceil(width / 64) * ceil(n_steps / 128) must be at most 2^22";
    return nullptr;
}

const char* wrong_gated(const pxr_gated_rollout* r, bool step) {
    if (!r) return "null argument";
    if (r->dtype > PXR_BF16) return "dtype must be fp32 or bfloat16";
    if (r->coupled > 1u) return "coupled must be 0 or 1";
    if (const char* why = wrong_gated_sizes(r->n_envs, r->n_steps, r->width)) return why;
    if (step && r->n_steps != 1) return "n_steps must be 1";
    if (!aligned(r->d_state, 4)) return "the state must be 4-byte aligned";
    return nullptr;
}

bool wrong_view(const pxr_steps* t, uint32_t dtype, uint32_t n_steps) { return !t || (n_steps && !t->data) || !aligned(t->data, element(dtype)); }

pxr::View view(const pxr_steps& t, const pxr_gated_rollout& r) {
    return {t.data, element(r.dtype), r.width, {{r.n_envs, t.env}, {r.n_steps, t.step}, {1, 0}}};
}

// Everything but the buffers.
const char* wrong_heads(const pxr_head_norm* n, const pxr_heads* r) {
    if (!n || !r) return "null argument";
    if (r->dtype > PXR_BF16 || (r->param_dtype != PXR_F32 && r->param_dtype != r->dtype)) return "dtype must be fp32 or bfloat16, param_dtype fp32 or dtype";
    if (r->position_bits != 32u && r->position_bits != 64u) return "position_bits must be 32 or 64";
    if ((uint64_t)r->n_envs * r->n_steps > 0x7FFFFFFFull) return "n_envs * n_steps must be below 2^31";
    if (r->n_heads > 65535u || r->n_key_heads > 65535u) return "n_heads and n_key_heads must be at most 65535";
    return nullptr;
}

// The buffers that all passes read, and views of the queries' and of the keys' layout.
bool wrong_head_buffers(const pxr_heads* r, std::initializer_list<const pxr_tokens*> of_q, std::initializer_list<const pxr_tokens*> of_k) {
    const uint32_t tokens = r->n_envs && r->n_steps;
    if (r->n_heads)
        for (const pxr_tokens* t : of_q)
            if (wrong_view(t, r->dtype, tokens)) return true;
    if (r->n_key_heads)
        for (const pxr_tokens* t : of_k)
            if (wrong_view(t, r->dtype, tokens)) return true;
    const size_t p = element(r->param_dtype);
    return !aligned(r->d_q_weight, p) || !aligned(r->d_k_weight, p) || !aligned(r->d_positions, r->position_bits / 8u);
}

// Whether heads that are written, of queries and of keys, lie where others are read or written: each may be in the place of what the same heads are read from (`own`), itself.
bool heads_overlap(const pxr_heads* r, uint32_t d, const pxr_tokens* q_to, const pxr_tokens* k_to, std::initializer_list<const pxr_tokens*> of_q, std::initializer_list<const pxr_tokens*> of_k) {
    const auto view = [&](const pxr_tokens* t, uint32_t heads) { return pxr::View{t->data, element(r->dtype), d, {{r->n_envs, t->env}, {r->n_steps, t->step}, {heads, t->head}}}; };
    const auto overlaps = [&](const pxr_tokens* to, uint32_t heads, std::initializer_list<const pxr_tokens*> own, uint32_t others, std::initializer_list<const pxr_tokens*> other) {
        if (!heads) return false;
        const pxr::View v = view(to, heads);
        for (const pxr_tokens* t : own)
            if (!pxr::itself(v, view(t, heads)) && pxr::share(v, view(t, heads))) return true;
        if (others)
            for (const pxr_tokens* t : other)
                if (pxr::share(v, view(t, others))) return true;
        return false;
    };
    return overlaps(q_to, r->n_heads, of_q, r->n_key_heads, of_k) || overlaps(k_to, r->n_key_heads, of_k, r->n_heads, of_q) ||
           (r->n_heads && r->n_key_heads && pxr::share(view(q_to, r->n_heads), view(k_to, r->n_key_heads)));
}

int finish(int rc, const char* call, const std::string& err) {
    return rc == PXR_OK ? PXR_OK : pxr::set_error(rc, std::string(call) + ": " + err);
}

int refuse(const char* call, const char* why) { return pxr::set_error(PXR_ERR_INVALID_ARG, std::string(call) + ": " + why); }

}  // namespace

extern "C" {

int pxr_layer_norm_forward(const pxr_layer_norm_desc* d, const void* d_x, const void* d_weight, const void* d_bias, void* d_y, float* d_mean,
                           float* d_rstd, void* hip_stream) {
    if (const char* why = wrong_norm(d, false)) return refuse("pxr_layer_norm_forward", why);
    if (d->n_rows == 0) return PXR_OK;
    if (!d_x || !d_y) return refuse("pxr_layer_norm_forward", "null argument");
    const size_t n = element(d->dtype), p = element(d->param_dtype);
    if (!aligned(d_x, n) || !aligned(d_y, n) || !aligned(d_weight, p) || !aligned(d_bias, p) || !aligned(d_mean, 4) || !aligned(d_rstd, 4))
        return refuse("pxr_layer_norm_forward", "a buffer is not aligned to its elements");
    std::string err;
    return finish(pxr::launch_layer_norm_forward(*d, d_x, d_weight, d_bias, d_y, d_mean, d_rstd, hip_stream, err), "pxr_layer_norm_forward", err);
}

int pxr_layer_norm_workspace(const pxr_layer_norm_desc* d, size_t* bytes) {
    if (const char* why = wrong_norm(d, true)) return refuse("pxr_layer_norm_workspace", why);
    if (!bytes) return refuse("pxr_layer_norm_workspace", "null argument");
    *bytes = pxr::layer_norm_workspace(*d);
    return PXR_OK;
}

int pxr_layer_norm_backward(const pxr_layer_norm_desc* d, const void* d_dy, const void* d_x, const float* d_mean, const float* d_rstd,
                            const void* d_weight, void* d_dx, void* d_dweight, void* d_dbias, void* d_workspace, size_t workspace_bytes,
                            void* hip_stream) {
    if (const char* why = wrong_norm(d, true)) return refuse("pxr_layer_norm_backward", why);
    if (d->n_rows && (!d_dy || !d_x || !d_mean || !d_rstd || !d_dx)) return refuse("pxr_layer_norm_backward", "null argument");
    const size_t n = element(d->dtype), p = element(d->param_dtype);
    if (!aligned(d_dy, n) || !aligned(d_x, n) || !aligned(d_dx, n) || !aligned(d_weight, p) || !aligned(d_dweight, p) || !aligned(d_dbias, p) ||
        !aligned(d_mean, 4) || !aligned(d_rstd, 4))
        return refuse("pxr_layer_norm_backward", "a buffer is not aligned to its elements");
    const size_t need = d_dweight || d_dbias ? pxr::layer_norm_workspace(*d) : 0;
    if (need && (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 16)))
        return refuse("pxr_layer_norm_backward", "the workspace is missing, too small or not 16-byte aligned");
    std::string err;
    return finish(pxr::launch_layer_norm_backward(*d, d_dy, d_x, d_mean, d_rstd, d_weight, d_dx, d_dweight, d_dbias, d_workspace, hip_stream, err),
                  "pxr_layer_norm_backward", err);
}

int pxr_linear_attention_create(const pxr_linear_attention_desc* d, pxr_linear_attention** out) {
    using pxr::set_error;
    const char* call = "pxr_linear_attention_create";
    if (!d || !out || !d->log_decay) return refuse(call, "null argument");
    if (d->n_heads == 0 || d->n_heads > 65535u || d->d_key == 0 || d->d_value == 0) return refuse(call, "n_heads must lie in [1,65535], d_key and d_value must be positive");
    if (d->d_key > 256u || d->d_value > 256u) return set_error(PXR_ERR_UNSUPPORTED, std::string(call) + ": d_key and d_value must be at most 256");
    if (!std::isfinite(d->scale)) return refuse(call, "non-finite scale");
    for (uint32_t h = 0; h < d->n_heads; ++h)
        if (!std::isfinite(d->log_decay[h]) || d->log_decay[h] > 0.0f) return refuse(call, "a log_decay is positive or not finite");
    pxr_linear_attention* a = new (std::nothrow) pxr_linear_attention();
    pxr::LinearAttentionHead* heads = new (std::nothrow) pxr::LinearAttentionHead[d->n_heads];
    if (!a || !heads) {
        delete a;
        delete[] heads;
        return set_error(PXR_ERR_OOM, std::string(call) + ": host allocation failed");
    }
    a->c.n_heads = d->n_heads;
    a->c.dk = d->d_key;
    a->c.dv = d->d_value;
    a->c.scale = d->scale;
    for (uint32_t h = 0; h < d->n_heads; ++h) pxr::fill_head(heads[h], d->log_decay[h]);
    const size_t bytes = sizeof(pxr::LinearAttentionHead) * d->n_heads;
    void* table = nullptr;
    hipError_t rc = hipMalloc(&table, bytes);
    const bool oom = rc == hipErrorOutOfMemory;
    if (rc == hipSuccess) rc = hipMemcpy(table, heads, bytes, hipMemcpyHostToDevice);
    int dev = 0, cus = 0;
    if (rc == hipSuccess) rc = hipGetDevice(&dev);
    if (rc == hipSuccess) rc = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
    delete[] heads;
    std::string err;
    if (rc != hipSuccess || pxr::prepare_linear_attention_kernels(err) != PXR_OK) {
        (void)hipFree(table);
        delete a;
        return set_error(oom ? PXR_ERR_OOM : PXR_ERR_DEVICE, std::string(call) + ": " + (rc != hipSuccess ? hipGetErrorString(rc) : err.c_str()));
    }
    a->c.heads = static_cast<const pxr::LinearAttentionHead*>(table);
    a->c.n_cus = (uint32_t)cus;
    *out = a;
    return PXR_OK;
}

int pxr_linear_attention_destroy(pxr_linear_attention* a) {
    if (!a) return PXR_OK;
    const hipError_t rc = hipFree(const_cast<pxr::LinearAttentionHead*>(a->c.heads));
    delete a;
    if (rc != hipSuccess) return pxr::set_error(PXR_ERR_DEVICE, std::string("pxr_linear_attention_destroy: hipFree failed: ") + hipGetErrorString(rc));
    return PXR_OK;
}

int pxr_linear_attention_workspace(const pxr_linear_attention* a, uint32_t dtype, uint32_t n_envs, uint32_t n_steps, uint32_t backward,
                                   size_t* bytes) {
    if (!a || !bytes || n_envs == 0 || (uint64_t)n_envs * a->c.n_heads > (1u << 21) || n_steps > 0x7FFFFFFFu || dtype > PXR_BF16)
        return refuse("pxr_linear_attention_workspace", "null argument, no or too many environments or steps, or a dtype that is none");
    *bytes = pxr::linear_attention_workspace(a->c, dtype, n_envs, n_steps, backward != 0);
    return PXR_OK;
}

int pxr_linear_attention_forward(pxr_linear_attention* a, const pxr_rollout* r, const pxr_tokens* out, float* d_state_out, void* d_workspace,
                                 size_t workspace_bytes, void* hip_stream) {
    const char* call = "pxr_linear_attention_forward";
    if (const char* why = wrong_rollout(a, r, false)) return refuse(call, why);
    if (wrong_view(&r->q, r->dtype, r->n_steps) || wrong_view(&r->k, r->dtype, r->n_steps) || wrong_view(&r->v, r->dtype, r->n_steps) ||
        wrong_view(out, r->dtype, r->n_steps) || !aligned(d_state_out, 4))
        return refuse(call, "a buffer is null or not aligned to its elements");
    if (overlap(r->d_state, d_state_out, (size_t)r->n_envs * a->c.n_heads * a->c.dk * a->c.dv)) return refuse(call, "the states overlap");
    const size_t need = pxr::linear_attention_workspace(a->c, r->dtype, r->n_envs, r->n_steps, false);
    if (need && (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 16)))
        return refuse(call, "the workspace is missing, too small or not 16-byte aligned");
    std::string err;
    return finish(pxr::launch_linear_attention_forward(a->c, *r, *out, d_state_out, d_workspace, hip_stream, err), call, err);
}

int pxr_linear_attention_backward(pxr_linear_attention* a, const pxr_rollout* r, const pxr_tokens* dout, const float* d_dstate_out,
                                  const pxr_tokens* dq, const pxr_tokens* dk, const pxr_tokens* dv, float* d_dstate, void* d_workspace,
                                  size_t workspace_bytes, void* hip_stream) {
    const char* call = "pxr_linear_attention_backward";
    if (const char* why = wrong_rollout(a, r, false)) return refuse(call, why);
    for (const pxr_tokens* t : {&r->q, &r->k, &r->v, dout, dq, dk, dv})
        if (wrong_view(t, r->dtype, r->n_steps)) return refuse(call, "a buffer is null or not aligned to its elements");
    if (!aligned(d_dstate_out, 4) || !aligned(d_dstate, 4)) return refuse(call, "a buffer is null or not aligned to its elements");
    const size_t n = (size_t)r->n_envs * a->c.n_heads * a->c.dk * a->c.dv;
    if (overlap(r->d_state, d_dstate, n) || overlap(d_dstate_out, d_dstate, n)) return refuse(call, "the states overlap");
    const size_t need = pxr::linear_attention_workspace(a->c, r->dtype, r->n_envs, r->n_steps, true);
    if (need && (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 16)))
        return refuse(call, "the workspace is missing, too small or not 16-byte aligned");
    std::string err;
    return finish(pxr::launch_linear_attention_backward(a->c, *r, *dout, d_dstate_out, *dq, *dk, *dv, d_dstate, d_workspace, hip_stream, err), call, err);
}

int pxr_linear_attention_step(pxr_linear_attention* a, const pxr_rollout* r, float* d_state, const pxr_tokens* out, void* hip_stream) {
    const char* call = "pxr_linear_attention_step";
    if (const char* why = wrong_rollout(a, r, true)) return refuse(call, why);
    if (wrong_view(&r->q, r->dtype, 1) || wrong_view(&r->k, r->dtype, 1) || wrong_view(&r->v, r->dtype, 1) || wrong_view(out, r->dtype, 1) ||
        !d_state || !aligned(d_state, 4))
        return refuse(call, "a buffer is null or not aligned to its elements");
    std::string err;
    return finish(pxr::launch_linear_attention_step(a->c, *r, d_state, *out, hip_stream, err), call, err);
}

int pxr_gated_recurrence_workspace(uint32_t n_envs, uint32_t n_steps, uint32_t width, uint32_t backward, size_t* bytes) {
    const char* call = "pxr_gated_recurrence_workspace";
    if (const char* why = wrong_gated_sizes(n_envs, n_steps, width)) return refuse(call, why);
    if (!bytes) return refuse(call, "null argument");
    *bytes = pxr::gated_recurrence_workspace(n_envs, n_steps, width, backward != 0);
    return PXR_OK;
}

int pxr_gated_recurrence_forward(const pxr_gated_rollout* r, const pxr_steps* out, float* d_state_out, void* d_workspace, size_t workspace_bytes,
                                 void* hip_stream) {
    const char* call = "pxr_gated_recurrence_forward";
    if (const char* why = wrong_gated(r, false)) return refuse(call, why);
    if (wrong_view(&r->x, r->dtype, r->n_steps) || wrong_view(&r->gate, r->dtype, r->n_steps) || wrong_view(out, r->dtype, r->n_steps) ||
        !aligned(d_state_out, 4))
        return refuse(call, "a buffer is null or not aligned to its elements");
    if (overlap(r->d_state, d_state_out, (size_t)r->n_envs * r->width)) return refuse(call, "the states overlap");
    if (pxr::share(view(*out, *r), {view(r->x, *r), view(r->gate, *r)})) return refuse(call, "out overlaps what is read");
    const size_t need = pxr::gated_recurrence_workspace(r->n_envs, r->n_steps, r->width, false);
    if (need && (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 16)))
        return refuse(call, "the workspace is missing, too small or not 16-byte aligned");
    std::string err;
    return finish(pxr::launch_gated_recurrence_forward(*r, *out, d_state_out, d_workspace, hip_stream, err), call, err);
}

int pxr_gated_recurrence_backward(const pxr_gated_rollout* r, const pxr_steps* dout, const float* d_dstate_out, const pxr_steps* dx,
                                  const pxr_steps* dgate, float* d_dstate, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    const char* call = "pxr_gated_recurrence_backward";
    if (const char* why = wrong_gated(r, false)) return refuse(call, why);
    for (const pxr_steps* t : {&r->x, &r->gate, dout, dx, dgate})
        if (wrong_view(t, r->dtype, r->n_steps)) return refuse(call, "a buffer is null or not aligned to its elements");
    if (!aligned(d_dstate_out, 4) || !aligned(d_dstate, 4)) return refuse(call, "a buffer is null or not aligned to its elements");
    const size_t n = (size_t)r->n_envs * r->width;
    if (overlap(r->d_state, d_dstate, n) || overlap(d_dstate_out, d_dstate, n)) return refuse(call, "the states overlap");
    const pxr::View x = view(r->x, *r), gate = view(r->gate, *r), given = view(*dout, *r), to_gate = view(*dgate, *r);
    if (pxr::share(view(*dx, *r), {x, gate, given, to_gate}) || pxr::share(to_gate, {x, gate, given})) return refuse(call, "dx or dgate overlaps what is read, or each other");
    const size_t need = pxr::gated_recurrence_workspace(r->n_envs, r->n_steps, r->width, true);
    if (need && (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 16)))
        return refuse(call, "the workspace is missing, too small or not 16-byte aligned");
    std::string err;
    return finish(pxr::launch_gated_recurrence_backward(*r, *dout, d_dstate_out, *dx, *dgate, d_dstate, d_workspace, hip_stream, err), call, err);
}

int pxr_gated_recurrence_step(const pxr_gated_rollout* r, float* d_state, const pxr_steps* out, void* hip_stream) {
    const char* call = "pxr_gated_recurrence_step";
    if (const char* why = wrong_gated(r, true)) return refuse(call, why);
    if (wrong_view(&r->x, r->dtype, 1) || wrong_view(&r->gate, r->dtype, 1) || wrong_view(out, r->dtype, 1) || !d_state || !aligned(d_state, 4))
        return refuse(call, "a buffer is null or not aligned to its elements");
    for (const pxr_steps* t : {&r->x, &r->gate})  // (a lane has read its values before it writes them)
        if (!pxr::itself(view(*out, *r), view(*t, *r)) && pxr::share(view(*out, *r), view(*t, *r))) return refuse(call, "out overlaps what is read");
    std::string err;
    return finish(pxr::launch_gated_recurrence_step(*r, d_state, *out, hip_stream, err), call, err);
}

int pxr_head_norm_create(const pxr_head_norm_desc* d, pxr_head_norm** out) {
    using pxr::set_error;
    const char* call = "pxr_head_norm_create";
    if (!d || !out || (d->d_rotary && !d->frequencies)) return refuse(call, "null argument");
    if (d->d_head == 0 || d->d_rotary % 2u || d->d_rotary > d->d_head) return refuse(call, "d_head must be positive, d_rotary even and at most d_head");
    if (d->d_head > 256u) return set_error(PXR_ERR_UNSUPPORTED, std::string(call) + ": d_head must be at most 256");
    if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return refuse(call, "eps must be finite and not negative");
    uint64_t turns[128] = {};
    for (uint32_t i = 0; i < d->d_rotary / 2u; ++i) {
        if (!(std::fabs(d->frequencies[i]) <= 1048576.0)) return refuse(call, "a frequency is not finite or above 2^20");
        turns[i] = pxr::turns_of(d->frequencies[i]);
    }
    pxr_head_norm* n = new (std::nothrow) pxr_head_norm();
    if (!n) return set_error(PXR_ERR_OOM, std::string(call) + ": host allocation failed");
    void* table = nullptr;
    hipError_t rc = hipMalloc(&table, sizeof(turns));
    const bool oom = rc == hipErrorOutOfMemory;
    if (rc == hipSuccess) rc = hipMemcpy(table, turns, sizeof(turns), hipMemcpyHostToDevice);
    if (rc != hipSuccess) {
        (void)hipFree(table);
        delete n;
        return set_error(oom ? PXR_ERR_OOM : PXR_ERR_DEVICE, std::string(call) + ": " + hipGetErrorString(rc));
    }
    n->c.d = d->d_head;
    n->c.r = d->d_rotary;
    n->c.eps = d->eps;
    n->c.turns = static_cast<const uint64_t*>(table);
    *out = n;
    return PXR_OK;
}

int pxr_head_norm_destroy(pxr_head_norm* n) {
    if (!n) return PXR_OK;
    const hipError_t rc = hipFree(const_cast<uint64_t*>(n->c.turns));
    delete n;
    if (rc != hipSuccess) return pxr::set_error(PXR_ERR_DEVICE, std::string("pxr_head_norm_destroy: hipFree failed: ") + hipGetErrorString(rc));
    return PXR_OK;
}

int pxr_head_norm_forward(pxr_head_norm* n, const pxr_heads* r, const pxr_tokens* q_out, const pxr_tokens* k_out, void* hip_stream) {
    const char* call = "pxr_head_norm_forward";
    if (const char* why = wrong_heads(n, r)) return refuse(call, why);
    if (wrong_head_buffers(r, {&r->q, q_out}, {&r->k, k_out})) return refuse(call, "a buffer is null or not aligned to its elements");
    if (heads_overlap(r, n->c.d, q_out, k_out, {&r->q}, {&r->k})) return refuse(call, "q_out or k_out overlaps heads that it is not itself");
    std::string err;
    return finish(pxr::launch_head_norm_forward(n->c, *r, q_out, k_out, hip_stream, err), call, err);
}

int pxr_head_norm_workspace(const pxr_head_norm* n, const pxr_heads* r, size_t* bytes) {
    const char* call = "pxr_head_norm_workspace";
    if (const char* why = wrong_heads(n, r)) return refuse(call, why);
    if (!bytes) return refuse(call, "null argument");
    *bytes = pxr::head_norm_workspace(n->c, *r);
    return PXR_OK;
}

int pxr_head_norm_backward(pxr_head_norm* n, const pxr_heads* r, const pxr_tokens* dq_out, const pxr_tokens* dk_out, const pxr_tokens* dq, const pxr_tokens* dk,
                           void* d_dq_weight, void* d_dk_weight, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    const char* call = "pxr_head_norm_backward";
    if (const char* why = wrong_heads(n, r)) return refuse(call, why);
    const size_t p = element(r->param_dtype);
    if (wrong_head_buffers(r, {&r->q, dq_out, dq}, {&r->k, dk_out, dk}) || !aligned(d_dq_weight, p) || !aligned(d_dk_weight, p))
        return refuse(call, "a buffer is null or not aligned to its elements");
    if (heads_overlap(r, n->c.d, dq, dk, {&r->q, dq_out}, {&r->k, dk_out})) return refuse(call, "dq or dk overlaps heads that it is not itself");
    const size_t need = d_dq_weight || d_dk_weight ? pxr::head_norm_workspace(n->c, *r) : 0;
    if (need && (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 16)))
        return refuse(call, "the workspace is missing, too small or not 16-byte aligned");
    std::string err;
    return finish(pxr::launch_head_norm_backward(n->c, *r, dq_out, dk_out, dq, dk, d_dq_weight, d_dk_weight, d_workspace, hip_stream, err), call, err);
}

}  // extern "C"

void pxr::fill_head(LinearAttentionHead& h, float log_decay) {
    const auto split = [](double g, float& head, float& rest) {
        head = (float)g;
        rest = (float)(g - (double)head);
    };
    h.log_decay = (double)log_decay;
    split(std::exp((double)log_decay), h.decay, h.decay_rest);
    split(std::exp((double)log_decay * 32.0), h.decay_chunk, h.decay_chunk_rest);
    for (int n = 0; n <= 32; ++n) h.power[n] = (float)std::exp((double)log_decay * n);
}

// frequency / 2 pi as a fraction of 2^64, modulo whole turns, rounded once: the frequency's 53 bits times 128 bits of 1 / 2 pi in whole numbers (frequencies are below 2^21, so of the bits in front of the point
// at most 18 go, and what is cut off before the rounding is below 2^-31 of a unit).
uint64_t pxr::turns_of(double frequency) {
    typedef unsigned __int128 wide;
    constexpr uint64_t kHigh = 0x28BE60DB9391054Aull, kLow = 0x7F09D5F47D4D3770ull;  // 1 / 2 pi in fractions of 2^128
    int exponent;
    const uint64_t bits = (uint64_t)std::ldexp(std::frexp(std::fabs(frequency), &exponent), 53);  // times 2^(exponent - 53)
    const wide high = (wide)bits * kHigh + (((wide)bits * kLow) >> 64);  // in fractions of 2^64, times 2^(exponent - 53)
    const int down = 53 - exponent;  // at least 32
    const uint64_t turns = down > 127 ? 0u : (uint64_t)(((high >> (down - 1)) + 1u) >> 1);
    return frequency < 0.0 ? 0u - turns : turns;
}
