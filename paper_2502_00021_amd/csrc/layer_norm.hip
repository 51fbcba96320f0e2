// Layer norm over rows, forward and backward (pxr_layer_norm_* in include/pxr.h).  gfx950 only.
//
//   mean = sum x / D,  rstd = 1 / sqrt(sum (x - mean)^2 / D + eps),  y = (x - mean) rstd w + b
//   dx = rstd (g - sum g / D - xh sum(g xh) / D),  g = w dy,  xh = (x - mean) rstd;  dw = sum_rows dy xh,  db = sum_rows dy
//
// All sums are fp32; the deviations are squared after the mean is taken off, so a row far from zero keeps its variance.

#include <hip/hip_runtime.h>

#include "pxr_internal.h"

namespace pxr {
namespace {

constexpr uint32_t kThreads = 256;

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __bf16* p) { return (float)*p; }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__bf16* p, float v) { *p = (__bf16)v; }  // round to nearest even

// Sum over the workgroup, the same bits in every lane.
__device__ __forceinline__ float group_sum(float v, float* lds) {
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m);
    __syncthreads();
    if ((threadIdx.x & 63u) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <class T, class P>
__global__ __launch_bounds__(kThreads) void norm_forward_kernel(const T* x, const P* weight, const P* bias, T* y, float* mean_out,
                                                                float* rstd_out, uint32_t D, int64_t x_stride, int64_t y_stride, float eps) {
    __shared__ float lds[4];
    const T* xr = x + (int64_t)blockIdx.x * x_stride;
    T* yr = y + (int64_t)blockIdx.x * y_stride;
    float s = 0.0f;
    for (uint32_t i = threadIdx.x; i < D; i += kThreads) s += load1(xr + i);
    const float mean = group_sum(s, lds) / (float)D;
    s = 0.0f;
    for (uint32_t i = threadIdx.x; i < D; i += kThreads) {
        const float c = load1(xr + i) - mean;
        s = __builtin_fmaf(c, c, s);
    }
    const float rstd = 1.0f / sqrtf(group_sum(s, lds) / (float)D + eps);
    for (uint32_t i = threadIdx.x; i < D; i += kThreads) {
        const float h = (load1(xr + i) - mean) * rstd;
        store1(yr + i, __builtin_fmaf(h, weight ? load1(weight + i) : 1.0f, bias ? load1(bias + i) : 0.0f));
    }
    if (threadIdx.x == 0) {
        if (mean_out) mean_out[blockIdx.x] = mean;
        if (rstd_out) rstd_out[blockIdx.x] = rstd;
    }
}

template <class T, class P>
__global__ __launch_bounds__(kThreads) void norm_dx_kernel(const T* dy, const T* x, const float* mean, const float* rstd, const P* weight,
                                                           T* dx, uint32_t D, int64_t dy_stride, int64_t x_stride, int64_t dx_stride) {
    __shared__ float lds[4];
    const T* dyr = dy + (int64_t)blockIdx.x * dy_stride;
    const T* xr = x + (int64_t)blockIdx.x * x_stride;
    T* dxr = dx + (int64_t)blockIdx.x * dx_stride;
    const float m = mean[blockIdx.x], r = rstd[blockIdx.x];
    float sg = 0.0f, sgx = 0.0f;
    for (uint32_t i = threadIdx.x; i < D; i += kThreads) {
        const float g = load1(dyr + i) * (weight ? load1(weight + i) : 1.0f);
        sg += g;
        sgx = __builtin_fmaf(g, (load1(xr + i) - m) * r, sgx);
    }
    sg = group_sum(sg, lds) / (float)D;
    sgx = group_sum(sgx, lds) / (float)D;
    for (uint32_t i = threadIdx.x; i < D; i += kThreads) {
        const float g = load1(dyr + i) * (weight ? load1(weight + i) : 1.0f);
        const float h = (load1(xr + i) - m) * r;
        store1(dxr + i, r * __builtin_fmaf(-h, sgx, g - sg));
    }
}

template <class T, class P>
__global__ __launch_bounds__(kThreads) void norm_dw_kernel(const T* dy, const T* x, const float* mean, const float* rstd, P* dweight,
                                                           P* dbias, uint32_t n, uint32_t D, int64_t dy_stride, int64_t x_stride) {
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= D) return;
    float w = 0.0f, b = 0.0f;
    for (uint32_t k = 0; k < n; ++k) {
        const float g = load1(dy + k * dy_stride + i);
        w = __builtin_fmaf(g, (load1(x + k * x_stride + i) - mean[k]) * rstd[k], w);
        b += g;
    }
    if (dweight) store1(dweight + i, w);
    if (dbias) store1(dbias + i, b);
}

template <class T, class P>
void forward_as(const pxr_layer_norm_desc& d, const void* x, const void* w, const void* b, void* y, float* mean, float* rstd, hipStream_t st) {
    hipLaunchKernelGGL((norm_forward_kernel<T, P>), dim3((uint32_t)d.n_rows), dim3(kThreads), 0, st, static_cast<const T*>(x),
                       static_cast<const P*>(w), static_cast<const P*>(b), static_cast<T*>(y), mean, rstd, d.width, d.x_stride, d.y_stride, d.eps);
}

template <class T, class P>
void backward_as(const pxr_layer_norm_desc& d, const void* dy, const void* x, const float* mean, const float* rstd, const void* w,
                 void* dx, void* dw, void* db, void*, hipStream_t st) {
    // (the sums over rows first: dx may be dy or x itself)
    if (dw || db)
        hipLaunchKernelGGL((norm_dw_kernel<T, P>), dim3((d.width + kThreads - 1) / kThreads), dim3(kThreads), 0, st,
                           static_cast<const T*>(dy), static_cast<const T*>(x), mean, rstd, static_cast<P*>(dw), static_cast<P*>(db),
                           (uint32_t)d.n_rows, d.width, d.y_stride, d.x_stride);
    if (d.n_rows)
        hipLaunchKernelGGL((norm_dx_kernel<T, P>), dim3((uint32_t)d.n_rows), dim3(kThreads), 0, st, static_cast<const T*>(dy),
                           static_cast<const T*>(x), mean, rstd, static_cast<const P*>(w), static_cast<T*>(dx), d.width, d.y_stride,
                           d.x_stride, d.dx_stride);
}

int launched(std::string& err) {
    const hipError_t rc = hipGetLastError();
    if (rc == hipSuccess) return PXR_OK;
    err = std::string("kernel launch failed: ") + hipGetErrorString(rc);
    return PXR_ERR_DEVICE;
}

}  // namespace

size_t layer_norm_workspace(const pxr_layer_norm_desc&) { return 0; }

int launch_layer_norm_forward(const pxr_layer_norm_desc& d, const void* x, const void* w, const void* b, void* y, float* mean, float* rstd,
                              void* stream, std::string& err) {
    if (d.n_rows == 0) return PXR_OK;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (d.dtype == PXR_F32)
        forward_as<float, float>(d, x, w, b, y, mean, rstd, st);
    else if (d.param_dtype == PXR_F32)
        forward_as<__bf16, float>(d, x, w, b, y, mean, rstd, st);
    else
        forward_as<__bf16, __bf16>(d, x, w, b, y, mean, rstd, st);
    return launched(err);
}

int launch_layer_norm_backward(const pxr_layer_norm_desc& d, const void* dy, const void* x, const float* mean, const float* rstd,
                               const void* w, void* dx, void* dw, void* db, void* ws, void* stream, std::string& err) {
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (d.dtype == PXR_F32)
        backward_as<float, float>(d, dy, x, mean, rstd, w, dx, dw, db, ws, st);
    else if (d.param_dtype == PXR_F32)
        backward_as<__bf16, float>(d, dy, x, mean, rstd, w, dx, dw, db, ws, st);
    else
        backward_as<__bf16, __bf16>(d, dy, x, mean, rstd, w, dx, dw, db, ws, st);
    return launched(err);
}

}  // namespace pxr
