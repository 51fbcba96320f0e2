// C ABI of a learner's update (pxr_orthogonalise in include/pxr.h): validation, bounds of the singular values, launch.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "pxr_internal.h"
#include "views.h"

namespace {

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int refuse(const char* call, const char* why, int code = PXR_ERR_INVALID_ARG) { return pxr::set_error(code, std::string(call) + ": " + why); }

// Everything but the buffers: PXR_OK, or the code of a refusal that has been recorded.
int check(const char* call, const pxr_orthogonalise_desc* d) {
    if (!d || !d->coefficients) return refuse(call, "null argument");
    if (d->dtype > PXR_BF16) return refuse(call, "dtype must be fp32 or bfloat16");
    if (d->rows == 0 || d->cols == 0) return refuse(call, "rows and cols must be positive");
    if (d->n_matrices > 65535u) return refuse(call, "n_matrices must be at most 65535");
    if (d->n_steps == 0 || d->n_steps > 64u) return refuse(call, "n_steps must lie in [1,64]");
    if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return refuse(call, "eps must be finite and not negative");
    if ((d->rows > 1 && (d->x_row < (int64_t)d->cols || d->out_row < (int64_t)d->cols))) return refuse(call, "a row stride is smaller than cols");
    if (std::min(d->rows, d->cols) > (1u << 15) || std::max(d->rows, d->cols) > (1u << 28) || (uint64_t)d->rows * d->cols > (1ull << 32))
        return refuse(call, "the smaller of rows and cols must be at most 2^15, the larger 2^28, rows * cols 2^32", PXR_ERR_UNSUPPORTED);
    // (a row stride of 2^40 and more is no row of any memory: the product below does not wrap)
    if (d->out_row > (1ll << 40)) return refuse(call, "a row stride is too large");
    const int64_t extent = (int64_t)(d->rows - 1u) * (d->rows > 1 ? d->out_row : 0) + d->cols;
    if (d->n_matrices > 1 && d->out_matrix < extent && d->out_matrix > -extent) return refuse(call, "matrices of the result overlap");
    double most = 1.0;
    for (uint32_t k = 0; k < d->n_steps; ++k) {
        const float* c = d->coefficients + 3 * k;
        if (!std::isfinite(c[0]) || !std::isfinite(c[1]) || !std::isfinite(c[2])) return refuse(call, "a coefficient is not finite");
        const pxr::OrthogonaliseBounds next = pxr::orthogonalise_bounds(c[0], c[1], c[2], most);
        if (!(next.most <= 1048576.0) || !(next.factor <= 1e12)) return refuse(call, "steps under which a singular value may pass 2^20");
        most = next.most;
    }
    return PXR_OK;
}

}  // namespace

pxr::OrthogonaliseBounds pxr::orthogonalise_bounds(double a, double b, double c, double most) {
    const double end = most * most;
    OrthogonaliseBounds r{0.0, std::max(std::fabs(a), std::fabs(a + b * end + c * end * end))};
    const auto value = [&](double z) { return std::fabs(std::sqrt(z) * (a + z * (b + z * c))); };
    const auto see = [&](double z) {  // z = t^2
        if (z > 0.0 && z < end) r.most = std::max(r.most, value(z));
    };
    r.most = value(end);
    // a + 3 b z + 5 c z^2 = 0, and the factor's own turning point
    if (c != 0.0) {
        const double under = 9.0 * b * b - 20.0 * a * c;
        if (under >= 0.0) {
            const double root = std::sqrt(under);
            see((-3.0 * b + root) / (10.0 * c));
            see((-3.0 * b - root) / (10.0 * c));
        }
        const double turn = -b / (2.0 * c);
        if (turn > 0.0 && turn < end) r.factor = std::max(r.factor, std::fabs(a + turn * (b + turn * c)));
    } else if (b != 0.0) {
        see(-a / (3.0 * b));
    }
    // (what is computed is off by its roundings, and the next step's values with it)
    r.most *= 1.0 + 0x1p-10;
    return r;
}

extern "C" {

int pxr_orthogonalise_workspace(const pxr_orthogonalise_desc* d, size_t* bytes) {
    const char* call = "pxr_orthogonalise_workspace";
    if (const int rc = check(call, d)) return rc;
    if (!bytes) return refuse(call, "null argument");
    *bytes = d->n_matrices ? pxr::orthogonalise_workspace(*d) : 0;
    return PXR_OK;
}

int pxr_orthogonalise(const pxr_orthogonalise_desc* d, const void* d_x, void* d_out, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    const char* call = "pxr_orthogonalise";
    if (const int rc = check(call, d)) return rc;
    if (d->n_matrices == 0) return PXR_OK;
    const size_t n = d->dtype == PXR_F32 ? 4u : 2u;
    if (!d_x || !d_out || !aligned(d_x, n) || !aligned(d_out, n)) return refuse(call, "a buffer is null or not aligned to its elements");
    const auto view = [&](const void* data, int64_t matrix, int64_t row) { return pxr::View{data, n, d->cols, {{d->n_matrices, matrix}, {d->rows, row}, {1, 0}}}; };
    const pxr::View x = view(d_x, d->x_matrix, d->x_row), out = view(d_out, d->out_matrix, d->out_row);
    if (!pxr::itself(out, x) && pxr::share(out, x)) return refuse(call, "the result overlaps x, and is not x itself");
    const size_t need = pxr::orthogonalise_workspace(*d);
    if (need && (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 16)))
        return refuse(call, "the workspace is missing, too small or not 16-byte aligned");
    std::string err;
    const int rc = pxr::launch_orthogonalise(*d, d_x, d_out, d_workspace, hip_stream, err);
    return rc == PXR_OK ? PXR_OK : pxr::set_error(rc, std::string(call) + ": " + err);
}

}  // extern "C"
