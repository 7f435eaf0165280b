// ops_api.cpp -- C entries of the operators around a quantum layer (qlayer.h):
// argument checks, workspace layout, launches on the caller's stream. They hold
// no state and allocate nothing.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "errors.hpp"
#include "norm.hpp"
#include "ortho.hpp"
#include "qlayer.h"

using namespace qlayer;

namespace {

int fail(int code, const char* what, const char* detail = nullptr) { return set_error(code, what, detail); }

bool known_type(int t) { return t >= QL_F32 && t <= QL_F16; }

// A device array's address is a multiple of its element's size (NULL is).
bool aligned(const void* p, int type) { return (uintptr_t)p % elem_size(type) == 0; }

const int64_t MOST_ELEMENTS = (int64_t)1 << 46;

int check_norm(int type, int wtype, int64_t rows, int64_t features) {
    if (!known_type(type) || !known_type(wtype)) return fail(QL_EINVAL, "unknown type");
    if (wtype != type && !(wtype == QL_F32 && (type == QL_BF16 || type == QL_F16)))
        return fail(QL_EUNSUPPORTED, "weight_type is neither the rows' type nor QL_F32 beside 16-bit rows");
    if (rows < 0) return fail(QL_EINVAL, "rows must be >= 0");
    if (features < 1 || features > 1 << 30) return fail(QL_EINVAL, "features out of range [1, 2^30]");
    if (rows > MOST_ELEMENTS / features) return fail(QL_EINVAL, "rows * features too large");
    return QL_OK;
}

bool stride_ok(int64_t rows, int64_t stride) {
    return stride >= 0 && (rows <= 1 || stride <= MOST_ELEMENTS / rows);
}

// The array's addresses: strides that are no overflow, and for one that is
// written, no two elements at one address by a stride of 0.
bool strides_ok(const int64_t* s, int64_t batch, int64_t rows, int64_t cols, bool written) {
    const int64_t n[3] = {batch, rows, cols};
    for (int k = 0; k < 3; k++)
        if (n[k] > 1 && (s[k] < 0 || s[k] > MOST_ELEMENTS / n[k] || (written && s[k] == 0))) return false;
    return true;
}

int check_shapes(int type, const ql_matrix* mats, int32_t count) {
    if (!known_type(type)) return fail(QL_EINVAL, "unknown type");
    if (count < 0) return fail(QL_EINVAL, "count must be >= 0");
    if (count > 0 && !mats) return fail(QL_EINVAL, "matrices is NULL");
    int64_t tiles = 0;  // of 64x64, and rows
    for (int32_t k = 0; k < count; k++) {
        const ql_matrix& q = mats[k];
        if (q.rows < 1 || q.cols < 1 || q.rows > 65536 || q.cols > 65536)
            return fail(QL_EINVAL, "rows or cols out of range [1, 65536]");
        const int64_t each = ((q.rows + 63) / 64) * ((q.cols + 63) / 64) + q.rows;
        if (q.batch < 0 || q.batch > INT32_MAX / each) return fail(QL_EINVAL, "batch out of range");
        tiles += q.batch * each;
        if (tiles > INT32_MAX) return fail(QL_EINVAL, "too many matrices for one call");
    }
    if (!ortho_launchable(type, mats, count)) return fail(QL_EINVAL, "too many matrices for one call");
    return QL_OK;
}

int run_ortho(OrthoCall& c, const ql_ortho_options* o, void* ws, size_t ws_bytes, hipStream_t stream, const char* what) {
    if (int rc = check_shapes(c.type, c.mats, c.count)) return rc;
    c.a = o ? o->a : 3.4445, c.b = o ? o->b : -4.7750, c.c = o ? o->c : 2.0315;
    c.eps = o ? o->eps : 1e-7, c.steps = o ? o->steps : 5;
    if (!(c.eps >= 0) || std::isinf(c.eps)) return fail(QL_EINVAL, "eps must be finite and >= 0");
    if (c.steps < 1 || c.steps > 64) return fail(QL_EINVAL, "steps out of range [1, 64]");
    double most_x, most_q;
    if (!ortho_bounds(c.a, c.b, c.c, c.steps, most_x, most_q))
        return fail(QL_EINVAL, "coefficients let singular values grow past 64");
    const int state = c.type == QL_F64 ? QL_F64 : QL_F32;
    for (int32_t k = 0; k < c.count; k++) {
        const ql_matrix& q = c.mats[k];
        if (q.batch == 0) continue;
        if (!q.grad || !q.out || (c.muon && !q.momentum)) return fail(QL_EINVAL, "grad, out or momentum is NULL");
        if (!aligned(q.grad, c.type) || !aligned(q.out, c.type) || (c.muon && !aligned(q.momentum, state)))
            return fail(QL_EINVAL, "misaligned pointer");
        if (!strides_ok(q.grad_stride, q.batch, q.rows, q.cols, false) ||
            !strides_ok(q.out_stride, q.batch, q.rows, q.cols, true) ||
            (c.muon && !strides_ok(q.momentum_stride, q.batch, q.rows, q.cols, true)))
            return fail(QL_EINVAL, "stride out of range");
    }
    if (const size_t need = ortho_workspace(c.type, c.mats, c.count)) {
        if (!ws) return fail(QL_EINVAL, "workspace is NULL");
        if ((uintptr_t)ws % 16) return fail(QL_EINVAL, "misaligned workspace");
        if (ws_bytes < need) return fail(QL_ENOMEM, "workspace too small");
    }
    const hipError_t e = launch_ortho(c, ws, stream);
    if (e != hipSuccess) return fail(QL_EHIP, what, hipGetErrorString(e));
    return set_error(QL_OK, "");
}

}  // namespace

extern "C" {

int ql_orthogonalize_workspace_bytes(ql_type type, const ql_matrix* matrices, int32_t count, size_t* out) {
    if (!out) return fail(QL_EINVAL, "NULL argument");
    if (int rc = check_shapes(type, matrices, count)) return rc;
    *out = ortho_workspace(type, matrices, count);
    return set_error(QL_OK, "");
}

int ql_orthogonalize(ql_type type, const ql_matrix* matrices, int32_t count, const ql_ortho_options* options, void* ws,
                     size_t ws_bytes, hipStream_t stream) {
    OrthoCall c{};
    c.type = type, c.mats = matrices, c.count = count;
    return run_ortho(c, options, ws, ws_bytes, stream, "orthogonalize");
}

int ql_muon_step(ql_type type, const ql_matrix* matrices, int32_t count, const ql_muon_options* muon,
                 const ql_ortho_options* options, void* ws, size_t ws_bytes, hipStream_t stream) {
    OrthoCall c{};
    c.type = type, c.mats = matrices, c.count = count, c.muon = true;
    const double lr = muon ? muon->lr : 0.02, decay = muon ? muon->weight_decay : 0;
    c.momentum = muon ? muon->momentum : 0.95, c.nesterov = muon ? muon->nesterov != 0 : true;
    if (!std::isfinite(lr) || !std::isfinite(decay) || !std::isfinite(c.momentum))
        return fail(QL_EINVAL, "lr, momentum and weight_decay must be finite");
    c.keep = 1 - lr * decay, c.step = lr;
    return run_ortho(c, options, ws, ws_bytes, stream, "muon step");
}

int ql_layer_norm_forward(ql_type type, ql_type weight_type, int64_t rows, int64_t features, const void* x,
                          int64_t x_stride, const void* weight, const void* bias, double eps, void* y, void* mean,
                          void* rstd, void* ws, size_t ws_bytes, hipStream_t stream) {
    if (int rc = check_norm(type, weight_type, rows, features)) return rc;
    if (!(eps >= 0) || std::isinf(eps)) return fail(QL_EINVAL, "eps must be finite and >= 0");
    if (!stride_ok(rows, x_stride)) return fail(QL_EINVAL, "x_stride out of range");
    if (rows > 0 && (!x || !y)) return fail(QL_EINVAL, "x or y is NULL");
    const int stat = type == QL_F64 ? QL_F64 : QL_F32;
    if (!aligned(x, type) || !aligned(y, type) || !aligned(weight, weight_type) || !aligned(bias, weight_type) ||
        !aligned(mean, stat) || !aligned(rstd, stat))
        return fail(QL_EINVAL, "misaligned pointer");
    if (const size_t need = norm_workspace(type, rows, features, false)) {
        if (!ws) return fail(QL_EINVAL, "workspace is NULL");
        if (!aligned(ws, QL_F64)) return fail(QL_EINVAL, "misaligned workspace");
        if (ws_bytes < need) return fail(QL_ENOMEM, "workspace too small");
    }
    NormArgs a{};
    a.x = x, a.weight = weight, a.bias = bias, a.y = y, a.mean = mean, a.rstd = rstd, a.sums = ws;
    a.rows = rows, a.D = features, a.x_stride = x_stride, a.eps = eps;
    const hipError_t e = launch_norm_forward(type, weight_type, a, stream);
    if (e != hipSuccess) return fail(QL_EHIP, "layer norm", hipGetErrorString(e));
    return set_error(QL_OK, "");
}

int ql_layer_norm_workspace_bytes(ql_type type, int64_t rows, int64_t features, int backward, size_t* out) {
    if (!out) return fail(QL_EINVAL, "NULL argument");
    if (int rc = check_norm(type, type, rows, features)) return rc;
    *out = norm_workspace(type, rows, features, backward != 0);
    return set_error(QL_OK, "");
}

int ql_layer_norm_backward(ql_type type, ql_type weight_type, int64_t rows, int64_t features, const void* grad_y,
                           int64_t grad_stride, const void* x, int64_t x_stride, const void* mean, const void* rstd,
                           const void* weight, void* grad_x, void* grad_weight, void* grad_bias, void* ws,
                           size_t ws_bytes, hipStream_t stream) {
    if (int rc = check_norm(type, weight_type, rows, features)) return rc;
    if (!stride_ok(rows, x_stride) || !stride_ok(rows, grad_stride)) return fail(QL_EINVAL, "stride out of range");
    if (rows > 0 && (!grad_y || !x || !mean || !rstd)) return fail(QL_EINVAL, "grad_y, x, mean or rstd is NULL");
    const int stat = type == QL_F64 ? QL_F64 : QL_F32;
    if (!aligned(grad_y, type) || !aligned(x, type) || !aligned(grad_x, type) || !aligned(weight, weight_type) ||
        !aligned(grad_weight, weight_type) || !aligned(grad_bias, weight_type) || !aligned(mean, stat) ||
        !aligned(rstd, stat))
        return fail(QL_EINVAL, "misaligned pointer");
    if (grad_x || grad_weight || grad_bias) {
        if (!ws) return fail(QL_EINVAL, "workspace is NULL");
        if (!aligned(ws, QL_F64)) return fail(QL_EINVAL, "misaligned workspace");
        if (ws_bytes < norm_workspace(type, rows, features, true)) return fail(QL_ENOMEM, "workspace too small");
    }
    NormArgs a{};
    a.grad = grad_y, a.x = x, a.mean = (void*)mean, a.rstd = (void*)rstd, a.weight = weight;
    a.grad_x = grad_x, a.grad_weight = grad_weight, a.grad_bias = grad_bias, a.part = ws;
    a.rows = rows, a.D = features, a.x_stride = x_stride, a.grad_stride = grad_stride;
    const hipError_t e = launch_norm_backward(type, weight_type, a, stream);
    if (e != hipSuccess) return fail(QL_EHIP, "layer norm backward", hipGetErrorString(e));
    return set_error(QL_OK, "");
}

}  // extern "C"
