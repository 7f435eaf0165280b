// seq_api.cpp -- C entries of the operators of a network that reads sequences
// (qlayer.h): argument checks, workspace layout, launches on the caller's
// stream. They hold no state and allocate nothing.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "checks.hpp"
#include "dropout.hpp"
#include "embed.hpp"
#include "rms.hpp"
#include "scan.hpp"

using namespace qlayer;

namespace {

int check_embedding(int type, int64_t count, int64_t rows, int64_t features) {
    if (!known_type(type)) return fail(QL_EINVAL, "unknown type");
    if (count < 0 || count > INT32_MAX) return fail(QL_EINVAL, "count out of range [0, 2^31)");
    if (rows < 1 || rows > INT32_MAX) return fail(QL_EINVAL, "rows out of range [1, 2^31)");
    if (features < 1 || features > 1 << 22) return fail(QL_EINVAL, "features out of range [1, 2^22]");
    if (std::max(rows, count) > MOST_ELEMENTS / features) return fail(QL_EINVAL, "too many elements");
    return QL_OK;
}

// A factor that the arithmetic (fp64 for QL_F64, else fp32) holds.
bool scale_ok(int type, double scale) {
    return std::isfinite(scale) && (type == QL_F64 || std::isfinite((float)scale));
}

static_assert(QL_SCAN_BLOCK == SCAN_BLOCK, "the header's block is the kernels'");

int check_scan(int type, int64_t batch, int64_t steps, int64_t features) {
    if (!known_type(type)) return fail(QL_EINVAL, "unknown type");
    if (steps < 0 || steps > 1 << 30) return fail(QL_EINVAL, "steps out of range [0, 2^30]");
    if (features < 1 || features > 1 << 22) return fail(QL_EINVAL, "features out of range [1, 2^22]");
    if (batch < 0 || batch > ((int64_t)1 << 27) / features) return fail(QL_EINVAL, "batch * features out of range [0, 2^27]");
    if (batch * features > MOST_ELEMENTS / std::max<int64_t>(steps, 1)) return fail(QL_EINVAL, "too many elements");
    return QL_OK;
}

bool strided_ok(int64_t batch, int64_t steps, const Strided& s) {
    return stride_ok(batch, s.batch) && stride_ok(steps, s.step);
}

int launched(hipError_t e, const char* what) {
    if (e != hipSuccess) return fail(QL_EHIP, what, hipGetErrorString(e));
    return set_error(QL_OK, "");
}

}  // namespace

extern "C" {

int ql_rms_norm_forward(ql_type type, ql_type weight_type, int64_t rows, int64_t features, const void* x,
                        int64_t x_stride, const void* residual, int64_t residual_stride, const void* weight, double eps,
                        void* summed, void* y, void* rstd, float* scale, void* ws, size_t ws_bytes, hipStream_t stream) {
    if (int rc = check_norm(type, weight_type, rows, features)) return rc;
    if (scale && type == QL_F64) return fail(QL_EUNSUPPORTED, "no output in 8 bits for QL_F64 rows");
    if (!(eps >= 0) || std::isinf(eps)) return fail(QL_EINVAL, "eps must be finite and >= 0");
    if (!stride_ok(rows, x_stride) || (residual && !stride_ok(rows, residual_stride)))
        return fail(QL_EINVAL, "stride out of range");
    if (rows > 0 && (!x || !y || (residual && !summed))) return fail(QL_EINVAL, "x, y or summed is NULL");
    if (!aligned(x, type) || !aligned(residual, type) || !aligned(summed, type) || (!scale && !aligned(y, type)) ||
        !aligned(weight, weight_type) || !aligned(rstd, wide_type(type)) || !aligned(scale, QL_F32))
        return fail(QL_EINVAL, "misaligned pointer");
    if (int rc = check_workspace(ws, ws_bytes, rms_workspace(type, rows, features, false))) return rc;
    RmsArgs a{};
    a.x = x, a.residual = residual, a.weight = weight, a.summed = summed, a.y = y, a.rstd = rstd, a.scale = scale;
    a.rows = rows, a.D = features, a.x_stride = x_stride, a.residual_stride = residual_stride, a.eps = eps;
    return launched(launch_rms_forward(type, weight_type, a, ws, stream), "rms norm");
}

int ql_rms_norm_workspace_bytes(ql_type type, int64_t rows, int64_t features, int backward, size_t* out) {
    if (!out) return fail(QL_EINVAL, "NULL argument");
    if (int rc = check_norm(type, type, rows, features)) return rc;
    *out = rms_workspace(type, rows, features, backward != 0);
    return set_error(QL_OK, "");
}

int ql_rms_norm_backward(ql_type type, ql_type weight_type, int64_t rows, int64_t features, const void* grad_y,
                         int64_t grad_stride, const void* grad_summed, int64_t grad_summed_stride, const void* s,
                         int64_t s_stride, const void* rstd, const void* weight, void* grad_x, void* grad_weight,
                         void* ws, size_t ws_bytes, hipStream_t stream) {
    if (int rc = check_norm(type, weight_type, rows, features)) return rc;
    if (!stride_ok(rows, s_stride) || !stride_ok(rows, grad_stride) ||
        (grad_summed && !stride_ok(rows, grad_summed_stride)))
        return fail(QL_EINVAL, "stride out of range");
    if (rows > 0 && (!grad_y || !s || !rstd)) return fail(QL_EINVAL, "grad_y, s or rstd is NULL");
    if (!aligned(grad_y, type) || !aligned(grad_summed, type) || !aligned(s, type) || !aligned(grad_x, type) ||
        !aligned(weight, weight_type) || !aligned(grad_weight, weight_type) || !aligned(rstd, wide_type(type)))
        return fail(QL_EINVAL, "misaligned pointer");
    if (grad_x || grad_weight)
        if (int rc = check_workspace(ws, ws_bytes, rms_workspace(type, rows, features, true))) return rc;
    RmsArgs a{};
    a.grad = grad_y, a.grad_sum = grad_summed, a.x = s, a.rstd = (void*)rstd, a.weight = weight;
    a.grad_x = grad_x, a.grad_weight = grad_weight;
    a.rows = rows, a.D = features, a.x_stride = s_stride, a.grad_stride = grad_stride;
    a.grad_sum_stride = grad_summed_stride;
    return launched(launch_rms_backward(type, weight_type, a, ws, stream), "rms norm backward");
}

int ql_embedding_forward(ql_type type, int tokens_64, int64_t count, int64_t rows, int64_t features, const void* tokens,
                         const void* weight, int64_t weight_stride, double scale, int has_padding, int64_t padding,
                         void* y, hipStream_t stream) {
    if (int rc = check_embedding(type, count, rows, features)) return rc;
    if (!scale_ok(type, scale)) return fail(QL_EINVAL, "scale must be finite, beside other rows than QL_F64 in QL_F32");
    if (!stride_ok(rows, weight_stride)) return fail(QL_EINVAL, "weight_stride out of range");
    if (count > 0 && (!tokens || !weight || !y)) return fail(QL_EINVAL, "tokens, weight or y is NULL");
    if (!aligned(tokens, tokens_64 ? QL_F64 : QL_F32) || !aligned(weight, type) || !aligned(y, type))
        return fail(QL_EINVAL, "misaligned pointer");
    EmbedArgs a{};
    a.tokens = tokens, a.weight = weight, a.y = y, a.n = count, a.rows = rows, a.D = features;
    a.weight_stride = weight_stride, a.padding = padding, a.padded = has_padding != 0, a.wide = tokens_64 != 0;
    a.scale = scale;
    return launched(launch_embed_forward(type, a, stream), "embedding");
}

int ql_embedding_workspace_bytes(ql_type type, int64_t count, int64_t rows, int64_t features, size_t* out) {
    if (!out) return fail(QL_EINVAL, "NULL argument");
    if (int rc = check_embedding(type, count, rows, features)) return rc;
    *out = embed_workspace(type, count, rows, features);
    return set_error(QL_OK, "");
}

int ql_embedding_backward(ql_type type, int tokens_64, int64_t count, int64_t rows, int64_t features,
                          const void* tokens, const void* grad_y, int64_t grad_stride, double scale, int has_padding,
                          int64_t padding, void* grad_weight, void* ws, size_t ws_bytes, hipStream_t stream) {
    if (int rc = check_embedding(type, count, rows, features)) return rc;
    if (!scale_ok(type, scale)) return fail(QL_EINVAL, "scale must be finite, beside other rows than QL_F64 in QL_F32");
    if (!stride_ok(count, grad_stride)) return fail(QL_EINVAL, "grad_stride out of range");
    if (!grad_weight || (count > 0 && (!tokens || !grad_y)))
        return fail(QL_EINVAL, "tokens, grad_y or grad_weight is NULL");
    if (!aligned(tokens, tokens_64 ? QL_F64 : QL_F32) || !aligned(grad_y, type) || !aligned(grad_weight, type))
        return fail(QL_EINVAL, "misaligned pointer");
    if (int rc = check_workspace(ws, ws_bytes, embed_workspace(type, count, rows, features))) return rc;
    EmbedArgs a{};
    a.tokens = tokens, a.grad = grad_y, a.grad_weight = grad_weight, a.n = count, a.rows = rows, a.D = features;
    a.grad_stride = grad_stride, a.padding = padding, a.padded = has_padding != 0, a.wide = tokens_64 != 0;
    a.scale = scale;
    return launched(launch_embed_backward(type, a, ws, stream), "embedding backward");
}

int ql_gated_scan_forward(ql_type type, int64_t batch, int64_t steps, int64_t features, const void* x, int64_t x_batch,
                          int64_t x_step, const void* gate, int64_t gate_batch, int64_t gate_step,
                          const uint8_t* starts, const void* initial, void* h, void* last, void* states, void* ws,
                          size_t ws_bytes, hipStream_t stream) {
    if (int rc = check_scan(type, batch, steps, features)) return rc;
    ScanArgs a{};
    a.x = {(void*)x, x_batch, x_step}, a.gate = {(void*)gate, gate_batch, gate_step};
    if (!strided_ok(batch, steps, a.x) || !strided_ok(batch, steps, a.gate))
        return fail(QL_EINVAL, "stride out of range");
    if (batch > 0 && steps > 0 && (!x || !gate || !h)) return fail(QL_EINVAL, "x, gate or h is NULL");
    const int wide = wide_type(type);
    if (!aligned(x, type) || !aligned(gate, type) || !aligned(h, type) || !aligned(initial, wide) ||
        !aligned(last, wide) || !aligned(states, wide))
        return fail(QL_EINVAL, "misaligned pointer");
    if (int rc = check_workspace(ws, ws_bytes, scan_workspace(type, batch, steps, features))) return rc;
    a.starts = starts, a.initial = initial, a.h = h, a.last = last, a.states = states, a.ws = ws;
    a.batch = batch, a.steps = steps, a.D = features;
    return launched(launch_scan_forward(type, a, stream), "gated scan");
}

int ql_gated_scan_workspace_bytes(ql_type type, int64_t batch, int64_t steps, int64_t features, size_t* out) {
    if (!out) return fail(QL_EINVAL, "NULL argument");
    if (int rc = check_scan(type, batch, steps, features)) return rc;
    *out = scan_workspace(type, batch, steps, features);
    return set_error(QL_OK, "");
}

int ql_gated_scan_backward(ql_type type, int64_t batch, int64_t steps, int64_t features, const void* grad_h,
                           int64_t grad_batch, int64_t grad_step, const void* x, int64_t x_batch, int64_t x_step,
                           const void* gate, int64_t gate_batch, int64_t gate_step, const void* states,
                           const uint8_t* starts, const void* grad_last, void* grad_x, void* grad_gate,
                           void* grad_initial, void* ws, size_t ws_bytes, hipStream_t stream) {
    if (int rc = check_scan(type, batch, steps, features)) return rc;
    ScanArgs a{};
    a.x = {(void*)x, x_batch, x_step}, a.gate = {(void*)gate, gate_batch, gate_step};
    a.grad = {(void*)grad_h, grad_batch, grad_step};
    if (!strided_ok(batch, steps, a.x) || !strided_ok(batch, steps, a.gate) || !strided_ok(batch, steps, a.grad))
        return fail(QL_EINVAL, "stride out of range");
    if (batch > 0 && steps > 0 && (!grad_h || !x || !gate || !states || !grad_x || !grad_gate))
        return fail(QL_EINVAL, "grad_h, x, gate, states, grad_x or grad_gate is NULL");
    const int wide = wide_type(type);
    if (!aligned(grad_h, type) || !aligned(x, type) || !aligned(gate, type) || !aligned(grad_x, type) ||
        !aligned(grad_gate, type) || !aligned(states, wide) || !aligned(grad_last, wide) || !aligned(grad_initial, wide))
        return fail(QL_EINVAL, "misaligned pointer");
    if (int rc = check_workspace(ws, ws_bytes, scan_workspace(type, batch, steps, features))) return rc;
    a.states = (void*)states, a.starts = starts, a.grad_last = grad_last, a.ws = ws;
    a.grad_x = grad_x, a.grad_gate = grad_gate, a.grad_initial = grad_initial;
    a.batch = batch, a.steps = steps, a.D = features;
    return launched(launch_scan_backward(type, a, stream), "gated scan backward");
}

int ql_gated_scan_step(ql_type type, int64_t batch, int64_t features, const void* x, int64_t x_batch, const void* gate,
                       int64_t gate_batch, const uint8_t* starts, void* state, void* h, hipStream_t stream) {
    if (int rc = check_scan(type, batch, 1, features)) return rc;
    ScanArgs a{};
    a.x = {(void*)x, x_batch, 0}, a.gate = {(void*)gate, gate_batch, 0};
    if (!strided_ok(batch, 1, a.x) || !strided_ok(batch, 1, a.gate)) return fail(QL_EINVAL, "stride out of range");
    if (batch > 0 && (!x || !gate || !state || !h)) return fail(QL_EINVAL, "x, gate, state or h is NULL");
    if (!aligned(x, type) || !aligned(gate, type) || !aligned(h, type) || !aligned(state, wide_type(type)))
        return fail(QL_EINVAL, "misaligned pointer");
    a.starts = starts, a.h = h, a.batch = batch, a.steps = 1, a.D = features;
    return launched(launch_scan_step(type, a, state, stream), "gated scan step");
}

int ql_dropout(ql_type type, int64_t rows, int64_t features, const void* x, int64_t x_stride, double p, uint64_t seed,
               uint64_t offset, const uint64_t* key, void* y, hipStream_t stream) {
    if (int rc = check_norm(type, type, rows, features)) return rc;
    if (!(p >= 0 && p <= 1)) return fail(QL_EINVAL, "p out of range [0, 1]");
    if (!stride_ok(rows, x_stride)) return fail(QL_EINVAL, "x_stride out of range");
    if (rows > 0 && (!x || !y)) return fail(QL_EINVAL, "x or y is NULL");
    if (!aligned(x, type) || !aligned(y, type) || !aligned(key, QL_F64)) return fail(QL_EINVAL, "misaligned pointer");
    const double t = std::nearbyint(std::ldexp(p, 32));
    DropoutArgs a{};
    a.x = x, a.y = y, a.key = key, a.seed = seed, a.offset = offset;
    a.rows = rows, a.D = features, a.x_stride = x_stride;
    a.none = t >= 4294967296.0, a.threshold = a.none ? 0 : (uint32_t)t, a.scale = a.none ? 0 : 1 / (1 - p);
    return launched(launch_dropout(type, a, stream), "dropout");
}

}  // extern "C"
