// checks.hpp -- argument checks that the C entries of the operators share.
#pragma once

#include <cmath>
#include <cstdint>

#include "errors.hpp"
#include "norm.hpp"
#include "qlayer.h"

namespace qlayer {
namespace {

[[maybe_unused]] int fail(int code, const char* what, const char* detail = nullptr) {
    return set_error(code, what, detail);
}

[[maybe_unused]] bool known_type(int t) { return t >= QL_F32 && t <= QL_F16; }

// A device array's address is a multiple of its element's size (NULL is).
[[maybe_unused]] bool aligned(const void* p, int type) { return (uintptr_t)p % elem_size(type) == 0; }

// The type of statistics and states beside arrays of a type.
[[maybe_unused]] int wide_type(int type) { return type == QL_F64 ? QL_F64 : QL_F32; }

const int64_t MOST_ELEMENTS = (int64_t)1 << 46;

[[maybe_unused]] bool stride_ok(int64_t count, int64_t stride) {
    return stride >= 0 && (count <= 1 || stride <= MOST_ELEMENTS / count);
}

// A workspace of `need` bytes, if any are needed.
[[maybe_unused]] int check_workspace(const void* ws, size_t ws_bytes, size_t need) {
    if (need == 0) return QL_OK;
    if (!ws) return fail(QL_EINVAL, "workspace is NULL");
    if ((uintptr_t)ws % 16) return fail(QL_EINVAL, "misaligned workspace");
    if (ws_bytes < need) return fail(QL_ENOMEM, "workspace too small");
    return QL_OK;
}

// Rows of features, and a weight beside them.
[[maybe_unused]] int check_norm(int type, int wtype, int64_t rows, int64_t features) {
    if (!known_type(type) || !known_type(wtype)) return fail(QL_EINVAL, "unknown type");
    if (wtype != type && !(wtype == QL_F32 && (type == QL_BF16 || type == QL_F16)))
        return fail(QL_EUNSUPPORTED, "weight_type is neither the rows' type nor QL_F32 beside 16-bit rows");
    if (rows < 0) return fail(QL_EINVAL, "rows must be >= 0");
    if (features < 1 || features > 1 << 30) return fail(QL_EINVAL, "features out of range [1, 2^30]");
    if (rows > MOST_ELEMENTS / features) return fail(QL_EINVAL, "rows * features too large");
    return QL_OK;
}

}  // namespace
}  // namespace qlayer
