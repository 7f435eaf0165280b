// dropout.hpp -- dropout by a counter-based generator: host-side launcher of
// dropout.hip.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "norm.hpp"

namespace qlayer {

struct DropoutArgs {
    const void* x;        // [rows] rows of D elements, x_stride elements apart
    void* y;              // [rows][D]
    const uint64_t* key;  // seed and offset on the device, or null: those below
    uint64_t seed, offset;
    int64_t rows, D, x_stride;
    uint32_t threshold;  // words below it drop their element,
    bool none;           // or every one does
    double scale;        // of what is kept
};

hipError_t launch_dropout(int type, const DropoutArgs& a, hipStream_t s);

}  // namespace qlayer
