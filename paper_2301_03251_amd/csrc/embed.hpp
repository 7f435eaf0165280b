// embed.hpp -- embedding lookup and its gradient by sorted tokens: host-side
// launchers of embed.hip.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

#include "norm.hpp"

namespace qlayer {

struct EmbedArgs {
    const void* tokens;  // [n] of int64, or of int32
    const void* weight;  // [rows] rows of D elements, weight_stride apart (forward)
    void* y;             // [n][D] (forward)
    const void* grad;    // [n] rows, grad_stride apart (backward)
    void* grad_weight;   // [rows][D] (backward)
    int64_t n, rows, D, weight_stride, grad_stride;
    int64_t padding;  // the token of no row,
    bool padded;      // if there is one
    bool wide;        // int64 tokens
    double scale;
};

// Bytes of the backward call's workspace.
size_t embed_workspace(int type, int64_t n, int64_t rows, int64_t D);
hipError_t launch_embed_forward(int type, const EmbedArgs& a, hipStream_t s);
hipError_t launch_embed_backward(int type, const EmbedArgs& a, void* ws, hipStream_t s);

}  // namespace qlayer
