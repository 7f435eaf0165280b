// rms.hpp -- root-mean-square norm of rows with the residual's addition:
// host-side launchers of rms.hip.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

#include "norm.hpp"

namespace qlayer {

// Statistics, partial sums and arithmetic are fp64 for E_F64 and fp32 otherwise.
struct RmsArgs {
    const void* x;         // [rows] rows of D elements, x_stride elements apart (backward: the sum's)
    const void* residual;  // [rows] rows, residual_stride apart, or null: none (forward)
    const void* weight;    // [D] or null: 1
    void* summed;          // [rows][D]: x + residual, with a residual (forward)
    void* y;               // [rows][D], or of bytes where quantized (forward)
    void* rstd;            // [rows] or null (forward); [rows] (backward)
    float* scale;          // [rows] where quantized, else null (forward)
    const void* grad;      // [rows] rows, grad_stride apart (backward)
    const void* grad_sum;  // [rows] rows, grad_sum_stride apart, or null: 0 (backward)
    void* grad_x;          // [rows][D] or null (backward)
    void* grad_weight;     // [D] or null (backward)
    void* part;            // workspace: the column sums of each workgroup (backward),
    void* sums;            // of long rows the sums (forward also the largest) of each segment,
    void* joined;          // and of each row
    int64_t rows, D, x_stride, residual_stride, grad_stride, grad_sum_stride;
    double eps;
};

// Bytes of the workspace: RmsArgs::sums forward (0: none), part backward.
size_t rms_workspace(int type, int64_t rows, int64_t D, bool backward);
hipError_t launch_rms_forward(int type, int wtype, const RmsArgs& a, void* ws, hipStream_t s);
hipError_t launch_rms_backward(int type, int wtype, const RmsArgs& a, void* ws, hipStream_t s);

}  // namespace qlayer
