// norm.hpp -- layer norm over rows of features: host-side launchers of norm.hip.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

namespace qlayer {

// Element types of the operators around a quantum layer (QL_F32 ... of qlayer.h).
enum ElemType { E_F32 = 0, E_F64 = 1, E_BF16 = 2, E_F16 = 3 };

inline size_t elem_size(int t) { return t == E_F64 ? 8 : t == E_F32 ? 4 : 2; }

// Statistics, partial sums and arithmetic are fp64 for E_F64 and fp32 otherwise.
struct NormArgs {
    const void* x;       // [rows] rows of D elements, x_stride elements apart
    const void* weight;  // [D] or null: 1
    const void* bias;    // [D] or null: 0 (forward)
    void* y;             // [rows][D] (forward)
    void* mean;          // [rows] or null (forward)
    void* rstd;          // [rows] or null (forward)
    const void* grad;    // [rows] rows, grad_stride elements apart (backward)
    void* grad_x;        // [rows][D] or null (backward)
    void* grad_weight;   // [D] or null (backward)
    void* grad_bias;     // [D] or null (backward)
    void* part;          // workspace: the column sums of each workgroup,
    void* sums;          // of long rows the sums of each segment,
    void* joined;        // and of very long ones the rows' own, or null
    int64_t rows, D, x_stride, grad_stride;
    double eps;
};

// Bytes of the workspace: NormArgs::sums forward (0: none), part backward.
size_t norm_workspace(int type, int64_t rows, int64_t D, bool backward);
hipError_t launch_norm_forward(int type, int wtype, const NormArgs& a, hipStream_t s);
hipError_t launch_norm_backward(int type, int wtype, const NormArgs& a, hipStream_t s);

}  // namespace qlayer
