// scan.hpp -- gated linear recurrence over long sequences: host-side launchers
// of scan.hip.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

#include "norm.hpp"

namespace qlayer {

// A [batch][steps][D] array whose sequences and steps lie these many elements apart.
struct Strided {
    void* p;
    int64_t batch, step;
};

// States are fp64 for E_F64 and fp32 otherwise.
struct ScanArgs {
    Strided x, gate;
    Strided grad;           // of h (backward)
    const uint8_t* starts;  // [batch][steps]: not 0 where a sequence begins, or null
    const void* initial;    // [batch][D] or null: 0 (forward)
    void* h;                // [batch][steps][D] (forward)
    void* last;             // [batch][D] or null (forward)
    void* states;           // [batch][blocks][D]: the state before each block of steps, or null (forward); (backward)
    const void* grad_last;  // [batch][D] or null: 0 (backward)
    void* grad_x;           // [batch][steps][D] (backward)
    void* grad_gate;        // [batch][steps][D] (backward)
    void* grad_initial;     // [batch][D] or null (backward)
    void* ws;
    int64_t batch, steps, D;
};

// Steps of a block, before each of which the forward call keeps the state.
constexpr int SCAN_BLOCK = 16;

// Bytes of the workspace of a forward or backward call.
size_t scan_workspace(int type, int64_t batch, int64_t steps, int64_t D);
hipError_t launch_scan_forward(int type, const ScanArgs& a, hipStream_t s);
hipError_t launch_scan_backward(int type, const ScanArgs& a, hipStream_t s);
// One step: state [batch][D] in place; x.step and gate.step are not used, starts [batch].
hipError_t launch_scan_step(int type, const ScanArgs& a, void* state, hipStream_t s);

}  // namespace qlayer
