// ortho.hpp -- orthogonalised updates: host-side launchers of ortho.hip.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

#include "qlayer.h"

namespace qlayer {

// What a call does with the matrices' update U and its orthogonalised form O:
// out = O, or (muon) U from the momentum and out = keep * out - step * O.
struct OrthoCall {
    int type;             // ElemType of grad and out
    const ql_matrix* mats;
    int count;
    double a, b, c, eps;  // a X + (b A + c A^2) X, A = X X^T
    int steps;
    bool muon, nesterov;
    double momentum, keep, step;
};

// The largest |x| that any step starts from (x -> a x + b x^3 + c x^5, first from
// [0, 1]), and of the polynomial's inner factor b x^2 + c x^4. False: x grows
// past 64, or is no number.
bool ortho_bounds(double a, double b, double c, int steps, double& most_x, double& most_q);

// Whether every launch of a call stays below 2^32 threads. (What fails it has a
// workspace of more than 288 GB.)
bool ortho_launchable(int type, const ql_matrix* mats, int count);
size_t ortho_workspace(int type, const ql_matrix* mats, int count);
hipError_t launch_ortho(const OrthoCall& c, void* ws, hipStream_t s);

}  // namespace qlayer
