// elem.hpp -- device helpers of norm.hip and ortho.hip: element types, vectors
// of them at any alignment, and sums over groups of lanes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace qlayer {
namespace {

// bfloat16 as its 16 bits: the upper half of a float.
struct bf16 {
    uint16_t u;
};

// The arithmetic type of an element type.
template <typename T> struct AccOf { using type = float; };
template <> struct AccOf<double> { using type = double; };
template <typename T> using Acc = typename AccOf<T>::type;

__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ double up(double v) { return v; }
__device__ __forceinline__ float up(_Float16 v) { return (float)v; }
__device__ __forceinline__ float up(bf16 v) { return __builtin_bit_cast(float, (uint32_t)v.u << 16); }

// Rounded once, to nearest even.
template <typename T> __device__ __forceinline__ T down(Acc<T> v) { return (T)v; }
template <> __device__ __forceinline__ bf16 down<bf16>(float v) {
    return {__builtin_bit_cast(uint16_t, (__bf16)v)};
}

// V elements at an address that is aligned to one element only: global memory
// takes loads and stores of 16 bytes at any address.
template <typename T, int V> struct Vec {
    T v[V];
};
typedef uint32_t raw16_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t raw16_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t raw16_at8 __attribute__((ext_vector_type(4), aligned(8)));
template <int ALIGN> struct Raw16;
template <> struct Raw16<2> { using type = raw16_at2; };
template <> struct Raw16<4> { using type = raw16_at4; };
template <> struct Raw16<8> { using type = raw16_at8; };

template <typename T, int V> __device__ __forceinline__ Vec<T, V> load_vec(const T* p) {
    if constexpr (V == 1) {
        return {{*p}};
    } else {
        using R = typename Raw16<alignof(T)>::type;
        static_assert(sizeof(T) * V % 16 == 0, "whole loads of 16 bytes");
        struct Q {
            uint32_t w[sizeof(T) * V / 4];
        } q;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) * V / 16); i++) {
            const R r = ((const R*)p)[i];
            q.w[4 * i] = r.x, q.w[4 * i + 1] = r.y, q.w[4 * i + 2] = r.z, q.w[4 * i + 3] = r.w;
        }
        return __builtin_bit_cast(Vec<T, V>, q);
    }
}

template <typename T, int V> __device__ __forceinline__ void store_vec(T* p, const Vec<T, V>& v) {
    if constexpr (V == 1) {
        *p = v.v[0];
    } else {
        using R = typename Raw16<alignof(T)>::type;
        struct Q {
            uint32_t w[sizeof(T) * V / 4];
        };
        const Q q = __builtin_bit_cast(Q, v);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) * V / 16); i++) {
            R r;
            r.x = q.w[4 * i], r.y = q.w[4 * i + 1], r.z = q.w[4 * i + 2], r.w = q.w[4 * i + 3];
            ((R*)p)[i] = r;
        }
    }
}

// The same bits, which the compiler takes for new ones: keeps it from holding
// what it has unpacked from them in registers until the next use.
template <typename T, int V> __device__ __forceinline__ void renew(Vec<T, V>& v) {
    if constexpr (V > 1 && sizeof(T) == 2) {
        struct Q {
            uint32_t w[sizeof(T) * V / 4];
        } q = __builtin_bit_cast(Q, v);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) * V / 4); i++) asm volatile("" : "+v"(q.w[i]));
        v = __builtin_bit_cast(Vec<T, V>, q);
    }
}

// Where a lane's vector of a row of D >= V elements lies. One that would pass the
// row's end is moved back to end with it: its first `skip` elements are then
// another lane's too (V of them: the lane has none of its own). Loads and
// stores need no branch, both lanes compute the same values for them, and only
// sums leave them out.
template <int V> struct Span {
    int at, skip;
    __device__ __forceinline__ Span(int first, int D) {
        at = min(first, D - V);
        skip = min(first - at, V);
    }
    __device__ __forceinline__ bool own(int e) const { return e >= skip; }
    __device__ __forceinline__ bool any() const { return skip < V; }
};

template <int CTRL> __device__ __forceinline__ float dpp_move(float v) {
    return __builtin_bit_cast(float,
                              __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}
template <int CTRL> __device__ __forceinline__ double dpp_move(double v) {
    const long long u = __builtin_bit_cast(long long, v);
    const int lo = __builtin_amdgcn_update_dpp(0, (int)(u & 0xffffffff), CTRL, 0xF, 0xF, false);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xF, 0xF, false);
    return __builtin_bit_cast(double, ((long long)hi << 32) | (unsigned int)lo);
}

// Sum over aligned groups of N = 16 or 64 lanes; every lane gets it. Inside 16
// lanes the steps are operand modifiers (quad_perm, row_half_mirror, row_mirror).
template <int N, typename R> __device__ __forceinline__ R lanes_sum(R v) {
    v += dpp_move<0xB1>(v);
    v += dpp_move<0x4E>(v);
    v += dpp_move<0x141>(v);
    v += dpp_move<0x140>(v);
    if constexpr (N == 64) {
        v += __shfl_xor(v, 16, 64);
        v += __shfl_xor(v, 32, 64);
    }
    return v;
}

// Sum over the N lanes of a row's group: 16, 64, or a whole workgroup of N
// threads, whose wavefronts meet in `lds` (N / 64 values; a row's consecutive
// sums take different ones, see the callers).
template <int N, typename R> __device__ __forceinline__ R group_sum(R v, R* lds) {
    if constexpr (N <= 64) {
        return lanes_sum<N>(v);
    } else {
        v = lanes_sum<64>(v);
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        R t = 0;
#pragma unroll
        for (int i = 0; i < N / 64; i++) t += lds[i];
        return t;
    }
}

}  // namespace
}  // namespace qlayer
