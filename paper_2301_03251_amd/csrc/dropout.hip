// dropout.hip -- dropout whose mask is computed where it is needed, forward and
// (the same map of the gradient) backward.
//
//   y_i = x_i / (1 - p)  where word(i) >= p 2^32,  0 elsewhere
//
// word(i) is word i mod 4 of Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and
// Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011) of the counter (i / 4,
// offset) under the key `seed`, i the element's place in row-major order: it
// depends on nothing else, so no mask is stored and any split of the work draws
// the same one. Ten rounds of two products of 32 x 32 bits make four words: 5
// products an element, beside its 4 to 8 bytes read and written.
#include <algorithm>

#include "dropout.hpp"
#include "elem.hpp"

namespace qlayer {
namespace {

__device__ __forceinline__ void philox(uint64_t counter, uint64_t offset, uint64_t seed, uint32_t (&out)[4]) {
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; r++) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0, out[1] = c1, out[2] = c2, out[3] = c3;
}

// Elements of a thread's step: whole generator blocks and whole loads.
template <typename T> constexpr int STEP = sizeof(T) == 2 ? 8 : 4;

// FLAT: the rows lie one behind the other, and the array is one row.
template <typename T, bool FLAT> __global__ __launch_bounds__(256) void k_dropout(DropoutArgs a) {
    using R = Acc<T>;
    constexpr int E = STEP<T>;
    const uint64_t seed = a.key ? a.key[0] : a.seed, offset = a.key ? a.key[1] : a.offset;
    const R scale = (R)a.scale;
    const int64_t n = a.rows * a.D, steps = (n + E - 1) / E;
    const bool whole = FLAT || a.D % E == 0;  // no step passes a row's end
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < steps; i += (int64_t)gridDim.x * 256) {
        const int64_t first = i * E;
        int64_t row = 0, col = first;
        if constexpr (!FLAT) row = first / a.D, col = first % a.D;
        const T* src = (const T*)a.x + row * a.x_stride + col;
        T* dst = (T*)a.y + first;
        const int count = (int)min((int64_t)E, n - first);
        Vec<T, E> x;
        if (whole && count == E) {
            x = load_vec<T, E>(src);
        } else {
#pragma unroll
            for (int e = 0; e < E; e++) {
                if (e >= count) break;
                x.v[e] = *src++;
                if (!FLAT && ++col == a.D) col = 0, src += a.x_stride - a.D;
            }
        }
        uint32_t words[E];
#pragma unroll
        for (int b = 0; b < E / 4; b++) {
            uint32_t w[4];
            philox((uint64_t)(first / 4 + b), offset, seed, w);
#pragma unroll
            for (int e = 0; e < 4; e++) words[4 * b + e] = w[e];
        }
        // chosen, not multiplied: what is dropped is 0 whatever it held
        Vec<T, E> y;
#pragma unroll
        for (int e = 0; e < E; e++)
            y.v[e] = down<T>(words[e] >= a.threshold && !a.none ? up(x.v[e]) * scale : (R)0);
        if (count == E) {
            store_vec<T, E>(dst, y);
        } else {
#pragma unroll
            for (int e = 0; e < E; e++)
                if (e < count) dst[e] = y.v[e];
        }
    }
}

template <typename T> hipError_t dropout(DropoutArgs a, hipStream_t s) {
    const int64_t steps = (a.rows * a.D + STEP<T> - 1) / STEP<T>;
    const int grid = (int)std::min<int64_t>((steps + 255) / 256, 1 << 20);
    if (a.rows == 1 || a.x_stride == a.D) k_dropout<T, true><<<grid, 256, 0, s>>>(a);
    else k_dropout<T, false><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int type, const DropoutArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    switch (type) {
        case E_F64: return dropout<double>(a, s);
        case E_BF16: return dropout<bf16>(a, s);
        case E_F16: return dropout<_Float16>(a, s);
        default: return dropout<float>(a, s);
    }
}

}  // namespace qlayer
