// norm.hip -- layer norm over rows of D features, forward and backward.
//
//   m = sum x / D,  v = sum (x - m)^2 / D,  r = 1 / sqrt(v + eps),  h = (x - m) r
//   y = h w + b
//   dx = r (g w - mean(g w) - h mean(g w h)),  dw = sum_rows g h,  db = sum_rows g
//
// About 8 operations per element of 2 to 8 bytes: HBM bounds every case but the
// smallest, which are bound by the launch. So x (and g) is read once: a row
// stays in the registers of its group of lanes (16 lanes, a wavefront or a
// workgroup, by its length) between the sums and the output. The variance is
// the sum of squares about the mean, taken from the registers: x^2 is never
// summed, so an offset of the features costs no precision.
#include <algorithm>
#include <type_traits>

#include "elem.hpp"
#include "norm.hpp"

namespace qlayer {
namespace {

template <typename T> constexpr int VEC = 16 / (int)sizeof(T);

__device__ __forceinline__ float inv_sqrt(float v) { return 1.0f / sqrtf(v); }
__device__ __forceinline__ double inv_sqrt(double v) { return 1.0 / sqrt(v); }

// Rows in registers: a group of G lanes holds a row as K vectors per lane
// (vector k of lane l starts at element (k G + l) V). Lanes past the row's end
// hold zeros, and after the mean is known the mean, so that they add nothing.
template <typename T, typename W, int G, int K>
__global__ __launch_bounds__(G > 256 ? G : 256) void k_norm_fwd(NormArgs a) {
    using R = Acc<T>;
    constexpr int V = VEC<T>, ROWS = (G > 256 ? G : 256) / G;
    __shared__ R lds[2][G > 64 ? G / 64 : 1];
    const int lane = threadIdx.x % G;
    const R d = (R)a.D;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / G; row < a.rows; row += (int64_t)gridDim.x * ROWS) {
        const T* xr = (const T*)a.x + row * a.x_stride;
        T* yr = (T*)a.y + row * a.D;
        R x[K][V];
        R sum = 0;
#pragma unroll
        for (int k = 0; k < K; k++) {
            const int64_t at = (int64_t)(k * G + lane) * V;
            const Vec<T, V> q = load_some<T, V>(xr + at, a.D - at);
#pragma unroll
            for (int e = 0; e < V; e++) sum += x[k][e] = up(q.v[e]);
        }
        const R mean = group_sum<G>(sum, lds[0]) / d;
        R sq = 0;
#pragma unroll
        for (int k = 0; k < K; k++) {
            const int64_t left = a.D - (int64_t)(k * G + lane) * V;
#pragma unroll
            for (int e = 0; e < V; e++) {
                x[k][e] -= mean;
                if (left < V && e >= left) x[k][e] = 0;
                sq += x[k][e] * x[k][e];
            }
        }
        const R rstd = inv_sqrt(group_sum<G>(sq, lds[1]) / d + (R)a.eps);
        if (lane == 0) {
            if (a.mean) ((R*)a.mean)[row] = mean;
            if (a.rstd) ((R*)a.rstd)[row] = rstd;
        }
#pragma unroll
        for (int k = 0; k < K; k++) {
            const int64_t at = (int64_t)(k * G + lane) * V, left = a.D - at;
            if (left <= 0) continue;
            Vec<W, V> w, b;
            if (a.weight) w = load_some<W, V>((const W*)a.weight + at, left);
            if (a.bias) b = load_some<W, V>((const W*)a.bias + at, left);
            Vec<T, V> q;
#pragma unroll
            for (int e = 0; e < V; e++) {
                R h = x[k][e] * rstd;
                if (a.weight) h *= (R)up(w.v[e]);
                if (a.bias) h += (R)up(b.v[e]);
                q.v[e] = down<T>(h);
            }
            store_some<T, V>(yr + at, q, left);
        }
    }
}

// Rows longer than the registers of a workgroup hold: read once for each sum
// and once for the output.
template <typename T, typename W> __global__ __launch_bounds__(1024) void k_norm_fwd_long(NormArgs a) {
    using R = Acc<T>;
    constexpr int V = VEC<T>;
    __shared__ R lds[2][16];
    const R d = (R)a.D;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* xr = (const T*)a.x + row * a.x_stride;
        T* yr = (T*)a.y + row * a.D;
        R sum = 0;
        for (int64_t at = threadIdx.x * V; at < a.D; at += 1024 * V) {
            const Vec<T, V> q = load_some<T, V>(xr + at, a.D - at);
#pragma unroll
            for (int e = 0; e < V; e++) sum += up(q.v[e]);
        }
        const R mean = group_sum<1024>(sum, lds[0]) / d;
        R sq = 0;
        for (int64_t at = threadIdx.x * V; at < a.D; at += 1024 * V) {
            const Vec<T, V> q = load_some<T, V>(xr + at, a.D - at);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const R c = up(q.v[e]) - mean;
                if (at + e < a.D) sq += c * c;
            }
        }
        const R rstd = inv_sqrt(group_sum<1024>(sq, lds[1]) / d + (R)a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) ((R*)a.mean)[row] = mean;
            if (a.rstd) ((R*)a.rstd)[row] = rstd;
        }
        for (int64_t at = threadIdx.x * V; at < a.D; at += 1024 * V) {
            const int64_t left = a.D - at;
            const Vec<T, V> p = load_some<T, V>(xr + at, left);
            Vec<W, V> w, b;
            if (a.weight) w = load_some<W, V>((const W*)a.weight + at, left);
            if (a.bias) b = load_some<W, V>((const W*)a.bias + at, left);
            Vec<T, V> q;
#pragma unroll
            for (int e = 0; e < V; e++) {
                R h = (up(p.v[e]) - mean) * rstd;
                if (a.weight) h *= (R)up(w.v[e]);
                if (a.bias) h += (R)up(b.v[e]);
                q.v[e] = down<T>(h);
            }
            store_some<T, V>(yr + at, q, left);
        }
    }
}

// dx of rows of any length; a row's second read comes from the caches.
template <typename T, typename W, int G> __global__ __launch_bounds__(G > 256 ? G : 256) void k_norm_dx(NormArgs a) {
    using R = Acc<T>;
    constexpr int V = VEC<T>, ROWS = (G > 256 ? G : 256) / G;
    __shared__ R lds[2][G > 64 ? G / 64 : 1];
    const int lane = threadIdx.x % G;
    const R d = (R)a.D;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / G; row < a.rows; row += (int64_t)gridDim.x * ROWS) {
        const T* xr = (const T*)a.x + row * a.x_stride;
        const T* gr = (const T*)a.grad + row * a.grad_stride;
        const R mean = ((const R*)a.mean)[row], rstd = ((const R*)a.rstd)[row];
        R s1 = 0, s2 = 0;
        for (int64_t at = lane * V; at < a.D; at += G * V) {
            const int64_t left = a.D - at;
            const Vec<T, V> x = load_some<T, V>(xr + at, left), g = load_some<T, V>(gr + at, left);
            Vec<W, V> w;
            if (a.weight) w = load_some<W, V>((const W*)a.weight + at, left);
#pragma unroll
            for (int e = 0; e < V; e++) {
                R h = up(g.v[e]);
                if (a.weight) h *= (R)up(w.v[e]);
                if (e < left) s1 += h, s2 += h * ((up(x.v[e]) - mean) * rstd);
            }
        }
        const R c1 = group_sum<G>(s1, lds[0]) / d, c2 = group_sum<G>(s2, lds[1]) / d;
        for (int64_t at = lane * V; at < a.D; at += G * V) {
            const int64_t left = a.D - at;
            const Vec<T, V> x = load_some<T, V>(xr + at, left), g = load_some<T, V>(gr + at, left);
            Vec<W, V> w;
            if (a.weight) w = load_some<W, V>((const W*)a.weight + at, left);
            Vec<T, V> q;
#pragma unroll
            for (int e = 0; e < V; e++) {
                R h = up(g.v[e]);
                if (a.weight) h *= (R)up(w.v[e]);
                q.v[e] = down<T>(rstd * (h - c1 - (up(x.v[e]) - mean) * rstd * c2));
            }
            store_some<T, V>((T*)a.grad_x + row * a.D + at, q, left);
        }
    }
}

// Column sums of a chunk of rows: lanes side by side on the columns, the
// workgroup's row groups joined in LDS. part[chunk][2][D]: g h, then g.
template <typename T> __global__ __launch_bounds__(256) void k_norm_columns(NormArgs a, int lanes, int64_t chunk_rows) {
    using R = Acc<T>;
    constexpr int V = VEC<T>;
    __shared__ R lds[256 * V];
    const int lane = threadIdx.x % lanes, group = threadIdx.x / lanes, groups = 256 / lanes;
    const int64_t at = ((int64_t)blockIdx.x * lanes + lane) * V, left = a.D - at;
    const int64_t r0 = blockIdx.y * chunk_rows, r1 = min(r0 + chunk_rows, a.rows);
    R dw[V] = {}, db[V] = {};
    if (left > 0)
        for (int64_t row = r0 + group; row < r1; row += groups) {
            const Vec<T, V> x = load_some<T, V>((const T*)a.x + row * a.x_stride + at, left);
            const Vec<T, V> g = load_some<T, V>((const T*)a.grad + row * a.grad_stride + at, left);
            const R mean = ((const R*)a.mean)[row], rstd = ((const R*)a.rstd)[row];
#pragma unroll
            for (int e = 0; e < V; e++) {
                const R v = up(g.v[e]);
                db[e] += v;
                dw[e] += v * ((up(x.v[e]) - mean) * rstd);
            }
        }
    R* out = (R*)a.part + (int64_t)blockIdx.y * 2 * a.D;
    for (int k = 0; k < 2; k++) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; e++) lds[threadIdx.x * V + e] = k ? db[e] : dw[e];
        __syncthreads();
        for (int i = threadIdx.x; i < lanes * V; i += 256) {
            const int64_t col = (int64_t)blockIdx.x * lanes * V + i;
            if (col >= a.D) break;
            R t = 0;
            for (int g = 0; g < groups; g++) t += lds[g * lanes * V + i];
            out[k * a.D + col] = t;
        }
    }
}

// Sum of the chunks' column sums, in fp64: 16 columns and 16 threads for each.
template <typename T, typename W> __global__ __launch_bounds__(256) void k_norm_reduce(NormArgs a, int64_t chunks) {
    using R = Acc<T>;
    __shared__ double lds[16][17];
    const int c = threadIdx.x % 16, g = threadIdx.x / 16;
    const int64_t col = (int64_t)blockIdx.x * 16 + c;  // of 2 D
    double t = 0;
    if (col < 2 * a.D)
        for (int64_t k = g; k < chunks; k += 16) t += (double)((const R*)a.part)[k * 2 * a.D + col];
    lds[g][c] = t;
    __syncthreads();
    if (g == 0 && col < 2 * a.D) {
        t = 0;
#pragma unroll
        for (int i = 0; i < 16; i++) t += lds[i][c];
        W* out = (W*)(col < a.D ? a.grad_weight : a.grad_bias);
        if (out) out[col < a.D ? col : col - a.D] = down<W>((Acc<W>)t);
    }
}

// Chunks of rows of the column sums: enough workgroups for the chip, and at
// least 16 rows for each row group.
struct Columns {
    int lanes;
    int64_t blocks, chunks, chunk_rows;
};
Columns columns_of(int type, int64_t rows, int64_t D) {
    const int64_t V = 16 / (int64_t)elem_size(type), need = (D + V - 1) / V;
    Columns c;
    c.lanes = 1;
    while (c.lanes < 64 && c.lanes < need) c.lanes *= 2;
    c.blocks = (need + c.lanes - 1) / c.lanes;
    const int64_t most = std::max<int64_t>(1, 1024 / c.blocks), least_rows = 16 * (256 / c.lanes);
    c.chunks = std::max<int64_t>(1, std::min(most, (rows + least_rows - 1) / least_rows));
    c.chunk_rows = std::max<int64_t>(1, (rows + c.chunks - 1) / c.chunks);
    c.chunks = std::max<int64_t>(1, (rows + c.chunk_rows - 1) / c.chunk_rows);
    return c;
}

int grid_of(int64_t groups) { return (int)std::min<int64_t>(groups, 4096); }

template <typename T, typename W, int G, int K> hipError_t forward_rows(const NormArgs& a, hipStream_t s) {
    constexpr int threads = G > 256 ? G : 256, rows = threads / G;
    k_norm_fwd<T, W, G, K><<<grid_of((a.rows + rows - 1) / rows), threads, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, typename W> hipError_t forward(const NormArgs& a, hipStream_t s) {
    constexpr int V = VEC<T>;
    if (a.D <= 16 * V) return forward_rows<T, W, 16, 1>(a, s);
    if (a.D <= 64 * V) return forward_rows<T, W, 64, 1>(a, s);
    if (a.D <= 128 * V) return forward_rows<T, W, 64, 2>(a, s);
    if (a.D <= 256 * V) return forward_rows<T, W, 64, 4>(a, s);
    if (a.D <= 512 * V) return forward_rows<T, W, 256, 2>(a, s);
    if (a.D <= 1024 * V) return forward_rows<T, W, 256, 4>(a, s);
    if (a.D <= 2048 * V) return forward_rows<T, W, 1024, 2>(a, s);
    if (a.D <= 4096 * V) return forward_rows<T, W, 1024, 4>(a, s);
    k_norm_fwd_long<T, W><<<grid_of(a.rows), 1024, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, typename W> hipError_t backward(int type, const NormArgs& a, hipStream_t s) {
    constexpr int V = VEC<T>;
    if (a.grad_x && a.rows > 0) {
        if (a.D <= 16 * V) k_norm_dx<T, W, 16><<<grid_of((a.rows + 15) / 16), 256, 0, s>>>(a);
        else if (a.D <= 256 * V) k_norm_dx<T, W, 64><<<grid_of((a.rows + 3) / 4), 256, 0, s>>>(a);
        else k_norm_dx<T, W, 256><<<grid_of(a.rows), 256, 0, s>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (!a.grad_weight && !a.grad_bias) return hipSuccess;
    const Columns c = columns_of(type, a.rows, a.D);
    k_norm_columns<T><<<dim3((unsigned)c.blocks, (unsigned)c.chunks), 256, 0, s>>>(a, c.lanes, c.chunk_rows);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    k_norm_reduce<T, W><<<(unsigned)((2 * a.D + 15) / 16), 256, 0, s>>>(a, c.chunks);
    return hipGetLastError();
}

// f(T, W) for the element types of x and of the weight.
template <typename F> hipError_t by_type(int type, int wtype, F f) {
    switch (type) {
        case E_F64: return f(double{}, double{});
        case E_BF16: return wtype == E_F32 ? f(bf16{}, float{}) : f(bf16{}, bf16{});
        case E_F16: return wtype == E_F32 ? f(_Float16{}, float{}) : f(_Float16{}, _Float16{});
        default: return f(float{}, float{});
    }
}

}  // namespace

size_t norm_workspace(int type, int64_t rows, int64_t D) {
    return (size_t)columns_of(type, rows, D).chunks * 2 * (size_t)D * (type == E_F64 ? 8 : 4);
}

hipError_t launch_norm_forward(int type, int wtype, const NormArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return by_type(type, wtype, [&](auto t, auto w) { return forward<decltype(t), decltype(w)>(a, s); });
}

hipError_t launch_norm_backward(int type, int wtype, const NormArgs& a, hipStream_t s) {
    return by_type(type, wtype, [&](auto t, auto w) { return backward<decltype(t), decltype(w)>(type, a, s); });
}

}  // namespace qlayer
