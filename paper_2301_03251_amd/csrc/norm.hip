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

// Rows in registers: a group of G lanes holds a row as K vectors of V elements
// per lane (vector k of lane l starts at element (k G + l) V), and takes row,
// row + stride, ...: weight and bias are read once, and the next row's loads
// are under way while a row is worked on.
template <typename T, typename W, int V, int G, int K>
__global__ __launch_bounds__(G > 256 ? G : 256) void k_norm_fwd(NormArgs a) {
    using R = Acc<T>;
    constexpr int ROWS = (G > 256 ? G : 256) / G;
    __shared__ R lds[2][G > 64 ? G / 64 : 1];
    const int lane = threadIdx.x % G;
    const R d = (R)a.D;
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / G;
    Vec<T, V> next[K];
    auto fetch = [&](int64_t r) {
        const T* xr = (const T*)a.x + r * a.x_stride;
#pragma unroll
        for (int k = 0; k < K; k++) next[k] = load_vec<T, V>(xr + Span<V>((k * G + lane) * V, (int)a.D).at);
    };
    if (row < a.rows) fetch(row);
    Vec<W, V> w[K], b[K];
#pragma unroll
    for (int k = 0; k < K; k++) {
        const Span<V> sp((k * G + lane) * V, (int)a.D);
        if (a.weight) w[k] = load_vec<W, V>((const W*)a.weight + sp.at);
        if (a.bias) b[k] = load_vec<W, V>((const W*)a.bias + sp.at);
    }
    for (; row < a.rows; row += stride) {
        Vec<T, V> x[K];
        R sum = 0;
#pragma unroll
        for (int k = 0; k < K; k++) x[k] = next[k];
        fetch(row + stride < a.rows ? row + stride : row);
#pragma unroll
        for (int k = 0; k < K; k++) {
            const Span<V> sp((k * G + lane) * V, (int)a.D);
#pragma unroll
            for (int e = 0; e < V; e++) sum += sp.own(e) ? up(x[k].v[e]) : 0;
        }
        const R mean = group_sum<G>(sum, lds[0]) / d;
        R sq = 0;
#pragma unroll
        for (int k = 0; k < K; k++) {
            renew(x[k]);
            const Span<V> sp((k * G + lane) * V, (int)a.D);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const R c = sp.own(e) ? up(x[k].v[e]) - mean : 0;
                sq += c * c;
            }
        }
        const R rstd = inv_sqrt(group_sum<G>(sq, lds[1]) / d + (R)a.eps);
        if (lane == 0) {
            if (a.mean) ((R*)a.mean)[row] = mean;
            if (a.rstd) ((R*)a.rstd)[row] = rstd;
        }
#pragma unroll
        for (int k = 0; k < K; k++) {
            const Span<V> sp((k * G + lane) * V, (int)a.D);
            if (!sp.any()) continue;
            renew(x[k]);
            Vec<T, V> q;
#pragma unroll
            for (int e = 0; e < V; e++) {
                R h = (up(x[k].v[e]) - mean) * rstd;
                if (a.weight) h *= (R)up(w[k].v[e]);
                if (a.bias) h += (R)up(b[k].v[e]);
                q.v[e] = down<T>(h);
            }
            store_vec<T, V>((T*)a.y + row * a.D + sp.at, q);
        }
    }
}

// Long rows go through the chip in segments of 256 vectors, one workgroup each,
// in two launches: every segment's mean and sum of squares about it; then each
// workgroup joins its row's (in the same order everywhere) and writes its
// segment of y. x is read twice, by as many workgroups as there are segments: no
// workgroup's registers hold such a row. That is 1.5 times the bytes where the
// array is larger than the caches; where it is not, the second read is theirs.
template <typename T> constexpr int SEGMENT = 256 * VEC<T>;

template <typename T> __global__ __launch_bounds__(256) void k_norm_fwd_sums(NormArgs a, int segments) {
    using R = Acc<T>;
    constexpr int V = VEC<T>;
    __shared__ R lds[2][4];
    R* sums = (R*)a.sums;
    for (int64_t i = blockIdx.x; i < a.rows * segments; i += gridDim.x) {
        const int64_t row = i / segments;
        const int first = (int)(i % segments) * SEGMENT<T>;
        const Span<V> sp(first + threadIdx.x * V, (int)a.D);
        const R n = (R)min(SEGMENT<T>, (int)a.D - first);
        const Vec<T, V> x = load_vec<T, V>((const T*)a.x + row * a.x_stride + sp.at);
        R sum = 0, sq = 0;
#pragma unroll
        for (int e = 0; e < V; e++) sum += sp.own(e) ? up(x.v[e]) : 0;
        const R mean = group_sum<256>(sum, lds[0]) / n;
#pragma unroll
        for (int e = 0; e < V; e++) {
            const R c = sp.own(e) ? up(x.v[e]) - mean : 0;
            sq += c * c;
        }
        sq = group_sum<256>(sq, lds[1]);
        if (threadIdx.x == 0) sums[2 * i] = mean, sums[2 * i + 1] = sq;
    }
}

// A row's mean and rstd from its segments, by a launch of its own for a very long
// row: joined again by every segment, the time of a row goes with the square of
// its length. Forward, one row of 128, 256 and 1024 segments takes 6.2, 7.3 and
// 13.4 us joined by each and 7.3, 7.3 and 9.6 joined once, 8 rows 7.7, 10.6 and 52
// against 8.9, 10.5 and 23; 2^26 float32 features took 15 ms.
constexpr int JOINED_EACH = 256;

template <typename T> __global__ __launch_bounds__(256) void k_norm_fwd_join(NormArgs a, int segments) {
    using R = Acc<T>;
    __shared__ R lds[2][4];
    const R d = (R)a.D;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const R* s = (const R*)a.sums + 2 * row * segments;
        auto count = [&](int j) { return (R)min(SEGMENT<T>, (int)a.D - j * SEGMENT<T>); };
        R t = 0;
        for (int j = threadIdx.x; j < segments; j += 256) t += s[2 * j] * count(j);
        const R mean = group_sum<256>(t, lds[0]) / d;
        t = 0;
        for (int j = threadIdx.x; j < segments; j += 256) {
            const R c = s[2 * j] - mean;
            t += s[2 * j + 1] + count(j) * c * c;
        }
        t = group_sum<256>(t, lds[1]);
        R* out = (R*)a.joined + 2 * row;
        if (threadIdx.x == 0) out[0] = mean, out[1] = inv_sqrt(t / d + (R)a.eps);
    }
}

template <typename T, typename W> __global__ __launch_bounds__(256) void k_norm_fwd_segment(NormArgs a, int segments) {
    using R = Acc<T>;
    constexpr int V = VEC<T>;
    const R d = (R)a.D;
    for (int64_t i = blockIdx.x; i < a.rows * segments; i += gridDim.x) {
        const int64_t row = i / segments;
        const int segment = (int)(i % segments);
        const Span<V> sp(segment * SEGMENT<T> + threadIdx.x * V, (int)a.D);
        const Vec<T, V> x = load_vec<T, V>((const T*)a.x + row * a.x_stride + sp.at);
        Vec<W, V> w, b;
        if (a.weight) w = load_vec<W, V>((const W*)a.weight + sp.at);
        if (a.bias) b = load_vec<W, V>((const W*)a.bias + sp.at);
        R mean, rstd;
        if (a.joined) {
            mean = ((const R*)a.joined)[2 * row], rstd = ((const R*)a.joined)[2 * row + 1];
        } else {
            const R* s = (const R*)a.sums + 2 * row * segments;
            auto count = [&](int j) { return (R)min(SEGMENT<T>, (int)a.D - j * SEGMENT<T>); };
            R t = 0;
            for (int j = threadIdx.x & 63; j < segments; j += 64) t += s[2 * j] * count(j);
            mean = lanes_sum<64>(t) / d;
            t = 0;
            for (int j = threadIdx.x & 63; j < segments; j += 64) {
                const R c = s[2 * j] - mean;
                t += s[2 * j + 1] + count(j) * c * c;
            }
            rstd = inv_sqrt(lanes_sum<64>(t) / d + (R)a.eps);
        }
        if (segment == 0 && threadIdx.x == 0) {
            if (a.mean) ((R*)a.mean)[row] = mean;
            if (a.rstd) ((R*)a.rstd)[row] = rstd;
        }
        if (!sp.any()) continue;
        Vec<T, V> q;
#pragma unroll
        for (int e = 0; e < V; e++) {
            R h = (up(x.v[e]) - mean) * rstd;
            if (a.weight) h *= (R)up(w.v[e]);
            if (a.bias) h += (R)up(b.v[e]);
            q.v[e] = down<T>(h);
        }
        store_vec<T, V>((T*)a.y + row * a.D + sp.at, q);
    }
}

// Backward of rows in registers, as k_norm_fwd: x and g are read once, and
// every lane sums its columns' g h and g over the rows that its group takes
// (row, row + stride, ...). The next row's loads are under way while a row is
// worked on. part[workgroup][2][D] gets the workgroup's sums, joined over its
// groups in LDS; a null part leaves them out. 16384x8192 bf16: 156 us (median),
// 5.2 of a copy's 5.3 TB/s (one kernel for dx and one for the columns: 310 us).
template <typename T, typename W, int V, int G, int K>
__global__ __launch_bounds__(G > 256 ? G : 256) void k_norm_bwd(NormArgs a) {
    using R = Acc<T>;
    constexpr int ROWS = (G > 256 ? G : 256) / G;
    __shared__ R lds[2][G > 64 ? G / 64 : 1];
    __shared__ R joined[ROWS > 1 ? ROWS * G * K * V : 1];
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    const R d = (R)a.D;
    Vec<W, V> w[K];
    R dw[K][V] = {}, db[K][V] = {};
#pragma unroll
    for (int k = 0; k < K; k++) {
        if (a.weight) w[k] = load_vec<W, V>((const W*)a.weight + Span<V>((k * G + lane) * V, (int)a.D).at);
        else
#pragma unroll
            for (int e = 0; e < V; e++) w[k].v[e] = down<W>((Acc<W>)1);
    }
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + group;
    Vec<T, V> x[K], g[K];
    R mean = 0, rstd = 0;
    auto fetch = [&](int64_t r) {
        mean = ((const R*)a.mean)[r], rstd = ((const R*)a.rstd)[r];
        const T *xr = (const T*)a.x + r * a.x_stride, *gr = (const T*)a.grad + r * a.grad_stride;
#pragma unroll
        for (int k = 0; k < K; k++) {
            const Span<V> sp((k * G + lane) * V, (int)a.D);
            x[k] = load_vec<T, V>(xr + sp.at);
            g[k] = load_vec<T, V>(gr + sp.at);
        }
    };
    if (row < a.rows) fetch(row);
    for (; row < a.rows; row += stride) {
        Vec<T, V> cx[K], cg[K];
        const R m = mean, r = rstd;
#pragma unroll
        for (int k = 0; k < K; k++) cx[k] = x[k], cg[k] = g[k];
        fetch(row + stride < a.rows ? row + stride : row);
        R s1 = 0, s2 = 0;
#pragma unroll
        for (int k = 0; k < K; k++) {
            const Span<V> sp((k * G + lane) * V, (int)a.D);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const R h = (up(cx[k].v[e]) - m) * r, gv = up(cg[k].v[e]);
                const R v = sp.own(e) ? gv * (R)up(w[k].v[e]) : 0;
                db[k][e] += gv;
                dw[k][e] += gv * h;
                s1 += v;
                s2 += v * h;
            }
        }
        if (!a.grad_x) continue;
        const R c1 = group_sum<G>(s1, lds[0]) / d, c2 = group_sum<G>(s2, lds[1]) / d;
#pragma unroll
        for (int k = 0; k < K; k++) {
            const Span<V> sp((k * G + lane) * V, (int)a.D);
            Vec<T, V> q;
#pragma unroll
            for (int e = 0; e < V; e++) {
                const R h = (up(cx[k].v[e]) - m) * r;
                q.v[e] = down<T>(r * (up(cg[k].v[e]) * (R)up(w[k].v[e]) - c1 - h * c2));
            }
            if (sp.any()) store_vec<T, V>((T*)a.grad_x + row * a.D + sp.at, q);
        }
    }
    if (!a.part) return;
    R* out = (R*)a.part + (int64_t)blockIdx.x * 2 * a.D;
#pragma unroll
    for (int which = 0; which < 2; which++) {
        if constexpr (ROWS > 1) __syncthreads();
#pragma unroll
        for (int k = 0; k < K; k++) {
            const Span<V> sp((k * G + lane) * V, (int)a.D);
            if (!sp.any()) continue;
            if constexpr (ROWS == 1) {
                Vec<R, V> q;
#pragma unroll
                for (int e = 0; e < V; e++) q.v[e] = which ? db[k][e] : dw[k][e];
                store_vec<R, V>(out + which * a.D + sp.at, q);
            } else {
#pragma unroll
                for (int e = 0; e < V; e++) joined[group * (G * K * V) + (int)sp.at + e] = which ? db[k][e] : dw[k][e];
            }
        }
        if constexpr (ROWS > 1) {
            __syncthreads();
            for (int i = threadIdx.x; i < G * K * V && i < a.D; i += 256) {
                R t = 0;
#pragma unroll
                for (int j = 0; j < ROWS; j++) t += joined[j * (G * K * V) + i];
                out[which * a.D + i] = t;
            }
        }
    }
}

// Longer rows take segments here too: the two sums of every segment of every
// row, then dx and the column sums, for which a workgroup keeps its segment's
// columns and takes the rows of a chunk one by one. x and g are read twice.
template <typename T, typename W> __global__ __launch_bounds__(256) void k_norm_bwd_sums(NormArgs a, int segments) {
    using R = Acc<T>;
    constexpr int V = VEC<T>;
    __shared__ R lds[2][4];
    R* sums = (R*)a.sums;
    for (int64_t i = blockIdx.x; i < a.rows * segments; i += gridDim.x) {
        const int64_t row = i / segments;
        const Span<V> sp((int)(i % segments) * SEGMENT<T> + threadIdx.x * V, (int)a.D);
        const R m = ((const R*)a.mean)[row], r = ((const R*)a.rstd)[row];
        R s1 = 0, s2 = 0;
        const Vec<T, V> x = load_vec<T, V>((const T*)a.x + row * a.x_stride + sp.at);
        const Vec<T, V> g = load_vec<T, V>((const T*)a.grad + row * a.grad_stride + sp.at);
        Vec<W, V> w;
        if (a.weight) w = load_vec<W, V>((const W*)a.weight + sp.at);
#pragma unroll
        for (int e = 0; e < V; e++) {
            R v = sp.own(e) ? up(g.v[e]) : 0;
            if (a.weight) v *= (R)up(w.v[e]);
            s1 += v;
            s2 += v * ((up(x.v[e]) - m) * r);
        }
        s1 = group_sum<256>(s1, lds[0]);
        s2 = group_sum<256>(s2, lds[1]);
        if (threadIdx.x == 0) sums[2 * i] = s1, sums[2 * i + 1] = s2;
    }
}

template <typename T> __global__ __launch_bounds__(256) void k_norm_bwd_join(NormArgs a, int segments) {
    using R = Acc<T>;
    __shared__ R lds[2][4];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const R* s = (const R*)a.sums + 2 * row * segments;
        R c1 = 0, c2 = 0;
        for (int j = threadIdx.x; j < segments; j += 256) c1 += s[2 * j], c2 += s[2 * j + 1];
        c1 = group_sum<256>(c1, lds[0]);
        c2 = group_sum<256>(c2, lds[1]);
        R* out = (R*)a.joined + 2 * row;
        if (threadIdx.x == 0) out[0] = c1 / (R)a.D, out[1] = c2 / (R)a.D;
    }
}

template <typename T, typename W>
__global__ __launch_bounds__(256) void k_norm_bwd_segment(NormArgs a, int segments, int64_t chunk_rows) {
    using R = Acc<T>;
    constexpr int V = VEC<T>;
    const Span<V> sp(blockIdx.x * SEGMENT<T> + threadIdx.x * V, (int)a.D);
    const int64_t r0 = blockIdx.y * chunk_rows, r1 = min(r0 + chunk_rows, a.rows);
    Vec<W, V> w;
    if (a.weight) w = load_vec<W, V>((const W*)a.weight + sp.at);
    R dw[V] = {}, db[V] = {};
    for (int64_t row = r0; row < r1; row++) {
        const Vec<T, V> x = load_vec<T, V>((const T*)a.x + row * a.x_stride + sp.at);
        const Vec<T, V> g = load_vec<T, V>((const T*)a.grad + row * a.grad_stride + sp.at);
        const R m = ((const R*)a.mean)[row], r = ((const R*)a.rstd)[row];
        R c1 = 0, c2 = 0;
        if (a.grad_x && a.joined) {
            c1 = ((const R*)a.joined)[2 * row], c2 = ((const R*)a.joined)[2 * row + 1];
        } else if (a.grad_x) {  // every wavefront joins the row's segments itself, in the same order
            const R* s = (const R*)a.sums + 2 * row * segments;
            for (int i = threadIdx.x & 63; i < segments; i += 64) c1 += s[2 * i], c2 += s[2 * i + 1];
            c1 = lanes_sum<64>(c1) / (R)a.D, c2 = lanes_sum<64>(c2) / (R)a.D;
        }
        Vec<T, V> q;
#pragma unroll
        for (int e = 0; e < V; e++) {
            const R h = (up(x.v[e]) - m) * r, gv = up(g.v[e]);
            db[e] += gv;
            dw[e] += gv * h;
            q.v[e] = down<T>(r * ((a.weight ? gv * (R)up(w.v[e]) : gv) - c1 - h * c2));
        }
        if (a.grad_x && sp.any()) store_vec<T, V>((T*)a.grad_x + row * a.D + sp.at, q);
    }
    if (!a.part || !sp.any()) return;
    R* out = (R*)a.part + (int64_t)blockIdx.y * 2 * a.D + sp.at;
    Vec<R, V> q;
#pragma unroll
    for (int e = 0; e < V; e++) q.v[e] = dw[e];
    store_vec<R, V>(out, q);
#pragma unroll
    for (int e = 0; e < V; e++) q.v[e] = db[e];
    store_vec<R, V>(out + a.D, q);
}

// Sum of the workgroups' column sums, in fp64: 16 columns and 16 threads for
// each, eight loads of a thread under way (4 us for 512 parts of 2x1024 columns,
// 11 us one by one). A launch's threads number less than 2^32: columns past the
// grid's go around.
constexpr int64_t REDUCE_BLOCKS = 65536;

template <typename T, typename W> __global__ __launch_bounds__(256) void k_norm_reduce(NormArgs a, int64_t chunks) {
    using R = Acc<T>;
    __shared__ double lds[16][17];
    const int c = threadIdx.x % 16, g = threadIdx.x / 16;
    for (int64_t first = (int64_t)blockIdx.x * 16; first < 2 * a.D; first += (int64_t)gridDim.x * 16) {
        const int64_t col = first + c;  // of 2 D
        double t = 0;
        if (col < 2 * a.D)
#pragma unroll 8
            for (int64_t k = g; k < chunks; k += 16) t += (double)((const R*)a.part)[k * 2 * a.D + col];
        __syncthreads();
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
}

// Segments of the forward pass; 0: rows in registers, which end at 4096 vectors.
// Where there are fewer rows than compute units, half of that is long enough
// for a second launch to pay.
int forward_segments(int type, int64_t rows, int64_t D) {
    const int64_t n = (D + 16 / (int64_t)elem_size(type) - 1) / (16 / (int64_t)elem_size(type));
    return n > 4096 || (n > 2048 && rows < 256) ? (int)((n + 255) / 256) : 0;
}

// How the backward pass is split.
struct Split {
    int lanes, per_lane;  // k_norm_bwd's G and K; lanes 0: segments
    int segments;
    int64_t parts;  // partial column sums: workgroups, or chunks of rows
    int64_t chunk_rows;
};
Split split_of(int type, int64_t rows, int64_t D) {
    const int64_t V = 16 / (int64_t)elem_size(type), n = (D + V - 1) / V;
    Split p{};
    // the column sums of a lane are 2 K V registers: K = 2 leaves room for two
    // rows of x and g at 128 to 170 registers (K = 4 took 270 for 16-bit rows)
    static const int shapes[][2] = {{16, 1}, {64, 1}, {64, 2}, {256, 1}, {256, 2}, {512, 2}, {1024, 2}};
    for (const auto& q : shapes)
        if (n <= q[0] * q[1]) {
            p.lanes = q[0], p.per_lane = q[1];
            break;
        }
    if (p.lanes) {
        // at least four rows for a group of lanes, whose column sums cost a write
        // and a read of two rows in fp32; no more workgroups than run at once
        const int64_t groups = std::max(1, 256 / p.lanes), most = p.lanes < 512 ? 512 : 256;
        p.parts = std::max<int64_t>(1, std::min(most, (rows + 4 * groups - 1) / (4 * groups)));
    } else {
        p.segments = (int)((n + 255) / 256);
        const int64_t most = std::max<int64_t>(1, 2048 / p.segments);
        p.chunk_rows = std::max<int64_t>(4, (rows + most - 1) / most);
        p.parts = std::max<int64_t>(1, (rows + p.chunk_rows - 1) / p.chunk_rows);
    }
    return p;
}
size_t part_bytes(const Split& p, int type, int64_t D) {
    const size_t b = (size_t)p.parts * 2 * (size_t)D * (type == E_F64 ? 8 : 4);
    return (b + 255) & ~(size_t)255;
}

// Bytes of the sums of a pass's segments; the joined ones lie behind them.
size_t sums_bytes(int type, int64_t rows, int segments) {
    return (size_t)(rows * segments) * 2 * (type == E_F64 ? 8 : 4);
}
size_t joined_bytes(int type, int64_t rows, int segments) {
    return segments > JOINED_EACH ? sums_bytes(type, rows, 1) : 0;
}

int grid_of(int64_t groups) { return (int)std::min<int64_t>(groups, 4096); }

template <typename T, typename W, int G, int K, int V = VEC<T>> hipError_t forward_rows(const NormArgs& a, hipStream_t s) {
    constexpr int threads = G > 256 ? G : 256, rows = threads / G;
    // many more workgroups than run at once, which leaves them out of step, but
    // few enough that each reads weight and bias for several rows: 16384x8192
    // bf16 takes 113 us (median between events; a copy of as much 102) with 4096
    // of them, 119 with 512 and 142 with one for every row
    k_norm_fwd<T, W, V, G, K><<<grid_of((a.rows + rows - 1) / rows), threads, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, typename W> hipError_t forward(int type, NormArgs a, hipStream_t s) {
    constexpr int V = VEC<T>;
    if (const int segments = forward_segments(type, a.rows, a.D)) {
        k_norm_fwd_sums<T><<<grid_of(a.rows * segments), 256, 0, s>>>(a, segments);
        if (segments > JOINED_EACH) {
            a.joined = (char*)a.sums + sums_bytes(type, a.rows, segments);
            k_norm_fwd_join<T><<<grid_of(a.rows), 256, 0, s>>>(a, segments);
        }
        k_norm_fwd_segment<T, W><<<grid_of(a.rows * segments), 256, 0, s>>>(a, segments);
        return hipGetLastError();
    }
    if (a.D < V) return forward_rows<T, W, 16, 1, 1>(a, s);
    if (a.D <= 16 * V) return forward_rows<T, W, 16, 1>(a, s);
    if (a.D <= 64 * V) return forward_rows<T, W, 64, 1>(a, s);
    if (a.D <= 128 * V) return forward_rows<T, W, 64, 2>(a, s);
    if (a.D <= 256 * V) return forward_rows<T, W, 256, 1>(a, s);
    if (a.D <= 512 * V) return forward_rows<T, W, 256, 2>(a, s);
    if (a.D <= 1024 * V) return forward_rows<T, W, 512, 2>(a, s);
    if (a.D <= 2048 * V) return forward_rows<T, W, 1024, 2>(a, s);
    return forward_rows<T, W, 1024, 4>(a, s);
}

template <typename T, typename W, int G, int K, int V = VEC<T>> hipError_t backward_rows(const NormArgs& a, const Split& p, hipStream_t s) {
    k_norm_bwd<T, W, V, G, K><<<(unsigned)p.parts, G > 256 ? G : 256, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, typename W> hipError_t backward(int type, NormArgs a, hipStream_t s) {
    const Split p = split_of(type, a.rows, (int)a.D);
    const bool columns = a.grad_weight || a.grad_bias;
    if (!columns && (!a.grad_x || a.rows == 0)) return hipSuccess;
    a.sums = (char*)a.part + part_bytes(p, type, (int)a.D);
    if (!columns) a.part = nullptr;
    hipError_t e;
    switch (p.lanes * 8 + p.per_lane) {
        case 16 * 8 + 1:
            e = a.D < VEC<T> ? backward_rows<T, W, 16, 1, 1>(a, p, s) : backward_rows<T, W, 16, 1>(a, p, s);
            break;
        case 64 * 8 + 1: e = backward_rows<T, W, 64, 1>(a, p, s); break;
        case 64 * 8 + 2: e = backward_rows<T, W, 64, 2>(a, p, s); break;
        case 256 * 8 + 1: e = backward_rows<T, W, 256, 1>(a, p, s); break;
        case 256 * 8 + 2: e = backward_rows<T, W, 256, 2>(a, p, s); break;
        case 512 * 8 + 2: e = backward_rows<T, W, 512, 2>(a, p, s); break;
        case 1024 * 8 + 2: e = backward_rows<T, W, 1024, 2>(a, p, s); break;
        default:
            if (a.grad_x && a.rows > 0) {
                k_norm_bwd_sums<T, W><<<grid_of(a.rows * p.segments), 256, 0, s>>>(a, p.segments);
                if (p.segments > JOINED_EACH) {
                    a.joined = (char*)a.sums + sums_bytes(type, a.rows, p.segments);
                    k_norm_bwd_join<T><<<grid_of(a.rows), 256, 0, s>>>(a, p.segments);
                }
            }
            k_norm_bwd_segment<T, W><<<dim3((unsigned)p.segments, (unsigned)p.parts), 256, 0, s>>>(a, p.segments, p.chunk_rows);
            e = hipGetLastError();
    }
    if (e != hipSuccess || !columns) return e;
    k_norm_reduce<T, W><<<(unsigned)std::min((2 * a.D + 15) / 16, REDUCE_BLOCKS), 256, 0, s>>>(a, p.parts);
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

size_t norm_workspace(int type, int64_t rows, int64_t D, bool backward) {
    size_t parts = 0;
    int segments = 0;
    if (backward) {
        const Split p = split_of(type, rows, D);
        parts = part_bytes(p, type, D), segments = p.segments;
    } else {
        segments = forward_segments(type, rows, D);
    }
    return parts + sums_bytes(type, rows, segments) + joined_bytes(type, rows, segments);
}

hipError_t launch_norm_forward(int type, int wtype, const NormArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return by_type(type, wtype, [&](auto t, auto w) { return forward<decltype(t), decltype(w)>(type, a, s); });
}

hipError_t launch_norm_backward(int type, int wtype, const NormArgs& a, hipStream_t s) {
    return by_type(type, wtype, [&](auto t, auto w) { return backward<decltype(t), decltype(w)>(type, a, s); });
}

}  // namespace qlayer
