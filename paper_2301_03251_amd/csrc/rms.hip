// rms.hip -- the residual's addition and the root-mean-square norm of the sum,
// over rows of D features, forward, backward and with an output in 8 bits.
//
//   s = x + residual (rounded to its type),  r = 1 / sqrt(sum s^2 / D + eps)
//   h = s r,  y = h w
//   ds = r (g w - h mean(g w h)) + gs,  dw = sum_rows g h
//   q = e4m3(y / scale),  scale = max |y| / 448
//
// The norm is of the rounded sum, which is what a network goes on with and what
// the backward pass reads. Some 6 operations per element of 2 to 8 bytes: HBM bounds every
// case but the smallest, which are bound by the launch. So every array is read
// once: a row stays in the registers of its group of lanes (16 lanes, a
// wavefront or a workgroup, by its length) between the sum and the output. In 8
// bits the row's largest |s w| comes from the same step as its sum of squares,
// and r drops out of y / scale = s w 448 / max |s w|.
#include <algorithm>

#include "elem.hpp"
#include "rms.hpp"

namespace qlayer {
namespace {

template <typename T> constexpr int VEC = 16 / (int)sizeof(T);

__device__ __forceinline__ float inv_sqrt(float v) { return 1.0f / sqrtf(v); }
__device__ __forceinline__ double inv_sqrt(double v) { return 1.0 / sqrt(v); }

constexpr float MOST_E4M3 = 448;

// A row's values in [-448, 448]: p 448 / most of p = s w, most = max |p|. A product by 448 /
// most in fp32 is off by 2^-23 and takes one in seven of the quotients that lie
// half-way between two e4m3 values (4e-4 of bfloat16's) to the wrong one. So the factor
// is the next fp32 number up, and the last two bits of the product go. The factor is 0 to
// 3 2^-24 of itself too large; a quotient of five bits (a half) then comes out less than
// four steps up, which the two bits take back, and goes to the even value. For bfloat16
// rows and weights, whose p and most have 16 bits, any other quotient is at least 2^-20.95
// of itself away from a half and stays on its side. (16384x8192 bfloat16 without a
// residual: 77 us, 74 without this, 80 with the remainder of a division, 94 in fp64.)
// Rows whose p may have lost bits, or is past fp32, and those with infinities are done in
// fp64, behind the others (16384x8192, half of the rows at 1e-35: 187 us).
__device__ __forceinline__ bool in_fp32(float most) { return most >= 0x1p-100f && most <= 0x1p127f; }

struct Narrow {
    float factor;
    __device__ __forceinline__ explicit Narrow(float most)
        : factor(most > 0 ? __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, MOST_E4M3 / most) + 1) : 0) {}
    __device__ __forceinline__ float operator()(float p) const {
        return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, p * factor) & ~3u);
    }
};
struct Wide {
    double factor;
    __device__ __forceinline__ explicit Wide(double most) : factor(most > 0 ? MOST_E4M3 / most : 0) {}
    __device__ __forceinline__ float operator()(double p) const { return (float)(p * factor); }
};
// The scales beside them. A row of zeros has 0 also where eps is 0 and rstd infinite; NaN stays.
__device__ __forceinline__ float scale_of(float rstd, float most) {
    return most > 0 ? rstd * (most / MOST_E4M3) : 0;
}
__device__ __forceinline__ float scale_of(float rstd, double most) {
    return most > 0 || rstd != rstd ? (float)((double)rstd * most / MOST_E4M3) : 0;
}

// Four values in e4m3, rounded to nearest even; NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

template <int V> __device__ __forceinline__ void store_e4m3(uint8_t* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = (uint8_t)(e4m3x4(v[0], 0, 0, 0) & 0xFF);
    } else if constexpr (V == 4) {
        typedef uint32_t word __attribute__((aligned(1)));
        *(word*)p = e4m3x4(v[0], v[1], v[2], v[3]);
    } else {
        typedef uint32_t pair __attribute__((ext_vector_type(2), aligned(1)));
        pair q;
        q.x = e4m3x4(v[0], v[1], v[2], v[3]);
        q.y = e4m3x4(v[4], v[5], v[6], v[7]);
        *(pair*)p = q;
    }
}

// Infinity if one of the elements is, else m.
template <typename T, int V, typename R> __device__ __forceinline__ R infinity_or(const Vec<T, V>& s, R m) {
    bool any = false;
#pragma unroll
    for (int e = 0; e < V; e++) any |= fabsf(up(s.v[e])) == INFINITY;
    return any ? (R)INFINITY : m;
}

// A row of k_rms_fwd in fp64. The lanes read their elements again.
template <typename T, typename W, int V, int G, int K>
__device__ __forceinline__ void wide_row(const RmsArgs& a, int64_t row, int lane, float rstd, double* lds) {
    const T* s = a.residual ? (const T*)a.summed + row * a.D : (const T*)a.x + row * a.x_stride;
    auto each = [&](auto f) {
#pragma unroll 1
        for (int k = 0; k < K; k++) {
            const Span<V> sp((k * G + lane) * V, (int)a.D);
            if (!sp.any()) break;
            const Vec<T, V> v = load_vec<T, V>(s + sp.at);
            Vec<W, V> w;
            if (a.weight) w = load_vec<W, V>((const W*)a.weight + sp.at);
            f(sp.at, v, w);
        }
    };
    auto product = [&](const Vec<T, V>& v, const Vec<W, V>& w, int e) {
        return (double)up(v.v[e]) * (a.weight ? (double)up(w.v[e]) : 1);
    };
    double most = 0;
    each([&](int, auto& v, auto& w) {
#pragma unroll
        for (int e = 0; e < V; e++) most = larger(most, fabs(product(v, w, e)));
        most = infinity_or(v, most);
    });
    most = group_max<G>(most, lds);
    if (lane == 0) a.scale[row] = scale_of(rstd, most);
    const Wide quotient(most);
    each([&](int at, auto& v, auto& w) {
        float q[V];
#pragma unroll
        for (int e = 0; e < V; e++) q[e] = quotient(product(v, w, e));
        store_e4m3<V>((uint8_t*)a.y + row * a.D + at, q);
    });
}

// Rows in registers: a group of G lanes holds a row as K vectors of V elements
// per lane (vector k of lane l starts at element (k G + l) V), and takes row,
// row + stride, ...: the weight is read once, and the next row's loads are under
// way while a row is worked on. In 8 bits with K = 2 the registers are held to six
// wavefronts a SIMD: 16384x8192 bfloat16 with float32 weights 80 us, 87 with five.
template <typename T, typename W, int V, int G, int K, bool Q>
__global__ __launch_bounds__(G > 256 ? G : 256, Q && K == 2 ? 6 : 1) void k_rms_fwd(RmsArgs a) {
    using R = Acc<T>;
    constexpr int ROWS = (G > 256 ? G : 256) / G;
    __shared__ R lds[2][2][G > 64 ? G / 64 : 1];
    __shared__ double lds_wide[Q && G > 64 ? G / 64 : 1];
    const int lane = threadIdx.x % G, D = (int)a.D;
    const R d = (R)a.D;
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / G;
    Vec<T, V> nx[K], nr[K];
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < K; k++) {
            const int at = Span<V>((k * G + lane) * V, D).at;
            nx[k] = load_vec<T, V>((const T*)a.x + r * a.x_stride + at);
            if (a.residual) nr[k] = load_vec<T, V>((const T*)a.residual + r * a.residual_stride + at);
        }
    };
    if (row < a.rows) fetch(row);
    Vec<W, V> w[K];
#pragma unroll
    for (int k = 0; k < K; k++) {
        if (a.weight) w[k] = load_vec<W, V>((const W*)a.weight + Span<V>((k * G + lane) * V, D).at);
    }
    bool waiting = false;  // the same for all of a row's lanes
    for (int turn = 0; row < a.rows; row += stride, turn ^= 1) {
        Vec<T, V> s[K];
#pragma unroll
        for (int k = 0; k < K; k++) {
            s[k] = nx[k];
            if (a.residual) {
#pragma unroll
                for (int e = 0; e < V; e++) s[k].v[e] = down<T>(up(nx[k].v[e]) + up(nr[k].v[e]));
            }
        }
        fetch(row + stride < a.rows ? row + stride : row);
        R sum = 0, most = 0;
#pragma unroll
        for (int k = 0; k < K; k++) {
            const Span<V> sp((k * G + lane) * V, D);
            if (a.residual && sp.any()) store_vec<T, V>((T*)a.summed + row * a.D + sp.at, s[k]);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const R v = up(s[k].v[e]);
                sum += sp.own(e) ? v * v : 0;
                if constexpr (Q) most = larger(most, fabsf(a.weight ? v * (R)up(w[k].v[e]) : v));
            }
        }
        // the turns' LDS values alternate: a wavefront that is a row ahead has
        // passed this row's barrier, but another may still read its values
        if constexpr (Q) group_sum_max<G>(sum, most, lds[turn][0], lds[turn][1]);
        else sum = group_sum<G>(sum, lds[turn][0]);
        const R rstd = inv_sqrt(sum / d + (R)a.eps);
        // Rows for fp64 wait until the others are done, their scale -rstd so far, and those that
        // may hold an infinity (under a weight of 0 no product tells). Rows of zeros
        // need not: no product is above 2^-150, and where 1 / rms is at most 2^10 the
        // scale is below 2^-148, two of fp32's least steps.
        const bool narrow = sum < (R)INFINITY && (in_fp32(most) || (most == 0 && sum >= d * (R)(0x1p-20 - a.eps)));
        if (lane == 0) {
            if (a.rstd) ((R*)a.rstd)[row] = rstd;
            if constexpr (Q) a.scale[row] = narrow ? scale_of(rstd, most) : -rstd;
        }
        if constexpr (Q) {
            waiting |= !narrow;
            const Narrow quotient(most);
#pragma unroll
            for (int k = 0; k < K; k++) {
                const Span<V> sp((k * G + lane) * V, D);
                if (!sp.any()) continue;
                renew(s[k]);
                if constexpr (K > 1) renew(w[k]);  // unpacked, 4 vectors of them do not fit: 54 us for 120 at 1000x32768
                float q[V];
#pragma unroll
                for (int e = 0; e < V; e++) q[e] = quotient(a.weight ? up(s[k].v[e]) * (float)up(w[k].v[e]) : up(s[k].v[e]));
                store_e4m3<V>((uint8_t*)a.y + row * a.D + sp.at, q);
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; k++) {
                const Span<V> sp((k * G + lane) * V, D);
                if (!sp.any()) continue;
                renew(s[k]);
                Vec<T, V> q;
#pragma unroll
                for (int e = 0; e < V; e++) {
                    R h = up(s[k].v[e]) * rstd;
                    if (a.weight) h *= (R)up(w[k].v[e]);
                    q.v[e] = down<T>(h);
                }
                store_vec<T, V>((T*)a.y + row * a.D + sp.at, q);
            }
        }
    }
    if constexpr (Q) {
        if (!waiting) return;
        if constexpr (G > 64) __syncthreads();
        else __threadfence_block();
        for (row = (int64_t)blockIdx.x * ROWS + threadIdx.x / G; row < a.rows; row += stride) {
            const float mark = a.scale[row];
            if (!(__builtin_bit_cast(uint32_t, mark) >> 31)) continue;
            if constexpr (G > 64) __syncthreads();  // the row before has been read from lds_wide
            wide_row<T, W, V, G, K>(a, row, lane, -mark, lds_wide);
        }
    }
}

// Long rows go through the chip in segments of 256 vectors, one workgroup each,
// in three launches: every segment's sum of squares (and largest |s w|), the
// rows' from their segments, and the output. The sum is read twice, by as many
// workgroups as there are segments: no workgroup's registers hold such a row.
template <typename T> constexpr int SEGMENT = 256 * VEC<T>;

// A segment's sum of squares and largest |s w|; a row's 1 / rms and largest.
struct Part {
    double sum, most;
};

template <typename T, typename W, bool Q> __global__ __launch_bounds__(256) void k_rms_fwd_sums(RmsArgs a, int segments) {
    using R = Acc<T>;
    constexpr int V = VEC<T>;
    __shared__ R lds[2][2][4];
    __shared__ double lds_wide[4];
    int turn = 0;
    for (int64_t i = blockIdx.x; i < a.rows * segments; i += gridDim.x, turn ^= 1) {
        const int64_t row = i / segments;
        const Span<V> sp((int)(i % segments) * SEGMENT<T> + threadIdx.x * V, (int)a.D);
        Vec<T, V> s = load_vec<T, V>((const T*)a.x + row * a.x_stride + sp.at);
        if (a.residual) {
            const Vec<T, V> r = load_vec<T, V>((const T*)a.residual + row * a.residual_stride + sp.at);
#pragma unroll
            for (int e = 0; e < V; e++) s.v[e] = down<T>(up(s.v[e]) + up(r.v[e]));
            if (sp.any()) store_vec<T, V>((T*)a.summed + row * a.D + sp.at, s);
        }
        Vec<W, V> w;
        if (Q && a.weight) w = load_vec<W, V>((const W*)a.weight + sp.at);
        R sum = 0, most = 0;
#pragma unroll
        for (int e = 0; e < V; e++) {
            const R v = up(s.v[e]);
            sum += sp.own(e) ? v * v : 0;
            if constexpr (Q) most = larger(most, fabsf(a.weight ? v * (R)up(w.v[e]) : v));
        }
        if constexpr (Q)
            if (sum == (R)INFINITY) most = infinity_or(s, most);
        group_sum_max<256>(sum, most, lds[turn][0], lds[turn][1]);
        double wide = most;
        if constexpr (Q) {
            if (!in_fp32(most)) {
                wide = 0;
#pragma unroll
                for (int e = 0; e < V; e++)
                    wide = larger(wide, fabs((double)up(s.v[e]) * (a.weight ? (double)up(w.v[e]) : 1)));
                wide = group_max<256>(infinity_or(s, wide), lds_wide);
            }
        }
        if (threadIdx.x == 0) ((Part*)a.sums)[i] = {sum, wide};
    }
}

template <typename T, bool Q> __global__ __launch_bounds__(256) void k_rms_fwd_join(RmsArgs a, int segments) {
    using R = Acc<T>;
    __shared__ R lds[2][4];
    __shared__ double lds_most[2][4];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const Part* s = (const Part*)a.sums + row * segments;
        R sum = 0;
        double most = 0;
        for (int j = threadIdx.x; j < segments; j += 256) sum += (R)s[j].sum, most = larger(most, s[j].most);
        group_sum_max<256>(sum, most, lds[turn], lds_most[turn]);
        const R rstd = inv_sqrt(sum / (R)a.D + (R)a.eps);
        if (threadIdx.x == 0) {
            ((Part*)a.joined)[row] = {rstd, most};
            if (a.rstd) ((R*)a.rstd)[row] = rstd;
            if constexpr (Q) a.scale[row] = in_fp32((float)most) ? scale_of(rstd, (float)most) : scale_of(rstd, most);
        }
    }
}

template <typename T, typename W, bool Q> __global__ __launch_bounds__(256) void k_rms_fwd_segment(RmsArgs a, int segments) {
    using R = Acc<T>;
    constexpr int V = VEC<T>;
    for (int64_t i = blockIdx.x; i < a.rows * segments; i += gridDim.x) {
        const int64_t row = i / segments;
        const Span<V> sp((int)(i % segments) * SEGMENT<T> + threadIdx.x * V, (int)a.D);
        if (!sp.any()) continue;
        const Vec<T, V> s = a.residual ? load_vec<T, V>((const T*)a.summed + row * a.D + sp.at)
                                       : load_vec<T, V>((const T*)a.x + row * a.x_stride + sp.at);
        Vec<W, V> w;
        if (a.weight) w = load_vec<W, V>((const W*)a.weight + sp.at);
        const Part part = ((const Part*)a.joined)[row];
        if constexpr (Q) {
            float q[V];
            if (in_fp32((float)part.most)) {
                const Narrow quotient((float)part.most);
#pragma unroll
                for (int e = 0; e < V; e++) q[e] = quotient(a.weight ? up(s.v[e]) * (float)up(w.v[e]) : up(s.v[e]));
            } else {
                const Wide quotient(part.most);
#pragma unroll
                for (int e = 0; e < V; e++) q[e] = quotient((double)up(s.v[e]) * (a.weight ? (double)up(w.v[e]) : 1));
            }
            store_e4m3<V>((uint8_t*)a.y + row * a.D + sp.at, q);
        } else {
            const R rstd = (R)part.sum;
            Vec<T, V> q;
#pragma unroll
            for (int e = 0; e < V; e++) {
                R h = up(s.v[e]) * rstd;
                if (a.weight) h *= (R)up(w.v[e]);
                q.v[e] = down<T>(h);
            }
            store_vec<T, V>((T*)a.y + row * a.D + sp.at, q);
        }
    }
}

// Backward of rows in registers, as k_rms_fwd: s, g and gs are read once, and
// every lane sums its columns' g h over the rows that its group takes (row, row
// + stride, ...). part[workgroup][D] gets the workgroup's sums, joined over its
// groups in LDS; a null part leaves them out.
template <typename T, typename W, int V, int G, int K>
__global__ __launch_bounds__(G > 256 ? G : 256) void k_rms_bwd(RmsArgs a) {
    using R = Acc<T>;
    constexpr int ROWS = (G > 256 ? G : 256) / G;
    __shared__ R lds[2][G > 64 ? G / 64 : 1];
    __shared__ R joined[ROWS > 1 ? ROWS * G * K * V : 1];
    const int lane = threadIdx.x % G, group = threadIdx.x / G, D = (int)a.D;
    const R d = (R)a.D;
    Vec<W, V> w[K];
    R dw[K][V] = {};
#pragma unroll
    for (int k = 0; k < K; k++) {
        if (a.weight) w[k] = load_vec<W, V>((const W*)a.weight + Span<V>((k * G + lane) * V, D).at);
        else
#pragma unroll
            for (int e = 0; e < V; e++) w[k].v[e] = down<W>((Acc<W>)1);
    }
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + group;
    Vec<T, V> x[K], g[K], gs[K];
    R rstd = 0;
    auto fetch = [&](int64_t r) {
        rstd = ((const R*)a.rstd)[r];
#pragma unroll
        for (int k = 0; k < K; k++) {
            const int at = Span<V>((k * G + lane) * V, D).at;
            x[k] = load_vec<T, V>((const T*)a.x + r * a.x_stride + at);
            g[k] = load_vec<T, V>((const T*)a.grad + r * a.grad_stride + at);
            if (a.grad_sum) gs[k] = load_vec<T, V>((const T*)a.grad_sum + r * a.grad_sum_stride + at);
        }
    };
    if (row < a.rows) fetch(row);
    for (int turn = 0; row < a.rows; row += stride, turn ^= 1) {
        Vec<T, V> cx[K], cg[K], cs[K];
        const R r = rstd;
#pragma unroll
        for (int k = 0; k < K; k++) {
            cx[k] = x[k], cg[k] = g[k];
            if (a.grad_sum) cs[k] = gs[k];
        }
        fetch(row + stride < a.rows ? row + stride : row);
        R sum = 0;
#pragma unroll
        for (int k = 0; k < K; k++) {
            const Span<V> sp((k * G + lane) * V, D);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const R gh = up(cg[k].v[e]) * (up(cx[k].v[e]) * r);
                dw[k][e] += gh;
                sum += sp.own(e) ? gh * (R)up(w[k].v[e]) : 0;
            }
        }
        if (!a.grad_x) continue;
        const R c = group_sum<G>(sum, lds[turn]) / d;
#pragma unroll
        for (int k = 0; k < K; k++) {
            const Span<V> sp((k * G + lane) * V, D);
            Vec<T, V> q;
#pragma unroll
            for (int e = 0; e < V; e++) {
                R t = r * (up(cg[k].v[e]) * (R)up(w[k].v[e]) - up(cx[k].v[e]) * r * c);
                if (a.grad_sum) t += up(cs[k].v[e]);
                q.v[e] = down<T>(t);
            }
            if (sp.any()) store_vec<T, V>((T*)a.grad_x + row * a.D + sp.at, q);
        }
    }
    if (!a.part) return;
    R* out = (R*)a.part + (int64_t)blockIdx.x * a.D;
#pragma unroll
    for (int k = 0; k < K; k++) {
        const Span<V> sp((k * G + lane) * V, D);
        if (!sp.any()) continue;
        if constexpr (ROWS == 1) {
            Vec<R, V> q;
#pragma unroll
            for (int e = 0; e < V; e++) q.v[e] = dw[k][e];
            store_vec<R, V>(out + sp.at, q);
        } else {
#pragma unroll
            for (int e = 0; e < V; e++) joined[group * (G * K * V) + sp.at + e] = dw[k][e];
        }
    }
    if constexpr (ROWS > 1) {
        __syncthreads();
        for (int i = threadIdx.x; i < G * K * V && i < D; i += 256) {
            R t = 0;
#pragma unroll
            for (int j = 0; j < ROWS; j++) t += joined[j * (G * K * V) + i];
            out[i] = t;
        }
    }
}

// Longer rows take segments here too: the sum of g w h of every segment, the
// rows' means, then ds and the column sums, for which a workgroup keeps its segment's
// columns and takes the rows of a chunk one by one. s and g are read twice.
template <typename T, typename W> __global__ __launch_bounds__(256) void k_rms_bwd_sums(RmsArgs a, int segments) {
    using R = Acc<T>;
    constexpr int V = VEC<T>;
    __shared__ R lds[2][4];
    int turn = 0;
    for (int64_t i = blockIdx.x; i < a.rows * segments; i += gridDim.x, turn ^= 1) {
        const int64_t row = i / segments;
        const Span<V> sp((int)(i % segments) * SEGMENT<T> + threadIdx.x * V, (int)a.D);
        const R r = ((const R*)a.rstd)[row];
        const Vec<T, V> x = load_vec<T, V>((const T*)a.x + row * a.x_stride + sp.at);
        const Vec<T, V> g = load_vec<T, V>((const T*)a.grad + row * a.grad_stride + sp.at);
        Vec<W, V> w;
        if (a.weight) w = load_vec<W, V>((const W*)a.weight + sp.at);
        R sum = 0;
#pragma unroll
        for (int e = 0; e < V; e++) {
            R v = up(g.v[e]) * (up(x.v[e]) * r);
            if (a.weight) v *= (R)up(w.v[e]);
            sum += sp.own(e) ? v : 0;
        }
        sum = group_sum<256>(sum, lds[turn]);
        if (threadIdx.x == 0) ((R*)a.sums)[i] = sum;
    }
}

template <typename T> __global__ __launch_bounds__(256) void k_rms_bwd_join(RmsArgs a, int segments) {
    using R = Acc<T>;
    __shared__ R lds[2][4];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        R sum = 0;
        for (int j = threadIdx.x; j < segments; j += 256) sum += ((const R*)a.sums)[row * segments + j];
        sum = group_sum<256>(sum, lds[turn]);
        if (threadIdx.x == 0) ((R*)a.joined)[row] = sum / (R)a.D;
    }
}

template <typename T, typename W>
__global__ __launch_bounds__(256) void k_rms_bwd_segment(RmsArgs a, int64_t chunk_rows) {
    using R = Acc<T>;
    constexpr int V = VEC<T>;
    const Span<V> sp(blockIdx.x * SEGMENT<T> + threadIdx.x * V, (int)a.D);
    const int64_t r0 = blockIdx.y * chunk_rows, r1 = min(r0 + chunk_rows, a.rows);
    Vec<W, V> w;
    if (a.weight) w = load_vec<W, V>((const W*)a.weight + sp.at);
    R dw[V] = {};
    for (int64_t row = r0; row < r1; row++) {
        const Vec<T, V> x = load_vec<T, V>((const T*)a.x + row * a.x_stride + sp.at);
        const Vec<T, V> g = load_vec<T, V>((const T*)a.grad + row * a.grad_stride + sp.at);
        Vec<T, V> gs, q;
        if (a.grad_sum) gs = load_vec<T, V>((const T*)a.grad_sum + row * a.grad_sum_stride + sp.at);
        const R r = ((const R*)a.rstd)[row], c = a.grad_x ? ((const R*)a.joined)[row] : 0;
#pragma unroll
        for (int e = 0; e < V; e++) {
            const R h = up(x.v[e]) * r, gv = up(g.v[e]);
            dw[e] += gv * h;
            R t = r * ((a.weight ? gv * (R)up(w.v[e]) : gv) - h * c);
            if (a.grad_sum) t += up(gs.v[e]);
            q.v[e] = down<T>(t);
        }
        if (a.grad_x && sp.any()) store_vec<T, V>((T*)a.grad_x + row * a.D + sp.at, q);
    }
    if (!a.part || !sp.any()) return;
    Vec<R, V> q;
#pragma unroll
    for (int e = 0; e < V; e++) q.v[e] = dw[e];
    store_vec<R, V>((R*)a.part + (int64_t)blockIdx.y * a.D + sp.at, q);
}

// Sum of the workgroups' column sums, in fp64: 16 columns and 16 threads for
// each, eight loads of a thread under way. Columns past the grid's go around.
constexpr int64_t REDUCE_BLOCKS = 65536;

template <typename T, typename W> __global__ __launch_bounds__(256) void k_rms_reduce(RmsArgs a, int64_t chunks) {
    using R = Acc<T>;
    __shared__ double lds[16][17];
    const int c = threadIdx.x % 16, g = threadIdx.x / 16;
    for (int64_t first = (int64_t)blockIdx.x * 16; first < a.D; first += (int64_t)gridDim.x * 16) {
        const int64_t col = first + c;
        double t = 0;
        if (col < a.D)
#pragma unroll 8
            for (int64_t k = g; k < chunks; k += 16) t += (double)((const R*)a.part)[k * a.D + col];
        __syncthreads();
        lds[g][c] = t;
        __syncthreads();
        if (g == 0 && col < a.D) {
            t = 0;
#pragma unroll
            for (int i = 0; i < 16; i++) t += lds[i][c];
            ((W*)a.grad_weight)[col] = down<W>((Acc<W>)t);
        }
    }
}

// Segments of the forward pass; 0: rows in registers, which end at 4096 vectors
// (2048 where there are fewer rows than compute units).
int forward_segments(int type, int64_t rows, int64_t D) {
    const int64_t v = 16 / (int64_t)elem_size(type), n = (D + v - 1) / v;
    return n > 4096 || (n > 2048 && rows < 256) ? (int)((n + 255) / 256) : 0;
}

// How the backward pass is split.
struct Split {
    int lanes, per_lane;  // k_rms_bwd's G and K; lanes 0: segments
    int segments;
    int64_t parts;  // partial column sums: workgroups, or chunks of rows
    int64_t chunk_rows;
};
Split split_of(int type, int64_t rows, int64_t D) {
    const int64_t V = 16 / (int64_t)elem_size(type), n = (D + V - 1) / V;
    Split p{};
    static const int shapes[][2] = {{16, 1}, {64, 1}, {64, 2}, {256, 1}, {256, 2}, {512, 2}, {1024, 2}};
    for (const auto& q : shapes)
        if (n <= q[0] * q[1]) {
            p.lanes = q[0], p.per_lane = q[1];
            break;
        }
    if (p.lanes) {
        // at least four rows for a group of lanes, whose column sums cost a write
        // and a read of a row in fp32 (fewer rows are not measured); no more
        // workgroups than run at once
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
size_t acc_size(int type) { return type == E_F64 ? 8 : 4; }
size_t rounded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
size_t part_bytes(const Split& p, int type, int64_t D) { return rounded((size_t)p.parts * (size_t)D * acc_size(type)); }
// The segments' sums (Part forward), and as many of rows behind them.
size_t part_sums_bytes(int64_t rows, int segments) { return rounded((size_t)(rows * segments) * sizeof(Part)); }
size_t sums_bytes(int type, int64_t rows, int segments) { return rounded((size_t)(rows * segments) * acc_size(type)); }

int grid_of(int64_t groups) { return (int)std::min<int64_t>(groups, 4096); }

template <typename T, typename W, bool Q, int G, int K, int V = VEC<T>> hipError_t forward_rows(const RmsArgs& a, hipStream_t s) {
    constexpr int threads = G > 256 ? G : 256, rows = threads / G;
    k_rms_fwd<T, W, V, G, K, Q><<<grid_of((a.rows + rows - 1) / rows), threads, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, typename W, bool Q> hipError_t forward(int type, RmsArgs a, void* ws, hipStream_t s) {
    constexpr int V = VEC<T>;
    if (const int segments = forward_segments(type, a.rows, a.D)) {
        a.sums = ws, a.joined = (char*)ws + part_sums_bytes(a.rows, segments);
        k_rms_fwd_sums<T, W, Q><<<grid_of(a.rows * segments), 256, 0, s>>>(a, segments);
        k_rms_fwd_join<T, Q><<<grid_of(a.rows), 256, 0, s>>>(a, segments);
        k_rms_fwd_segment<T, W, Q><<<grid_of(a.rows * segments), 256, 0, s>>>(a, segments);
        return hipGetLastError();
    }
    if (a.D < V) return forward_rows<T, W, Q, 16, 1, 1>(a, s);
    if (a.D <= 16 * V) return forward_rows<T, W, Q, 16, 1>(a, s);
    if (a.D <= 64 * V) return forward_rows<T, W, Q, 64, 1>(a, s);
    if (a.D <= 128 * V) return forward_rows<T, W, Q, 64, 2>(a, s);
    if (a.D <= 256 * V) return forward_rows<T, W, Q, 256, 1>(a, s);
    if (a.D <= 512 * V) return forward_rows<T, W, Q, 256, 2>(a, s);
    if (a.D <= 1024 * V) return forward_rows<T, W, Q, 512, 2>(a, s);
    if (a.D <= 2048 * V) return forward_rows<T, W, Q, 1024, 2>(a, s);
    return forward_rows<T, W, Q, 1024, 4>(a, s);
}

template <typename T, typename W, int G, int K, int V = VEC<T>> hipError_t backward_rows(const RmsArgs& a, const Split& p, hipStream_t s) {
    k_rms_bwd<T, W, V, G, K><<<(unsigned)p.parts, G > 256 ? G : 256, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, typename W> hipError_t backward(int type, RmsArgs a, void* ws, hipStream_t s) {
    const Split p = split_of(type, a.rows, a.D);
    if (!a.grad_weight && (!a.grad_x || a.rows == 0)) return hipSuccess;
    a.part = a.grad_weight ? ws : nullptr;
    a.sums = (char*)ws + part_bytes(p, type, a.D);
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
                a.joined = (char*)a.sums + sums_bytes(type, a.rows, p.segments);
                k_rms_bwd_sums<T, W><<<grid_of(a.rows * p.segments), 256, 0, s>>>(a, p.segments);
                k_rms_bwd_join<T><<<grid_of(a.rows), 256, 0, s>>>(a, p.segments);
            }
            k_rms_bwd_segment<T, W><<<dim3((unsigned)p.segments, (unsigned)p.parts), 256, 0, s>>>(a, p.chunk_rows);
            e = hipGetLastError();
    }
    if (e != hipSuccess || !a.grad_weight) return e;
    k_rms_reduce<T, W><<<(unsigned)std::min((a.D + 15) / 16, REDUCE_BLOCKS), 256, 0, s>>>(a, p.parts);
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

size_t rms_workspace(int type, int64_t rows, int64_t D, bool backward) {
    if (backward) {
        const Split p = split_of(type, rows, D);
        return part_bytes(p, type, D) +
               (p.segments ? sums_bytes(type, rows, p.segments) + sums_bytes(type, rows, 1) : 0);
    }
    const int segments = forward_segments(type, rows, D);
    return segments ? part_sums_bytes(rows, segments) + part_sums_bytes(rows, 1) : 0;
}

hipError_t launch_rms_forward(int type, int wtype, const RmsArgs& a, void* ws, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return by_type(type, wtype, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        if constexpr (sizeof(T) < 8)
            if (a.scale) return forward<T, W, true>(type, a, ws, s);
        return forward<T, W, false>(type, a, ws, s);
    });
}

hipError_t launch_rms_backward(int type, int wtype, const RmsArgs& a, void* ws, hipStream_t s) {
    return by_type(type, wtype, [&](auto t, auto w) { return backward<decltype(t), decltype(w)>(type, a, ws, s); });
}

}  // namespace qlayer
