// ortho.hip -- orthogonalised updates of matrices, and the optimiser's step on them.
//
//   X = U / (|U|_F + eps), m <= n;   steps times:  A = X X^T,  B = b A + c A^2,
//   X = a X + B X.
//
// 3 m^2 n + m^3 operations a step (A and A^2 are symmetric: half of each is
// computed) on m n values: matrix products. If all matrices of a call
// are small (m <= 64, and X, A and B fit one workgroup's LDS), they take one
// launch, bound by its steps' latency; else all run together, tile by tile, in
// three launches a step: bound by the launches up to some 1000 rows and columns,
// by the matrix cores beyond.
//
// Products are fp16 ones summed in fp32. The singular values of X stay below
// about 1.2 (ortho_bounds), so X, A and B are held in fp16 at powers of two that
// use its range, in two parts, v = hi + lo (hi hi + hi lo + lo hi keeps 22 bits
// of every factor, at a third of fp16's rate, five times fp32's). In float32
// they cost the result less than fp32 sums do (2048x8192: 1.8e-6 off, 3.2e-6
// with fp32 products). fp64 uses fp64.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "elem.hpp"
#include "norm.hpp"
#include "ortho_plan.hpp"

namespace qlayer {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef double double4v __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// The update U of one matrix, oriented so that rows i are the shorter side.
struct Source {
    const void* grad;
    void* momentum;  // or null
    int64_t gb, gi, gj, mb, mi, mj;  // strides between matrices, rows and columns
};
struct Target {
    void* out;
    int64_t ob, oi, oj;
    double step;  // of the optimiser, with the matrix's factor
};
struct Rule {
    double momentum, keep, eps;
    int32_t muon, nesterov;
};

template <typename T> __device__ __forceinline__ Acc<T> grad_at(const Source& s, int64_t b, int64_t i, int64_t j) {
    return up(((const T*)s.grad)[b * s.gb + i * s.gi + j * s.gj]);
}
template <typename T> __device__ __forceinline__ Acc<T>& momentum_at(const Source& s, int64_t b, int64_t i, int64_t j) {
    return ((Acc<T>*)s.momentum)[b * s.mb + i * s.mi + j * s.mj];
}
template <typename T> __device__ __forceinline__ Acc<T> look_ahead(const Rule& r, Acc<T> g, Acc<T> m) {
    return r.nesterov ? g + (Acc<T>)r.momentum * m : m;
}
// U with the momentum's step, and U once that has been done.
template <typename T>
__device__ __forceinline__ Acc<T> first_update(const Source& s, const Rule& r, int64_t b, int64_t i, int64_t j) {
    const Acc<T> g = grad_at<T>(s, b, i, j);
    if (!s.momentum) return g;
    Acc<T>& m = momentum_at<T>(s, b, i, j);
    m = (Acc<T>)r.momentum * m + g;
    return look_ahead<T>(r, g, m);
}
template <typename T>
__device__ __forceinline__ Acc<T> same_update(const Source& s, const Rule& r, int64_t b, int64_t i, int64_t j) {
    const Acc<T> g = grad_at<T>(s, b, i, j);
    return s.momentum ? look_ahead<T>(r, g, momentum_at<T>(s, b, i, j)) : g;
}
template <typename T> __device__ __forceinline__ T* out_at(const Target& t, int64_t b, int64_t i, int64_t j) {
    return (T*)t.out + b * t.ob + i * t.oi + j * t.oj;
}
template <typename T>
__device__ __forceinline__ void write_out(const Target& t, const Rule& r, int64_t b, int64_t i, int64_t j, Acc<T> o) {
    T* p = out_at<T>(t, b, i, j);
    *p = down<T>(r.muon ? (Acc<T>)r.keep * up(*p) - (Acc<T>)t.step * o : o);
}

// Four values side by side in the caller's rows.
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Four {
    T v[4];
};
template <typename T> __device__ __forceinline__ Four<T>* four_at(const Target& t, int64_t b, int64_t i, int64_t j) {
    return (Four<T>*)((T*)t.out + b * t.ob + i * t.oi + j);
}

// The entry of a launch's table whose blocks (first[e] ..) hold this one.
template <typename E> __device__ __forceinline__ int entry_of(const E* e, int count, int block) {
    int k = 0;
    while (k + 1 < count && e[k + 1].first <= block) k++;
    return k;
}

__device__ __forceinline__ double4v mma4(double a, double b, double4v c) {
    return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, 0, 0, 0);
}
// Where register r of lane l of such a 16x16 product lies: the row (the first
// operand's); the column (the second's) is l % 16.
__device__ __forceinline__ int mma4_row(int lane, int r) { return lane / 16 + 4 * r; }

// Where |U| is far below eps, X is far below 1, and fp16 parts at the scale of 1
// would lose its bits. |X| <= 2^e (0: no information) in the Frobenius norm at
// first, and a step multiplies it by at most 2^growth: before step s, X is held
// times 2^raised, which is 0 until the bound leaves room.
__device__ __forceinline__ int norm_exponent(double norm, double eps) {
    const double f = norm / (norm + eps);
    return f > 0 && f < 1 ? ilogb(f) + 1 : 0;  // 0 and NaN as 1
}
__device__ __forceinline__ int raised(int e, int step, float growth) {
    return max(0, min(120, (int)floorf(-(float)e - (float)step * growth)));
}
__device__ __forceinline__ float power_of_two(int e) { return __builtin_ldexpf(1.0f, e); }

// ---------------------------------------------------------------------------
// Small matrices in fp64: one workgroup each, X, A and B in its LDS, products of 16x16x4.
struct SmallEntry {
    Source s;
    Target t;
    int32_t m, n, first;
};
struct SmallArgs {
    SmallEntry e[ENTRIES];
    Rule r;
    double a, b, c;
    int32_t count, steps;
};

__global__ __launch_bounds__(SMALL_THREADS) void k_ortho_small(SmallArgs a) {
    extern __shared__ double lds_small[];
    __shared__ double norm_part[SMALL_THREADS / 64];
    const SmallEntry& e = a.e[entry_of(a.e, a.count, blockIdx.x)];
    const int64_t b = blockIdx.x - e.first;
    const int m = e.m, n = e.n, mp = up16(m), np = up16(n), ldx = np + 4, lda = mp + 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = SMALL_THREADS / 64;
    double *X = lds_small, *A = X + mp * ldx, *B = A + mp * lda;

    const bool by_row = e.s.gj == 1 || e.s.gi != 1;  // the order of the addresses
    double sq = 0;
    for (int k = threadIdx.x; k < mp * np; k += SMALL_THREADS) {
        const int i = by_row ? k / np : k % mp, j = by_row ? k % np : k / mp;
        double u = 0;
        if (i < m && j < n) u = first_update<double>(e.s, a.r, b, i, j);
        X[i * ldx + j] = u;
        sq += u * u;
    }
    const double inv = 1.0 / (sqrt(group_sum<SMALL_THREADS>(sq, norm_part)) + a.r.eps);
    for (int k = threadIdx.x; k < mp * np; k += SMALL_THREADS) {
        double& x = X[(k / np) * ldx + k % np];
        x *= inv;
    }
    __syncthreads();

    const int row = lane % 16, part = lane / 16, mt = mp / 16, nt = np / 16;
    for (int step = 0; step < a.steps; step++) {
        // A = X X^T, then B = b A + c A A: tiles on and below the diagonal, each written twice
        for (int which = 0; which < 2; which++) {
            const double *S = which ? A : X;
            double* D = which ? B : A;
            const int ld = which ? lda : ldx, depth = which ? mp : np;
            for (int t = wave; t < mt * (mt + 1) / 2; t += waves) {
                int ti = 0, tj = t;
                while (tj > ti) tj -= ++ti;
                double4v acc[2] = {};
                const double *p = S + (ti * 16 + row) * ld + part, *q = S + (tj * 16 + row) * ld + part;
                for (int k = 0; k < depth; k += 8) {
                    acc[0] = mma4(p[k], q[k], acc[0]);
                    acc[1] = mma4(p[k + 4], q[k + 4], acc[1]);
                }
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const int i = ti * 16 + mma4_row(lane, r), j = tj * 16 + row;
                    double v = acc[0][r] + acc[1][r];
                    if (which) v = a.b * A[i * lda + j] + a.c * v;
                    D[i * lda + j] = v;
                    if (ti != tj) D[j * lda + i] = v;
                }
            }
            __syncthreads();
        }
        // X = a X + B X, 16 columns at a time: only their own wavefront reads or writes them
        for (int t = wave; t < nt; t += waves) {
            double4v acc[SMALL_M / 16] = {};
            for (int k = 0; k < mp; k += 4) {
                const double x = X[(k + part) * ldx + t * 16 + row];
#pragma unroll
                for (int i = 0; i < SMALL_M / 16; i++)
                    if (i < mt) acc[i] = mma4(B[(i * 16 + row) * lda + k + part], x, acc[i]);
            }
#pragma unroll
            for (int i = 0; i < SMALL_M / 16; i++)
                if (i < mt)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        double& x = X[(i * 16 + mma4_row(lane, r)) * ldx + t * 16 + row];
                        x = a.a * x + acc[i][r];
                    }
        }
        __syncthreads();
    }
    const bool out_by_row = e.t.oj == 1 || e.t.oi != 1;
    for (int k = threadIdx.x; k < m * n; k += SMALL_THREADS) {
        const int i = out_by_row ? k / n : k % m, j = out_by_row ? k % n : k / m;
        write_out<double>(e.t, a.r, b, i, j, X[i * ldx + j]);
    }
}

// Small matrices of the other types: as above with the fp16 products of the
// large ones, X, its transpose and A (then B in its place) in LDS in two parts.
// Each of the 16 wavefronts (8 for up to 128 columns) takes a 16x16 tile of A and of
// B, and 16 or 32 columns of X, which nobody else reads or writes until the step's
// end. 16 matrices of 64x256 take 37 us, one of 20x72 16 us: 11 and 6 us of them
// for reading, the norm and writing, 5 and 1.8 us a step, which is the way from
// barrier to barrier of four phases. With fp32 products (16x16x4, a sixteenth of
// the rate) it was 95 and 19 us.
struct SmallScale {
    float sx, sa, sb, growth;
};
// A wavefront's 16x16 tile, K in steps of 32: rows p and q of two-part arrays,
// whose second part lies `behind` values after the first.
__device__ __forceinline__ float4v two_part(const _Float16* p, const _Float16* q, int behind, int depth) {
    float4v acc = {}, cross0 = {}, cross1 = {};  // three chains of products
    half8 ph = *(const half8*)p, pl = *(const half8*)(p + behind), qh = *(const half8*)q, ql = *(const half8*)(q + behind);
    for (int k = 0; k < depth; k += 32) {
        const int next = min(k + 32, depth - 32);  // read while these products run
        const half8 nph = *(const half8*)(p + next), npl = *(const half8*)(p + behind + next);
        const half8 nqh = *(const half8*)(q + next), nql = *(const half8*)(q + behind + next);
        cross0 = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl, ql, cross0, 0, 0, 0);  // little, but K may be short
        cross0 = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl, qh, cross0, 0, 0, 0);
        cross1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph, ql, cross1, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph, qh, acc, 0, 0, 0);
        ph = nph, pl = npl, qh = nqh, ql = nql;
    }
    return acc + (cross0 + cross1);
}
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef uint32_t word2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ half4 high(float4v v) { return __builtin_convertvector(v, half4); }
__device__ __forceinline__ half4 low(float4v v, half4 hi) {
#pragma unroll
    for (int r = 0; r < 4; r++) v[r] = __builtin_fmaf((float)hi[r], -1.0f, v[r]);  // exact, in one instruction
    return __builtin_convertvector(v, half4);
}

// Lanes 4 k + i of a wavefront hold row i of 4x4 values: afterwards column i.
__device__ __forceinline__ half4 turn4(half4 v) {
    const word2 x = __builtin_bit_cast(word2, v);
    const bool odd = threadIdx.x & 1, upper = threadIdx.x & 2;
    auto swap1 = [](uint32_t w) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0xB1, 0xF, 0xF, false); };
    auto swap2 = [](uint32_t w) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x4E, 0xF, 0xF, false); };
    // pairs of lanes: even (a0 b0)(a2 b2), odd (a1 b1)(a3 b3)
    const uint32_t select = odd ? 0x03020706 : 0x05040100;
    const uint32_t y0 = __builtin_amdgcn_perm(swap1(x.x), x.x, select), y1 = __builtin_amdgcn_perm(swap1(x.y), x.y, select);
    const uint32_t z = swap2(upper ? y0 : y1);
    return __builtin_bit_cast(half4, upper ? word2{z, y1} : word2{y0, z});
}

__device__ __forceinline__ float4v get_two4(const _Float16* p, int behind) {
    return __builtin_convertvector(*(const half4*)p, float4v) + __builtin_convertvector(*(const half4*)(p + behind), float4v);
}
// v + f times four values in two parts.
__device__ __forceinline__ float4v add_two4(float4v v, const _Float16* p, int behind, float f) {
    const half4 hi = *(const half4*)p, lo = *(const half4*)(p + behind);
#pragma unroll
    for (int r = 0; r < 4; r++) v[r] = __builtin_fmaf((float)hi[r], f, __builtin_fmaf((float)lo[r], f, v[r]));
    return v;
}
// A lane's four columns j .. of row i: to rows of pitch p, and to the transpose's rows of pitch q.
__device__ __forceinline__ void put_two4(_Float16* p, int behind, float4v v) {
    const half4 hi = high(v);
    *(half4*)p = hi;
    *(half4*)(p + behind) = low(v, hi);
}
__device__ __forceinline__ void put_turned(_Float16* p, int pitch, int behind, int i, int j, float4v v) {
    const half4 hi = high(v);
    _Float16* q = p + (j + (i & 3)) * pitch + (i & ~3);
    *(half4*)q = turn4(hi);
    *(half4*)(q + behind) = turn4(low(v, hi));
}

constexpr int BATCH = 4;  // groups of four loads of a thread under way together
// The first `count` of four elements a stride apart.
template <typename T> __device__ __forceinline__ float4v load_four(const T* p, int64_t stride, int count) {
    float4v v = {};
    if (stride == 1 && count == 4) {
        const Four<T> f = *(const Four<T>*)p;
#pragma unroll
        for (int r = 0; r < 4; r++) v[r] = up(f.v[r]);
    } else {
#pragma unroll
        for (int r = 0; r < 4; r++)
            if (r < count) v[r] = up(p[r * stride]);
    }
    return v;
}
template <typename T> __device__ __forceinline__ void store_four(T* p, int64_t stride, int count, float4v v) {
    if (stride == 1 && count == 4) {
        Four<T> f;
#pragma unroll
        for (int r = 0; r < 4; r++) f.v[r] = down<T>(v[r]);
        *(Four<T>*)p = f;
    } else {
#pragma unroll
        for (int r = 0; r < 4; r++)
            if (r < count) p[r * stride] = down<T>(v[r]);
    }
}
template <typename T, int THREADS> __global__ __launch_bounds__(THREADS) void k_ortho_tiny(SmallArgs a, SmallScale sc) {
    extern __shared__ double lds_tiny[];
    __shared__ double norm_part[THREADS / 64];
    const SmallEntry& e = a.e[entry_of(a.e, a.count, blockIdx.x)];
    const int64_t b = blockIdx.x - e.first;
    const int m = e.m, n = e.n, mp = up32(m), np = up32(n), px = np + PITCH, pt = mp + PITCH;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = THREADS / 64, row = lane % 16, part = lane / 16;
    _Float16 *X = (_Float16*)lds_tiny, *XT = X + 2 * mp * px, *A = XT + 2 * np * pt;
    const int xlow = mp * px, tlow = np * pt, alow = mp * pt;

    // This thread's groups of four elements in turn, along an array's lines: rows
    // or columns, whichever lie in the order of its addresses.
    struct Walk {
        int line, at, lines, step, groups;
        __device__ __forceinline__ Walk(int groups_) : groups(groups_) {
            line = threadIdx.x / groups, at = threadIdx.x % groups, lines = THREADS / groups, step = THREADS % groups;
        }
        __device__ __forceinline__ void next() {
            line += lines, at += step;
            if (at >= groups) at -= groups, line++;
        }
    };
    const bool by_row = e.s.gj == 1 || e.s.gi != 1, out_by_row = e.t.oj == 1 || e.t.oi != 1;
    // U waits for its norm where the second of X and X^T to be written will be
    _Float16 *first = by_row ? X : XT, *second = by_row ? XT : X;
    const int flow = by_row ? xlow : tlow, slow = by_row ? tlow : xlow, pf = by_row ? px : pt, ps = by_row ? pt : px;
    const int lines = by_row ? m : n, wide = by_row ? n : m, groups = (wide + 3) / 4, total = lines * groups;
    float4v* stage = (float4v*)second;
    double sq = 0;
    {
        const T* grad = (const T*)e.s.grad + b * e.s.gb;
        float* momentum = (float*)e.s.momentum + b * e.s.mb;
        const int64_t gl = by_row ? e.s.gi : e.s.gj, gs = by_row ? e.s.gj : e.s.gi;
        const int64_t ml = by_row ? e.s.mi : e.s.mj, ms = by_row ? e.s.mj : e.s.mi;
        Walk w(groups);
        for (int k0 = threadIdx.x; k0 < total; k0 += BATCH * THREADS) {
            float4v u[BATCH], mom[BATCH];
            float* at[BATCH];
            int count[BATCH];
#pragma unroll
            for (int c = 0; c < BATCH; c++, w.next()) {
                count[c] = k0 + c * THREADS < total ? min(4, wide - 4 * w.at) : 0;
                u[c] = load_four<T>(grad + w.line * gl + 4 * w.at * gs, gs, count[c]);
                at[c] = momentum + w.line * ml + 4 * w.at * ms;
                if (e.s.momentum) mom[c] = load_four<float>(at[c], ms, count[c]);
            }
#pragma unroll
            for (int c = 0; c < BATCH; c++)
                if (count[c]) {
                    if (e.s.momentum) {
                        const float4v now = (float)a.r.momentum * mom[c] + u[c];
                        store_four<float>(at[c], ms, count[c], now);
                        u[c] = a.r.nesterov ? u[c] + (float)a.r.momentum * now : now;
                    }
                    stage[k0 + c * THREADS] = u[c];
#pragma unroll
                    for (int r = 0; r < 4; r++) sq += (double)u[c][r] * (double)u[c][r];
                }
        }
    }
    typedef uint32_t word4 __attribute__((ext_vector_type(4)));
    for (int k = threadIdx.x; k < 2 * flow / 8; k += THREADS) ((word4*)first)[k] = word4{0, 0, 0, 0};
    for (int k = threadIdx.x; k < 2 * alow / 8; k += THREADS) ((word4*)A)[k] = word4{0, 0, 0, 0};
    const double norm = sqrt(group_sum<THREADS>(sq, norm_part));
    const int bound = norm_exponent(norm, a.r.eps);
    int lift = raised(bound, 0, sc.growth);  // X is held times sx 2^lift
    const double inv = (double)sc.sx * (double)power_of_two(lift) / (norm + a.r.eps);
    {
        Walk w(groups);
        for (int k = threadIdx.x; k < total; k += THREADS, w.next()) {
            float4v u = stage[k];
#pragma unroll
            for (int r = 0; r < 4; r++) u[r] = (float)((double)u[r] * inv);
            put_two4(first + w.line * pf + 4 * w.at, flow, u);
        }
    }
    __syncthreads();
    for (int t = wave; t < mp * np / 256; t += waves) {
        const int ft = (by_row ? mp : np) / 16, i = t % ft * 16 + row, j = t / ft * 16 + 4 * part;
        const _Float16* x = first + i * pf + j;
        _Float16* q = second + (j + (i & 3)) * ps + (i & ~3);
        *(half4*)q = turn4(*(const half4*)x);
        *(half4*)(q + slow) = turn4(*(const half4*)(x + flow));
    }
    __syncthreads();

    // tiles of A and B on and below the diagonal: at most 10
    constexpr int TILES_EACH = (10 + THREADS / 64 - 1) / (THREADS / 64);
    auto tile_row = [](int t) { return (t > 0) + (t > 2) + (t > 5); };
    const int mt = (m + 15) / 16, nt = (n + 15) / 16, lower = mt * (mt + 1) / 2;
    for (int step = 0; step < a.steps; step++) {
        const int now = lift;
        lift = raised(bound, step + 1, sc.growth);
        float4v acc[TILES_EACH];
#pragma unroll
        for (int which = 0; which < 2; which++) {
            const float f0 = (float)a.b * sc.sb / sc.sa;
            const float f1 = which ? (float)a.c * sc.sb / (sc.sa * sc.sa) : sc.sa / (sc.sx * sc.sx) * power_of_two(-2 * now);
#pragma unroll
            for (int c = 0; c < TILES_EACH; c++) {
                const int t = wave + c * waves, ti = tile_row(t), tj = t - ti * (ti + 1) / 2;
                if (t < lower) {
                    const _Float16* S = which ? A : X;
                    const int ps = which ? pt : px;
                    const int i = ti * 16, j = tj * 16 + 4 * part;
                    float4v v = two_part(S + (tj * 16 + row) * ps + 8 * part, S + (i + row) * ps + 8 * part, which ? alow : xlow, which ? mp : np) * f1;
                    if (which) v = add_two4(v, A + (i + row) * pt + j, alow, f0);
                    acc[c] = v;
                }
            }
            if (which) __syncthreads();  // B takes A's place
#pragma unroll
            for (int c = 0; c < TILES_EACH; c++) {
                const int t = wave + c * waves, ti = tile_row(t), tj = t - ti * (ti + 1) / 2;
                const int i = ti * 16 + row, j = tj * 16 + 4 * part;
                if (t < lower) {
                    put_two4(A + i * pt + j, alow, acc[c]);
                    if (ti != tj) put_turned(A, pt, alow, i, j, acc[c]);
                }
            }
            __syncthreads();
        }
        const float shift = power_of_two(lift - now), f0 = (float)a.a * shift, f1 = shift / sc.sb;
        // two columns of tiles at a time where there are many: B's rows are read half as often
        constexpr int WIDE = THREADS == 1024 ? 2 : 1;
        for (int t = WIDE * wave; t < nt; t += WIDE * waves) {
            const int j = t * 16 + 4 * part;
            float4v y[SMALL_M / 16][WIDE] = {};
            for (int k = 0; k < mp; k += 32) {
                half8 ph[WIDE], pl[WIDE];
#pragma unroll
                for (int c = 0; c < WIDE; c++) {
                    const _Float16* p = XT + (min(t + c, nt - 1) * 16 + row) * pt + 8 * part + k;
                    ph[c] = *(const half8*)p, pl[c] = *(const half8*)(p + tlow);
                }
#pragma unroll
                for (int i = 0; i < SMALL_M / 16; i++)
                    if (i < mt) {
                        const _Float16* q = A + (i * 16 + row) * pt + 8 * part + k;
                        const half8 qh = *(const half8*)q, ql = *(const half8*)(q + alow);
#pragma unroll
                        for (int c = 0; c < WIDE; c++) y[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl[c], ql, y[i][c], 0, 0, 0);
#pragma unroll
                        for (int c = 0; c < WIDE; c++) y[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl[c], qh, y[i][c], 0, 0, 0);
#pragma unroll
                        for (int c = 0; c < WIDE; c++) y[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph[c], ql, y[i][c], 0, 0, 0);
#pragma unroll
                        for (int c = 0; c < WIDE; c++) y[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph[c], qh, y[i][c], 0, 0, 0);
                    }
            }
            __builtin_amdgcn_wave_barrier();  // all of the old X^T has been read
#pragma unroll
            for (int c = 0; c < WIDE; c++)
#pragma unroll
                for (int i = 0; i < SMALL_M / 16; i++)
                    if (i < mt && t + c < nt) {
                        _Float16* p = X + (i * 16 + row) * px + j + c * 16;
                        const float4v v = add_two4(f1 * y[i][c], p, xlow, f0);
                        put_two4(p, xlow, v);
                        put_turned(XT, pt, tlow, i * 16 + row, j + c * 16, v);
                    }
        }
        __syncthreads();
    }
    {
        const _Float16* from = out_by_row ? X : XT;
        const int behind = out_by_row ? xlow : tlow, pitch = out_by_row ? px : pt, wide = out_by_row ? n : m, groups = (wide + 3) / 4;
        const int64_t ol = out_by_row ? e.t.oi : e.t.oj, os = out_by_row ? e.t.oj : e.t.oi;
        const int total = (out_by_row ? m : n) * groups;
        T* out = out_at<T>(e.t, b, 0, 0);
        Walk w(groups);
        for (int k0 = threadIdx.x; k0 < total; k0 += BATCH * THREADS) {
            float4v v[BATCH], old[BATCH];
            T* at[BATCH];
            int count[BATCH];
#pragma unroll
            for (int c = 0; c < BATCH; c++, w.next()) {
                count[c] = k0 + c * THREADS < total ? min(4, wide - 4 * w.at) : 0;
                at[c] = out + w.line * ol + 4 * w.at * os;
                if (a.r.muon) old[c] = load_four<T>(at[c], os, count[c]);
                if (count[c]) v[c] = get_two4(from + w.line * pitch + 4 * w.at, behind) * (power_of_two(-lift) / sc.sx);
            }
#pragma unroll
            for (int c = 0; c < BATCH; c++)
                store_four<T>(at[c], os, count[c], a.r.muon ? (float)a.r.keep * old[c] - (float)e.t.step * v[c] : v[c]);
        }
    }
}

// ---------------------------------------------------------------------------
__device__ __forceinline__ void put(char* p, int64_t row, int64_t ld, int col, double v) {
    ((double*)(p + row * ld))[col] = v;
}
__device__ __forceinline__ double get(const char* p, int64_t row, int64_t ld, int col) {
    return ((const double*)(p + row * ld))[col];
}

struct PackEntry {
    Source s;
    char* work;    // the first matrix's part of the workspace
    double* part;  // [batch][chunks + 1]: sums of squares, then X's exponent (norm_exponent)
    int32_t m, n, first, chunks;
};
struct PackArgs {
    PackEntry e[ENTRIES];
    Rule r;
    double scale;  // X is stored times this
    float growth;
    int32_t count;
};

// The momentum's step and the sums of squares, a chunk of lines each: lines lie
// along the arrays' unit stride where they have one, and are read in vectors.
template <typename T> __global__ __launch_bounds__(256) void k_ortho_norm(PackArgs a) {
    using R = Acc<T>;
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ double lds[4];
    const PackEntry& e = a.e[entry_of(a.e, a.count, blockIdx.x)];
    const int at = blockIdx.x - e.first, chunk = at % e.chunks;
    const int64_t b = at / e.chunks;
    const bool by_row = e.s.gj == 1 || e.s.gi != 1;
    const int lines = by_row ? e.m : e.n, length = by_row ? e.n : e.m;
    const int l0 = (int)((int64_t)lines * chunk / e.chunks), l1 = (int)((int64_t)lines * (chunk + 1) / e.chunks);
    const int64_t gl = by_row ? e.s.gi : e.s.gj, ml = by_row ? e.s.mi : e.s.mj;
    const bool vectors = (by_row ? e.s.gj : e.s.gi) == 1 && (!e.s.momentum || (by_row ? e.s.mj : e.s.mi) == 1);
    const int whole = vectors ? length / V : 0, rest = length - whole * V;
    double sq = 0;
    for (unsigned k = threadIdx.x; k < (unsigned)(l1 - l0) * (unsigned)whole; k += 256) {
        const int l = l0 + (int)(k / (unsigned)whole), f = (int)(k % (unsigned)whole) * V;
        const Vec<T, V> g = load_vec<T, V>((const T*)e.s.grad + b * e.s.gb + l * gl + f);
        Vec<R, V> u;
        if (e.s.momentum) {
            R* p = (R*)e.s.momentum + b * e.s.mb + l * ml + f;
            u = load_vec<R, V>(p);
#pragma unroll
            for (int i = 0; i < V; i++) u.v[i] = (R)a.r.momentum * u.v[i] + up(g.v[i]);
            store_vec<R, V>(p, u);
#pragma unroll
            for (int i = 0; i < V; i++) u.v[i] = look_ahead<T>(a.r, up(g.v[i]), u.v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V; i++) u.v[i] = up(g.v[i]);
        }
#pragma unroll
        for (int i = 0; i < V; i++) sq += (double)u.v[i] * (double)u.v[i];
    }
    for (unsigned k = threadIdx.x; k < (unsigned)(l1 - l0) * (unsigned)rest; k += 256) {
        const int l = l0 + (int)(k / (unsigned)rest), f = whole * V + (int)(k % (unsigned)rest);
        const R u = first_update<T>(e.s, a.r, b, by_row ? l : f, by_row ? f : l);
        sq += (double)u * (double)u;
    }
    sq = group_sum<256>(sq, lds);
    if (threadIdx.x == 0) e.part[b * (e.chunks + 1) + chunk] = sq;
}

// X and X^T of a 64x64 tile.
template <typename T, int F> __global__ __launch_bounds__(256) void k_ortho_pack(PackArgs a) {
    using R = Acc<T>;
    __shared__ R tile[64][65];
    __shared__ double lds[4];
    const PackEntry& e = a.e[entry_of(a.e, a.count, blockIdx.x)];
    const int mp = (int)up64(e.m), np = (int)up64(e.n), ti = mp / 64, tj = np / 64;
    const int at = blockIdx.x - e.first, i0 = at / tj % ti * 64, j0 = at % tj * 64;
    const int64_t b = at / (ti * tj);
    double sq = 0;
    double* part = e.part + b * (e.chunks + 1);
    for (int k = threadIdx.x; k < e.chunks; k += 256) sq += part[k];
    const double norm = sqrt(group_sum<256>(sq, lds));
    double inv = a.scale / (norm + a.r.eps);
    if constexpr (F == TWO) {
        const int bound = norm_exponent(norm, a.r.eps);
        inv *= (double)power_of_two(raised(bound, 0, a.growth));
        if (i0 == 0 && j0 == 0 && threadIdx.x == 0) part[e.chunks] = bound;
    }
    const bool by_row = e.s.gj == 1 || e.s.gi != 1;
    if constexpr (F == DOUBLE) {
        for (int k = threadIdx.x; k < 64 * 64; k += 256) {
            const int i = by_row ? k / 64 : k % 64, j = by_row ? k % 64 : k / 64;
            tile[i][j] = 0;
            if (i0 + i < e.m && j0 + j < e.n) tile[i][j] = same_update<T>(e.s, a.r, b, i0 + i, j0 + j) * inv;
        }
    } else {  // four elements of a line at a time
        const int l0 = by_row ? i0 : j0, f0 = by_row ? j0 : i0, lines = by_row ? e.m : e.n, wide = by_row ? e.n : e.m;
        const int64_t gl = by_row ? e.s.gi : e.s.gj, gs = by_row ? e.s.gj : e.s.gi;
        const int64_t ml = by_row ? e.s.mi : e.s.mj, ms = by_row ? e.s.mj : e.s.mi;
#pragma unroll
        for (int c = 0; c < 4; c++) {
            const int k = c * 256 + threadIdx.x, l = k / 16, f = k % 16 * 4;
            const int count = l0 + l < lines ? max(0, min(4, wide - f0 - f)) : 0;
            float4v u = load_four<T>((const T*)e.s.grad + b * e.s.gb + (l0 + l) * gl + (f0 + f) * gs, gs, count);
            if (e.s.momentum) {
                const float4v m = load_four<float>((const float*)e.s.momentum + b * e.s.mb + (l0 + l) * ml + (f0 + f) * ms, ms, count);
                u = a.r.nesterov ? u + (float)a.r.momentum * m : m;
            }
#pragma unroll
            for (int r = 0; r < 4; r++) (by_row ? tile[l][f + r] : tile[f + r][l]) = (float)((double)u[r] * inv);
        }
    }
    __syncthreads();
    const Layout l = layout_of(mp, np, unit_of(F));
    char *x = e.work + b * l.size + l.x, *xt = e.work + b * l.size + l.xt;
    const int64_t ldx = (int64_t)np * unit_of(F), ldt = (int64_t)mp * unit_of(F);
    if constexpr (F == DOUBLE) {
        for (int k = threadIdx.x; k < 64 * 64; k += 256) {
            put(x, i0 + k / 64, ldx, j0 + k % 64, tile[k / 64][k % 64]);
            put(xt, j0 + k / 64, ldt, i0 + k % 64, tile[k % 64][k / 64]);
        }
    } else {  // eight values and 16 bytes of a part at a time
#pragma unroll
        for (int c = 0; c < 2; c++) {
            const int k = c * 256 + threadIdx.x, r = k / 8, at = k % 8 * 8;
            half8 hi, lo, thi, tlo;
#pragma unroll
            for (int v = 0; v < 8; v++) {
                hi[v] = (_Float16)tile[r][at + v], lo[v] = (_Float16)(tile[r][at + v] - (float)hi[v]);
                thi[v] = (_Float16)tile[at + v][r], tlo[v] = (_Float16)(tile[at + v][r] - (float)thi[v]);
            }
            const int in = at / 32 * 64 + at % 32;
            _Float16 *p = (_Float16*)(x + (i0 + r) * ldx) + j0 * 2 + in, *q = (_Float16*)(xt + (j0 + r) * ldt) + i0 * 2 + in;
            *(half8*)p = hi, *(half8*)(p + 32) = lo;
            *(half8*)q = thi, *(half8*)(q + 32) = tlo;
        }
    }
}

// A product with few tiles and a long K is split along K: PART workgroups leave
// their sums in the workspace, and one JOIN workgroup a tile adds them in order
// and goes on as a WHOLE one does.
enum Split { WHOLE, PART, JOIN };
struct GemmEntry {
    char* work;
    const double* exponent;  // the first matrix's (norm_exponent), `apart` before the next one's
    Target t;
    int32_t m, n, first, apart;
};
struct GemmArgs {
    GemmEntry e[ENTRIES];
    Rule r;
    double f0, f1;  // C is stored as f0 * (what it adds to) + f1 * (the sum)
    float growth;
    int32_t step;
    int32_t count, from;  // from: which X^T is read
    int32_t splits;
    char* part;           // [tile][split][values of a tile] fp32, as the threads hold them
};

// 16 bytes of each lane from a buffer to LDS: lane l's lie 16 l past `to`.
__device__ __forceinline__ void load_lds(__amdgpu_buffer_rsrc_t from, uint32_t lane_offset, uint32_t offset, char* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, lane_offset, offset, 0, 0);
}

// Consecutive workgroups go to the eight XCDs in turn: give each XCD a run of
// consecutive tiles, whose operands its L2 then holds.
__device__ __forceinline__ int xcd_run(int block, int blocks) {
    const int x = block % 8, q = blocks / 8, r = blocks % 8;
    return x * q + min(x, r) + block / 8;
}

// Four consecutive values of a row in two parts (col % 4 = 0).
__device__ __forceinline__ float4v get4(const char* p, int64_t row, int64_t ld, int col) {
    return get_two4((const _Float16*)(p + row * ld) + col / 32 * 64 + col % 32, 32);
}

// A wavefront's operands of half a step: N tiles' rows of 32 values, or of 2 x 4 in fp64.
template <int F, int N> struct Operands {
    std::conditional_t<F == DOUBLE, double[2], half8> v[N];
};

// The schedule of a half: READS reads of LDS from its start, a product behind each.
template <int READS> __device__ __forceinline__ void spread() {
#pragma unroll
    for (int r = 0; r < READS; r++) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
}

// One step's operands in LDS, each of them an object of its own for the compiler:
// loads on their way to one do not hold up reads of another.
#define STAGE(name) __shared__ __attribute__((aligned(16))) char name[2 * BT * 128]

// BT x BT tiles of C, WI x WJ wavefronts. The operands' next 128 bytes of every
// row are on their way to LDS, STAGES steps ahead, while the products of a step
// run. Chunk q (16 bytes) of a row r lies at q ^ (r % 8): the rows that a
// wavefront reads together start in different banks (no conflicts counted).
// 256 is the tile whose products take longer than its LDS traffic; smaller ones
// fill the chip where there are fewer tiles than units. Measured: X of 4096x4096
// in 312 us (median; 0.44 PFLOP/s, 1.32 of fp16 products, of the 1.43 that a large
// fp16 product reaches), of 2048x8192 in 176 (0.39 and 1.17). What is left is the
// end: X read, X and X^T written at once by all units. Four wavefronts instead of
// eight a tile, with fewer LDS reads, took 1.1 to 1.3 times as long.
template <typename T, int F, int MODE, int SPLIT, int BT, int WI, int WJ, int STAGES>
__global__ __launch_bounds__(64 * WI * WJ, 2) void k_ortho_gemm(GemmArgs a) {
    constexpr int U = unit_of(F), THREADS = 64 * WI * WJ, TI = BT / WI / 16, TJ = BT / WJ / 16;
    constexpr int LOADS = BT * 8 / THREADS;  // of a thread, for each operand
    using Q = std::conditional_t<F == DOUBLE, double4v, float4v>;
    STAGE(s0);
    STAGE(s1);
    const int all = SPLIT == PART ? gridDim.x / a.splits : gridDim.x;
    const int run = xcd_run(blockIdx.x, gridDim.x), block = SPLIT == PART ? run % all : run;
    const GemmEntry& e = a.e[entry_of(a.e, a.count, block)];
    const int mp = (int)up64(e.m), np = (int)up64(e.n);
    const Layout l = layout_of(mp, np, U);
    const int64_t xt_from = l.xt + a.from * (l.a - l.xt) / 2, xt_to = l.xt + (1 - a.from) * (l.a - l.xt) / 2;
    const int mt = (mp + BT - 1) / BT, nt = (np + BT - 1) / BT;
    const int tiles = MODE <= POLY ? mt * (mt + 1) / 2 : mt * nt;
    const int t = (block - e.first) % tiles;
    const int64_t b = (block - e.first) / tiles;
    char* w = e.work + b * l.size;
    [[maybe_unused]] const int bound = F == TWO && MODE != POLY ? (int)e.exponent[b * e.apart] : 0;
    int ti, tj;
    if (MODE <= POLY) {
        ti = (int)((sqrtf(8.0f * t + 1) - 1) / 2);
        while (ti * (ti + 1) / 2 > t) ti--;
        while ((ti + 1) * (ti + 2) / 2 <= t) ti++;
        tj = t - ti * (ti + 1) / 2;
    } else {  // bands of eight tiles down, then across
        const int band = t / (8 * nt), high = min(8, mt - band * 8), at = t - band * 8 * nt;
        ti = band * 8 + at % high, tj = at / high;
    }
    const int left_rows = mp, right_rows = MODE >= APPLY ? np : mp;
    const int ld = (MODE == GRAM ? np : mp) * U;  // bytes of an operand's row
    const char* left = w + (MODE == GRAM ? l.x : MODE == POLY ? l.a : l.b) + (int64_t)ti * BT * ld;
    const char* right = w + (MODE == GRAM ? l.x : MODE == POLY ? l.a : xt_from) + (int64_t)tj * BT * ld;
    const int li = min(BT, left_rows - ti * BT), ri = min(BT, right_rows - tj * BT);
    const auto lbuf = __builtin_amdgcn_make_buffer_rsrc((void*)left, 0, li * ld, 0x00027000);
    const auto rbuf = __builtin_amdgcn_make_buffer_rsrc((void*)right, 0, ri * ld, 0x00027000);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave / WJ, wj = wave % WJ;
    const int row = lane % 16, part = lane / 16;
    int begin = 0, end = ld;  // bytes of the rows that this workgroup multiplies
    if constexpr (SPLIT == PART) {
        const int each = (ld / 128 + a.splits - 1) / a.splits * 128;
        begin = run / all * each, end = min(begin + each, ld);
    }
    // sums of up to 128 products do not average out what lo lo would add
    [[maybe_unused]] const bool few = ld <= 512;
    uint32_t lat[LOADS], rat[LOADS];
#pragma unroll
    for (int c = 0; c < LOADS; c++) {
        const int r = (c * THREADS + threadIdx.x) / 8, q = threadIdx.x % 8;
        lat[c] = (uint32_t)(min(r, li - 1) * ld + ((q ^ (r & 7)) * 16));
        rat[c] = (uint32_t)(min(r, ri - 1) * ld + ((q ^ (r & 7)) * 16));
    }
    auto load = [&](char* s, int k) {
#pragma unroll
        for (int c = 0; c < LOADS; c++) load_lds(lbuf, lat[c], k, s + (c * THREADS + wave * 64) * 16);
#pragma unroll
        for (int c = 0; c < LOADS; c++) load_lds(rbuf, rat[c], k, s + BT * 128 + (c * THREADS + wave * 64) * 16);
    };
    Q acc[TI][TJ] = {};
    // A step has two halves, of 64 bytes of every row. While the products of one
    // run, the operands of the next come from LDS: the second half's at first;
    // then, once the next step's loads have arrived everywhere and nobody reads
    // this step's any more, its first half's, and the loads that take this
    // step's place in LDS are sent off. Nothing waits for LDS or HBM but for what
    // a half's products do not hide.
    Operands<F, TI> p, p1;
    Operands<F, TJ> q, q1;
    const int at = F == DOUBLE ? row * 128 : row * 128 + ((part ^ (row & 7)) * 16);
    auto read = [&](const char* s, int half, Operands<F, TI>& pp, Operands<F, TJ>& qq) {
        const char *sl = s + wi * TI * 2048, *sr = s + BT * 128 + wj * TJ * 2048;
        if constexpr (F == DOUBLE) {
#pragma unroll
            for (int k = 0; k < 2; k++) {  // values 8 half + 4 k + part of the row
                const int c = at + (((half * 4 + k * 2 + part / 2) ^ (row & 7)) * 16) + part % 2 * 8;
#pragma unroll
                for (int i = 0; i < TI; i++) pp.v[i][k] = *(const double*)(sl + c + i * 2048);
#pragma unroll
                for (int j = 0; j < TJ; j++) qq.v[j][k] = *(const double*)(sr + c + j * 2048);
            }
        } else {
            const int c = half ? at ^ 64 : at;
#pragma unroll
            for (int i = 0; i < TI; i++) pp.v[i] = *(const half8*)(sl + c + i * 2048);
#pragma unroll
            for (int j = 0; j < TJ; j++) qq.v[j] = *(const half8*)(sr + c + j * 2048);
        }
    };
    auto product = [&](const Operands<F, TI>& pp, const Operands<F, TJ>& qq) {
#pragma unroll
        for (int i = 0; i < TI; i++)
#pragma unroll
            for (int j = 0; j < TJ; j++)
                if constexpr (F == DOUBLE) {
                    acc[i][j] = mma4(qq.v[j][0], pp.v[i][0], acc[i][j]);
                    acc[i][j] = mma4(qq.v[j][1], pp.v[i][1], acc[i][j]);
                } else {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(qq.v[j], pp.v[i], acc[i][j], 0, 0, 0);
                }
    };
    // All wavefronts' loads have arrived but for those of the later steps under
    // way, and all their reads too. Past the last step its loads are repeated, so
    // that the number of open loads is always the same.
    auto arrived = [](auto open) {
        constexpr int n = decltype(open)::value;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((n & 15) | 7 << 4 | (n >> 4) << 14);  // vmcnt(n) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto step = [&](char* now, char* next, int k) {
        read(now, 1, p1, q1);
        product(p, q);
        spread<TI + TJ>();
        __builtin_amdgcn_sched_barrier(0);
        arrived(std::integral_constant<int, 2 * LOADS*(STAGES - 2)>{});
        load(now, min(k + 128 * STAGES, end - 128));
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (F == TWO) {  // hi lo, then lo hi
            if constexpr (BT == 64)
                if (few) product(p1, q1);
            product(p, q1);
            __builtin_amdgcn_sched_barrier(0);
            product(p1, q);
            read(next, 0, p, q);
            spread<TI>();
        } else {
            read(next, 0, p, q);
            product(p1, q1);
            spread<TI + TJ>();
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // The matrix cores round a sum to fp32 after every eight products: 3 K / 8 times
    // in a chain of K values, and at the size that a sum of squares has grown to.
    // After FOLDED values the sums so far are put aside. Twelve rows of 5992, over
    // which nothing averages that out, were 6e-6 off in one chain, 1e-6 so. Tiles
    // past 128 have no registers for it (choose()).
    constexpr bool FOLD = MODE == GRAM && F == TWO && BT <= 128;
    [[maybe_unused]] Q aside[FOLD ? TI : 1][FOLD ? TJ : 1] = {};
    auto fold = [&](int k) {
        if constexpr (FOLD)
            if ((k - begin) % (FOLDED * U) == 0) {
#pragma unroll
                for (int i = 0; i < TI; i++)
#pragma unroll
                    for (int j = 0; j < TJ; j++) aside[i][j] += acc[i][j], acc[i][j] = Q{};
            }
    };
    if (SPLIT != JOIN && begin < end) {
        load(s0, begin);
        load(s1, min(begin + 128, end - 128));
        if constexpr (STAGES == 2) {
            arrived(std::integral_constant<int, 2 * LOADS>{});
            read(s0, 0, p, q);
            for (int k = begin;; k += 256) {
                step(s0, s1, k);
                if (k + 128 >= end) break;
                step(s1, s0, k + 128);
                if (k + 256 >= end) break;
                fold(k + 256);
            }
        } else if constexpr (STAGES == 3) {
            STAGE(s2);
            load(s2, min(begin + 256, end - 128));
            arrived(std::integral_constant<int, 4 * LOADS>{});
            read(s0, 0, p, q);
            for (int k = begin;; k += 384) {
                step(s0, s1, k);
                if (k + 128 >= end) break;
                step(s1, s2, k + 128);
                if (k + 256 >= end) break;
                step(s2, s0, k + 256);
                if (k + 384 >= end) break;
            }
        } else {
            STAGE(s2);
            STAGE(s3);
            load(s2, min(begin + 256, end - 128));
            load(s3, min(begin + 384, end - 128));
            arrived(std::integral_constant<int, 6 * LOADS>{});
            read(s0, 0, p, q);
            for (int k = begin;; k += 512) {
                step(s0, s1, k);
                if (k + 128 >= end) break;
                step(s1, s2, k + 128);
                if (k + 256 >= end) break;
                step(s2, s3, k + 256);
                if (k + 384 >= end) break;
                step(s3, s0, k + 384);
                if (k + 512 >= end) break;
                fold(k + 512);
            }
        }
        __builtin_amdgcn_s_waitcnt(0);
        fold(begin);
        if constexpr (FOLD) {
#pragma unroll
            for (int i = 0; i < TI; i++)
#pragma unroll
                for (int j = 0; j < TJ; j++) acc[i][j] = aside[i][j];
        }
    }
    if constexpr (SPLIT != WHOLE) {
        Q* part = (Q*)a.part + (int64_t)block * a.splits * (TI * TJ * THREADS) + threadIdx.x;
        if constexpr (SPLIT == PART) {
            part += (int64_t)(run / all) * (TI * TJ * THREADS);
#pragma unroll
            for (int k = 0; k < TI * TJ; k++) part[k * THREADS] = acc[k / TJ][k % TJ];
            return;
        }
        // several splits' loads under way together
        constexpr int TOGETHER = BT == 64 ? 8 : 2;
        for (int split = 0; split < a.splits; split += TOGETHER) {
            Q v[TOGETHER][TI * TJ];
#pragma unroll
            for (int c = 0; c < TOGETHER; c++)
#pragma unroll
                for (int k = 0; k < TI * TJ; k++) v[c][k] = part[(int64_t)(min(split + c, a.splits - 1) * TI * TJ + k) * THREADS];
#pragma unroll
            for (int c = 0; c < TOGETHER; c++)
                if (split + c < a.splits)
#pragma unroll
                    for (int k = 0; k < TI * TJ; k++) acc[k / TJ][k % TJ] += v[c][k];
        }
    }
    const int64_t lda = (int64_t)mp * U, ldx = (int64_t)np * U;
    const int i0 = ti * BT + wi * TI * 16 + row, j0 = tj * BT + wj * TJ * 16;
    if constexpr (F == DOUBLE) {
#pragma unroll
        for (int i = 0; i < TI; i++)
#pragma unroll
            for (int j = 0; j < TJ; j++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const int gi = i0 + i * 16, gj = j0 + j * 16 + mma4_row(lane, r);
                    if (gi >= left_rows || gj >= right_rows) continue;
                    double v = a.f1 * acc[i][j][r];
                    if constexpr (MODE == POLY) v += a.f0 * get(w + l.a, gi, lda, gj);
                    if constexpr (MODE >= APPLY) v += a.f0 * get(w + l.x, gi, ldx, gj);
                    if constexpr (MODE <= POLY) {
                        put(w + (MODE == GRAM ? l.a : l.b), gi, lda, gj, v);
                        if (ti != tj) put(w + (MODE == GRAM ? l.a : l.b), gj, lda, gi, v);
                    } else if constexpr (MODE == APPLY) {
                        put(w + l.x, gi, ldx, gj, v);
                        put(w + xt_to, gj, lda, gi, v);
                    } else if (gi < e.m && gj < e.n) {
                        write_out<T>(e.t, a.r, b, gi, gj, v);
                    }
                }
    } else {
        // A wavefront's tiles from the top: what a row of them is added to is read
        // while the row before is written, at places that are there for every lane.
        float f0 = (float)a.f0, f1 = (float)a.f1;
        if constexpr (MODE == GRAM) f1 *= power_of_two(-2 * raised(bound, a.step, a.growth));
        if constexpr (MODE >= APPLY) {
            const float shift = power_of_two((MODE == APPLY ? raised(bound, a.step + 1, a.growth) : 0) - raised(bound, a.step, a.growth));
            f0 *= shift, f1 *= shift;
        }
        const bool by_row = e.t.oj == 1 && e.n >= 4;  // LAST: four columns at a time to the caller
        struct Behind {
            float4v add[TJ];
            Four<T> old[TJ];
        };
        auto fetch = [&](int i) {
            Behind f;
            const int gi = min(i0 + i * 16, left_rows - 1);
#pragma unroll
            for (int j = 0; j < TJ; j++) {
                const int gj = min(j0 + j * 16, right_rows - 16) + 4 * part;
                if constexpr (MODE == POLY) f.add[j] = get4(w + l.a, gi, lda, gj);
                if constexpr (MODE >= APPLY) f.add[j] = get4(w + l.x, gi, ldx, gj);
                if constexpr (MODE == LAST)
                    if (a.r.muon) {
                        if (by_row) {
                            f.old[j] = *four_at<T>(e.t, b, min(gi, e.m - 1), min(gj, e.n - 4));
                        } else {
#pragma unroll
                            for (int r = 0; r < 4; r++) f.old[j].v[r] = *out_at<T>(e.t, b, min(gi, e.m - 1), min(gj + r, e.n - 1));
                        }
                    }
            }
            return f;
        };
        Behind now = fetch(0);
        if constexpr (MODE != LAST) {
            // the wavefront's own part of the LDS, to store whole rows of its tiles
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            _Float16* own = (_Float16*)(s0 + wave * (2 * BT * 128 / (WI * WJ)));
            constexpr int PLANES = 2;
            constexpr int WIDE = TJ * 16 + 8, HIGH = TI * 16 + 8;  // pitches, off a multiple of the banks
            static_assert(16 * HIGH * 2 <= 2 * BT * 128 / (WI * WJ) && 16 * WIDE * 2 * PLANES <= 2 * BT * 128 / (WI * WJ), "LDS");
            char* to = w + (MODE == GRAM ? l.a : MODE == POLY ? l.b : l.x);
            const int64_t to_ld = MODE == APPLY ? ldx : lda;
            auto in_row = [](int64_t c, int plane) { return c / 32 * 64 + plane * 32 + c % 32; };
#pragma unroll
            for (int i = 0; i < TI; i++) {
                const Behind next = fetch(min(i + 1, TI - 1));
#pragma unroll
                for (int j = 0; j < TJ; j++) {
                    float4v v = acc[i][j] * f1;
                    if constexpr (MODE != GRAM) v += now.add[j] * f0;
                    acc[i][j] = v;
                    const half4 hi = high(v);
                    *(half4*)(own + row * WIDE + j * 16 + 4 * part) = hi;
                    *(half4*)(own + (16 + row) * WIDE + j * 16 + 4 * part) = low(v, hi);
                }
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int c = 0; c < (16 * TJ * 2 * PLANES + 63) / 64; c++) {
                    const int id = c * 64 + lane, col = id % (TJ * 2) * 8, r = id / (TJ * 2) % 16, plane = id / (TJ * 32);
                    const int gi = ti * BT + (wi * TI + i) * 16 + r, gj = j0 + col;
                    if (id < 16 * TJ * 2 * PLANES && gi < left_rows && gj < right_rows)
                        *(half8*)((_Float16*)(to + gi * to_ld) + in_row(gj, plane)) = *(const half8*)(own + (plane * 16 + r) * WIDE + col);
                }
                __builtin_amdgcn_wave_barrier();
                now = next;
            }
            if (MODE == APPLY || ti != tj) {  // the same, transposed
                to = w + (MODE == GRAM ? l.a : MODE == POLY ? l.b : xt_to);
#pragma unroll
                for (int j = 0; j < TJ; j++)
#pragma unroll
                    for (int plane = 0; plane < PLANES; plane++) {
#pragma unroll
                        for (int i = 0; i < TI; i++) {
                            const half4 hi = high(acc[i][j]);
                            *(half4*)(own + (4 * part + (row & 3)) * HIGH + i * 16 + (row & ~3)) = turn4(plane ? low(acc[i][j], hi) : hi);
                        }
                        __builtin_amdgcn_wave_barrier();
#pragma unroll
                        for (int c = 0; c < (16 * TI * 2 + 63) / 64; c++) {
                            const int id = c * 64 + lane, col = id % (TI * 2) * 8, r = id / (TI * 2);
                            const int gj = j0 + j * 16 + r, gi = ti * BT + wi * TI * 16 + col;
                            if (id < 16 * TI * 2 && gj < right_rows && gi < left_rows)
                                *(half8*)((_Float16*)(to + gj * lda) + in_row(gi, plane)) = *(const half8*)(own + r * HIGH + col);
                        }
                        __builtin_amdgcn_wave_barrier();
                    }
            }
        } else {
            auto value = [&](float v, T was) { return down<T>(a.r.muon ? (float)a.r.keep * up(was) - (float)e.t.step * v : v); };
#pragma unroll
            for (int i = 0; i < TI; i++) {
                const Behind next = fetch(min(i + 1, TI - 1));
                const int gi = i0 + i * 16;
#pragma unroll
                for (int j = 0; j < TJ; j++) {
                    const int gj = j0 + j * 16 + 4 * part;
                    const float4v v = acc[i][j] * f1 + now.add[j] * f0;
                    if (by_row && gi < e.m && gj + 4 <= e.n) {
                        Four<T> f;
#pragma unroll
                        for (int r = 0; r < 4; r++) f.v[r] = value(v[r], now.old[j].v[r]);
                        *four_at<T>(e.t, b, gi, gj) = f;
                    } else if (gi < e.m) {
#pragma unroll
                        for (int r = 0; r < 4; r++)
                            if (gj + r < e.n) {
                                // where columns go four at a time, `old` holds others at the edge
                                T* p = out_at<T>(e.t, b, gi, gj + r);
                                *p = value(v[r], by_row && a.r.muon ? *p : now.old[j].v[r]);
                            }
                    }
                }
                now = next;
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Host side.

Source source_of(const ql_matrix& q, bool muon) {
    const bool t = shape_of(q).turned;
    Source s{};
    s.grad = q.grad;
    s.gb = q.grad_stride[0], s.gi = q.grad_stride[t ? 2 : 1], s.gj = q.grad_stride[t ? 1 : 2];
    if (muon) {
        s.momentum = q.momentum;
        s.mb = q.momentum_stride[0], s.mi = q.momentum_stride[t ? 2 : 1], s.mj = q.momentum_stride[t ? 1 : 2];
    }
    return s;
}
Target target_of(const ql_matrix& q, const OrthoCall& c) {
    const bool t = shape_of(q).turned;
    Target r{};
    r.out = q.out;
    r.ob = q.out_stride[0], r.oi = q.out_stride[t ? 2 : 1], r.oj = q.out_stride[t ? 1 : 2];
    r.step = c.step * std::sqrt(std::max(1.0, (double)q.rows / (double)q.cols));
    return r;
}

// Past 64 KiB the runtime wants a kernel's limit set, once on each device.
hipError_t allow_lds(const void* kernel, std::atomic<uint64_t>& ready, int bytes) {
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
    if (dev < 64 && (ready.load(std::memory_order_acquire) >> dev & 1)) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess && dev < 64) ready.fetch_or(1ull << dev, std::memory_order_release);
    return e;
}

template <typename T, int THREADS> hipError_t launch_tiny(const SmallArgs& a, unsigned blocks, size_t lds, const Scales& k, hipStream_t s) {
    static std::atomic<uint64_t> ready{0};
    if (hipError_t e = allow_lds((const void*)k_ortho_tiny<T, THREADS>, ready, TINY_LDS); e != hipSuccess) return e;
    k_ortho_tiny<T, THREADS><<<blocks, THREADS, lds, s>>>(a, SmallScale{(float)k.sx, (float)k.sa, (float)k.sb, (float)k.growth});
    return hipGetLastError();
}

template <typename T> hipError_t run_small(const OrthoCall& c, const Rule& rule, hipStream_t s) {
    constexpr int64_t SIZE = sizeof(T), STATE = sizeof(Acc<T>);
    int64_t done = 0;  // matrices of entry `at` that earlier launches took
    for (int at = 0; at < c.count;) {
        SmallArgs a{};
        a.r = rule, a.a = c.a, a.b = c.b, a.c = c.c, a.steps = c.steps;
        size_t lds = 0;
        int64_t blocks = 0;
        int widest = 0;
        while (at < c.count && a.count < ENTRIES && blocks < MOST_SMALL) {
            const ql_matrix& q = c.mats[at];
            const int64_t n = std::min(q.batch - done, MOST_SMALL - blocks);
            if (n > 0) {
                const Shape sh = shape_of(q);
                SmallEntry& e = a.e[a.count++];
                e = {source_of(q, c.muon), target_of(q, c), sh.m, sh.n, (int32_t)blocks};
                e.s.grad = (const char*)e.s.grad + done * e.s.gb * SIZE;
                if (c.muon) e.s.momentum = (char*)e.s.momentum + done * e.s.mb * STATE;
                e.t.out = (char*)e.t.out + done * e.t.ob * SIZE;
                blocks += n;
                widest = std::max(widest, sh.n);
                lds = std::max(lds, std::is_same_v<T, double> ? small_lds(sh.m, sh.n, 8) : tiny_lds(sh.m, sh.n));
            }
            done += n;
            if (done == q.batch) at++, done = 0;
        }
        if (!blocks) continue;
        hipError_t e;
        if constexpr (std::is_same_v<T, double>) {
            static std::atomic<uint64_t> ready{0};
            e = allow_lds((const void*)k_ortho_small, ready, SMALL_LDS);
            if (e != hipSuccess) return e;
            k_ortho_small<<<(unsigned)blocks, SMALL_THREADS, lds, s>>>(a);
            e = hipGetLastError();
        } else {
            const Scales k = scales_of(c);
            // eight wavefronts hold 128 columns at once; sixteen then only wait for each other
            // (32x128 16.5 us with 8 and 19.2 with 16, 64x128 27.1 and 28.8, 600 of 64x64 48 and
            // 80), but share what is wider (8x144 15.8 and 15.0, 64x144 34.4 and 30.3, 64x256 42 and 37)
            e = widest <= 128 ? launch_tiny<T, 512>(a, (unsigned)blocks, lds, k, s) : launch_tiny<T, 1024>(a, (unsigned)blocks, lds, k, s);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

static_assert(sizeof(SmallArgs) <= 4096 && sizeof(PackArgs) <= 4096 && sizeof(GemmArgs) <= 4096, "kernel arguments");

template <typename T, int F, int MODE, int SPLIT, int BT> hipError_t gemm(GemmArgs a, const int64_t* batch, hipStream_t s) {
    int64_t blocks = 0;
    for (int k = 0; k < a.count; k++) {
        a.e[k].first = (int32_t)blocks;
        blocks += batch[k] * tiles_of(MODE, BT, a.e[k].m, a.e[k].n);
    }
    if (SPLIT == PART) blocks *= a.splits;
    constexpr int WJ = BT >= 192 ? 4 : 2, STAGES = BT == 64 ? 4 : BT == 192 ? 3 : 2;
    // only the last product sees the caller's type
    using K = std::conditional_t<MODE == LAST, T, std::conditional_t<F == TWO, float, double>>;
    k_ortho_gemm<K, F, MODE, SPLIT, BT, 2, WJ, STAGES><<<(unsigned)blocks, 128 * WJ, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int F, int MODE> hipError_t gemm(GemmArgs a, const Chunk& c, const Choice& how, hipStream_t s) {
    if constexpr (F == DOUBLE) {
        return gemm<T, F, MODE, WHOLE, 64>(a, c.batch, s);
    } else {
        if constexpr (MODE == GRAM)
            if (how.splits > 1) {
                a.splits = how.splits;
                hipError_t e = how.which ? gemm<T, F, MODE, PART, 128>(a, c.batch, s) : gemm<T, F, MODE, PART, 64>(a, c.batch, s);
                if (e != hipSuccess) return e;
                return how.which ? gemm<T, F, MODE, JOIN, 128>(a, c.batch, s) : gemm<T, F, MODE, JOIN, 64>(a, c.batch, s);
            }
        if (how.which == 1) return gemm<T, F, MODE, WHOLE, 128>(a, c.batch, s);
        if (how.which == 2) return gemm<T, F, MODE, WHOLE, 192>(a, c.batch, s);
        if (how.which == 3) return gemm<T, F, MODE, WHOLE, 256>(a, c.batch, s);
        return gemm<T, F, MODE, WHOLE, 64>(a, c.batch, s);
    }
}

template <typename T, int F> hipError_t run_steps(const OrthoCall& c, GemmArgs g, const Chunk& chunk, const Scales& k, hipStream_t s) {
    const Choice gram = choose(F, GRAM, chunk), poly = choose(F, POLY, chunk), apply = choose(F, APPLY, chunk);
    hipError_t e = hipSuccess;
    for (int step = 0; step < c.steps && e == hipSuccess; step++) {
        g.from = step & 1, g.step = step;
        g.f0 = 0, g.f1 = k.sa / (k.sx * k.sx);
        e = gemm<T, F, GRAM>(g, chunk, gram, s);
        if (e != hipSuccess) break;
        g.f0 = c.b * k.sb / k.sa, g.f1 = c.c * k.sb / (k.sa * k.sa);
        e = gemm<T, F, POLY>(g, chunk, poly, s);
        if (e != hipSuccess) break;
        if (step + 1 < c.steps) {
            g.f0 = c.a, g.f1 = 1 / k.sb;
            e = gemm<T, F, APPLY>(g, chunk, apply, s);
        } else {
            g.f0 = c.a / k.sx, g.f1 = 1 / (k.sb * k.sx);
            e = gemm<T, F, LAST>(g, chunk, apply, s);
        }
    }
    return e;
}

template <typename T, int F> hipError_t run_large(const OrthoCall& c, const Rule& rule, char* ws, hipStream_t s) {
    const Scales scales = F == DOUBLE ? Scales{} : scales_of(c);
    for (int at = 0; at < c.count;) {
        Chunk chunk;
        const ql_matrix* entry[ENTRIES];
        at = next_chunk(c.mats, c.count, at, chunk, entry);
        if (!chunk.count) break;
        PackArgs p{};
        GemmArgs g{};
        int64_t norm_blocks = 0, pack_blocks = 0;
        p.r = g.r = rule, p.scale = scales.sx, p.growth = g.growth = (float)scales.growth, p.count = g.count = chunk.count;
        for (int k = 0; k < chunk.count; k++) {
            const Shape& sh = chunk.shape[k];
            PackEntry& e = p.e[k];
            e.s = source_of(*entry[k], c.muon), e.work = ws, e.m = sh.m, e.n = sh.n, e.chunks = chunks_of(sh);
            ws += chunk.batch[k] * large_bytes(F, sh);
            e.part = (double*)ws;
            ws += chunk.batch[k] * norm_bytes(sh);
            e.first = (int32_t)norm_blocks;
            norm_blocks += chunk.batch[k] * e.chunks;
            g.e[k] = {e.work, e.part + e.chunks, target_of(*entry[k], c), sh.m, sh.n, 0, e.chunks + 1};
        }
        g.part = ws;
        ws += choose(F, GRAM, chunk).bytes;
        k_ortho_norm<T><<<(unsigned)norm_blocks, 256, 0, s>>>(p);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        for (int k = 0; k < chunk.count; k++) {
            p.e[k].first = (int32_t)pack_blocks;
            pack_blocks += chunk.batch[k] * (up64(p.e[k].m) / 64) * (up64(p.e[k].n) / 64);
        }
        k_ortho_pack<T, F><<<(unsigned)pack_blocks, 256, 0, s>>>(p);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        if (hipError_t e = run_steps<T, F>(c, g, chunk, scales, s); e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T> hipError_t run(const OrthoCall& c, void* ws, hipStream_t s) {
    Rule r{};
    r.momentum = c.momentum, r.keep = c.keep, r.eps = c.eps, r.muon = c.muon, r.nesterov = c.nesterov;
    if (all_small(c.type, c.mats, c.count)) return run_small<T>(c, r, s);
    if constexpr (std::is_same_v<T, double>) {
        return run_large<T, DOUBLE>(c, r, (char*)ws, s);
    } else {
        return run_large<T, TWO>(c, r, (char*)ws, s);
    }
}

}  // namespace

hipError_t launch_ortho(const OrthoCall& c, void* ws, hipStream_t s) {
    switch (c.type) {
        case E_F64: return run<double>(c, ws, s);
        case E_BF16: return run<bf16>(c, ws, s);
        case E_F16: return run<_Float16>(c, ws, s);
        default: return run<float>(c, ws, s);
    }
}

}  // namespace qlayer
