// ortho.hip -- orthogonalised updates of matrices, and the optimiser's step on them.
//
//   X = U / (|U|_F + eps), m <= n;   steps times:  A = X X^T,  B = b A + c A^2,
//   X = a X + B X.
//
// m^2 n + m^3 + 2 m^2 n operations a step (A and A^2 are symmetric: half of
// each is computed) on m n values: matrix products, bound by the matrix cores
// for all but small matrices. Those (m <= 64, and X, A and B in one workgroup's
// LDS) take one launch in fp32; all others of a call run together, tile by
// tile, in three launches a step.
//
// Products of large matrices are fp16 ones summed in fp32. The singular values
// of X stay below about 1.2 (ortho_bounds), so X, A and B are held in fp16 at
// powers of two that use its range: in two parts, v = hi + lo, for float32 and
// float16 updates (hi hi + hi lo + lo hi keeps 22 bits of every factor), and in
// one for bfloat16 (11 bits, of which the result keeps 8). fp64 uses fp64.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "elem.hpp"
#include "norm.hpp"
#include "ortho.hpp"

namespace qlayer {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef double double4v __attribute__((ext_vector_type(4)));

constexpr int ENTRIES = 24;  // of a launch's table, which is a kernel argument (4 KiB at most)

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
template <typename T>
__device__ __forceinline__ void write_out(const Target& t, const Rule& r, int64_t b, int64_t i, int64_t j, Acc<T> o) {
    T* p = (T*)t.out + b * t.ob + i * t.oi + j * t.oj;
    *p = down<T>(r.muon ? (Acc<T>)r.keep * up(*p) - (Acc<T>)t.step * o : o);
}

// The entry of a launch's table whose blocks (first[e] ..) hold this one.
template <typename E> __device__ __forceinline__ int entry_of(const E* e, int count, int block) {
    int k = 0;
    while (k + 1 < count && e[k + 1].first <= block) k++;
    return k;
}

__device__ __forceinline__ float4v mma4(float a, float b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ double4v mma4(double a, double b, double4v c) {
    return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, 0, 0, 0);
}
template <typename R> struct Quad;
template <> struct Quad<float> { using type = float4v; };
template <> struct Quad<double> { using type = double4v; };
// Where register r of lane l of a 16x16 product lies: the row (the first
// operand's); the column (the second's) is l % 16.
template <typename R> __device__ __forceinline__ int mma_row(int lane, int r) {
    return sizeof(R) == 4 ? 4 * (lane / 16) + r : lane / 16 + 4 * r;
}

// ---------------------------------------------------------------------------
// Small matrices: one workgroup each, X, A and B in its LDS, products of 16x16x4.
struct SmallEntry {
    Source s;
    Target t;
    int32_t m, n, first, batch;
};
struct SmallArgs {
    SmallEntry e[ENTRIES];
    Rule r;
    double a, b, c;
    int32_t count, steps;
};

constexpr int SMALL_M = 64, SMALL_THREADS = 512;

__host__ __device__ constexpr int up16(int v) { return (v + 15) / 16 * 16; }
// Leading dimensions: four words past a multiple of 16, so that the 16 rows of
// an operand start in different banks.
size_t small_lds(int m, int n, size_t size) {
    return size * ((size_t)up16(m) * (up16(n) + 4) + 2 * (size_t)up16(m) * (up16(m) + 4));
}
constexpr int SMALL_LDS = 160 * 1024 - SMALL_THREADS / 64 * 8;  // with the norm's sums

template <typename T> __global__ __launch_bounds__(SMALL_THREADS) void k_ortho_small(SmallArgs a) {
    using R = Acc<T>;
    using Q = typename Quad<R>::type;
    extern __shared__ double lds_small[];
    __shared__ double norm_part[SMALL_THREADS / 64];
    const SmallEntry& e = a.e[entry_of(a.e, a.count, blockIdx.x)];
    const int64_t b = blockIdx.x - e.first;
    const int m = e.m, n = e.n, mp = up16(m), np = up16(n), ldx = np + 4, lda = mp + 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = SMALL_THREADS / 64;
    R *X = (R*)lds_small, *A = X + mp * ldx, *B = A + mp * lda;

    const bool by_row = e.s.gj == 1 || e.s.gi != 1;  // the order of the addresses
    double sq = 0;
    for (int k = threadIdx.x; k < mp * np; k += SMALL_THREADS) {
        const int i = by_row ? k / np : k % mp, j = by_row ? k % np : k / mp;
        R u = 0;
        if (i < m && j < n) u = first_update<T>(e.s, a.r, b, i, j);
        X[i * ldx + j] = u;
        sq += (double)u * (double)u;
    }
    const double inv = 1.0 / (sqrt(group_sum<SMALL_THREADS>(sq, norm_part)) + a.r.eps);
    for (int k = threadIdx.x; k < mp * np; k += SMALL_THREADS) {
        R& x = X[(k / np) * ldx + k % np];
        x = (R)((double)x * inv);
    }
    __syncthreads();

    const int row = lane % 16, part = lane / 16, mt = mp / 16, nt = np / 16;
    for (int step = 0; step < a.steps; step++) {
        // A = X X^T, then B = b A + c A A: tiles on and below the diagonal, each written twice
        for (int which = 0; which < 2; which++) {
            const R *S = which ? A : X;
            R* D = which ? B : A;
            const int ld = which ? lda : ldx, depth = which ? mp : np;
            for (int t = wave; t < mt * (mt + 1) / 2; t += waves) {
                int ti = 0, tj = t;
                while (tj > ti) tj -= ++ti;
                Q acc[2] = {};
                const R *p = S + (ti * 16 + row) * ld + part, *q = S + (tj * 16 + row) * ld + part;
                for (int k = 0; k < depth; k += 8) {
                    acc[0] = mma4(p[k], q[k], acc[0]);
                    acc[1] = mma4(p[k + 4], q[k + 4], acc[1]);
                }
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const int i = ti * 16 + mma_row<R>(lane, r), j = tj * 16 + row;
                    R v = acc[0][r] + acc[1][r];
                    if (which) v = (R)a.b * A[i * lda + j] + (R)a.c * v;
                    D[i * lda + j] = v;
                    if (ti != tj) D[j * lda + i] = v;
                }
            }
            __syncthreads();
        }
        // X = a X + B X, 16 columns at a time: only their own wavefront reads or writes them
        for (int t = wave; t < nt; t += waves) {
            Q acc[SMALL_M / 16] = {};
            for (int k = 0; k < mp; k += 4) {
                const R x = X[(k + part) * ldx + t * 16 + row];
#pragma unroll
                for (int i = 0; i < SMALL_M / 16; i++)
                    if (i < mt) acc[i] = mma4(B[(i * 16 + row) * lda + k + part], x, acc[i]);
            }
#pragma unroll
            for (int i = 0; i < SMALL_M / 16; i++)
                if (i < mt)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        R& x = X[(i * 16 + mma_row<R>(lane, r)) * ldx + t * 16 + row];
                        x = (R)a.a * x + acc[i][r];
                    }
        }
        __syncthreads();
    }
    const bool out_by_row = e.t.oj == 1 || e.t.oi != 1;
    for (int k = threadIdx.x; k < m * n; k += SMALL_THREADS) {
        const int i = out_by_row ? k / n : k % m, j = out_by_row ? k % n : k / m;
        write_out<T>(e.t, a.r, b, i, j, X[i * ldx + j]);
    }
}

// ---------------------------------------------------------------------------
// Large matrices in the workspace. Formats of X, A and B: one fp16 part, two
// (32 columns of hi, then the same 32 of lo), or fp64. A row of K values is
// K * unit bytes, and 128 bytes of it are one step of a product's main loop.
enum Format { ONE = 1, TWO = 2, DOUBLE = 3 };
template <typename T> constexpr int FORMAT = std::is_same_v<T, bf16> ? ONE : std::is_same_v<T, double> ? DOUBLE : TWO;
constexpr int unit_of(int format) { return format == ONE ? 2 : format == TWO ? 4 : 8; }

// Padded sides: multiples of 64 hold whole main-loop steps of every format.
// Padding is zero: zero rows and columns of X stay zero.
constexpr int64_t up64(int64_t v) { return (v + 63) / 64 * 64; }

struct Layout {  // of one matrix's part of the workspace
    int64_t x, xt, a, b, size;  // two X^T: one is read while the other is written
};
__host__ __device__ inline Layout layout_of(int mp, int np, int unit) {
    const int64_t x = (int64_t)mp * np * unit, s = (int64_t)mp * mp * unit;
    return {0, x, 3 * x, 3 * x + s, 3 * x + 2 * s};
}

template <int F> __device__ __forceinline__ void put(char* p, int64_t row, int64_t ld, int col, double v) {
    ((double*)(p + row * ld))[col] = v;
}
template <int F> __device__ __forceinline__ void put(char* p, int64_t row, int64_t ld, int col, float v) {
    _Float16* r = (_Float16*)(p + row * ld);
    const _Float16 hi = (_Float16)v;
    if constexpr (F == ONE) {
        r[col] = hi;
    } else {
        r += col / 32 * 64 + col % 32;
        r[0] = hi;
        r[32] = (_Float16)(v - (float)hi);
    }
}
template <int F> __device__ __forceinline__ std::conditional_t<F == DOUBLE, double, float> get(const char* p, int64_t row, int64_t ld, int col) {
    if constexpr (F == DOUBLE) {
        return ((const double*)(p + row * ld))[col];
    } else {
        const _Float16* r = (const _Float16*)(p + row * ld);
        if constexpr (F == ONE) return (float)r[col];
        r += col / 32 * 64 + col % 32;
        return (float)r[0] + (float)r[32];
    }
}

struct PackEntry {
    Source s;
    char* work;    // the first matrix's part of the workspace
    double* part;  // [batch][chunks] sums of squares
    int32_t m, n, first, chunks;
};
struct PackArgs {
    PackEntry e[ENTRIES];
    Rule r;
    double scale;  // X is stored times this
    int32_t count;
};

// The momentum's step and the sums of squares, a chunk of lines each.
template <typename T> __global__ __launch_bounds__(256) void k_ortho_norm(PackArgs a) {
    __shared__ double lds[4];
    const PackEntry& e = a.e[entry_of(a.e, a.count, blockIdx.x)];
    const int at = blockIdx.x - e.first, chunk = at % e.chunks;
    const int64_t b = at / e.chunks;
    const bool by_row = e.s.gj == 1 || e.s.gi != 1;
    const int lines = by_row ? e.m : e.n, length = by_row ? e.n : e.m;
    const int l0 = (int)((int64_t)lines * chunk / e.chunks), l1 = (int)((int64_t)lines * (chunk + 1) / e.chunks);
    double sq = 0;
    for (int64_t k = threadIdx.x; k < (int64_t)(l1 - l0) * length; k += 256) {
        const int l = l0 + (int)(k / length), f = (int)(k % length);
        const Acc<T> u = first_update<T>(e.s, a.r, b, by_row ? l : f, by_row ? f : l);
        sq += (double)u * (double)u;
    }
    sq = group_sum<256>(sq, lds);
    if (threadIdx.x == 0) e.part[at] = sq;
}

// X and X^T of a 64x64 tile.
template <typename T> __global__ __launch_bounds__(256) void k_ortho_pack(PackArgs a) {
    using R = Acc<T>;
    constexpr int F = FORMAT<T>;
    __shared__ R tile[64][65];
    __shared__ double lds[4];
    const PackEntry& e = a.e[entry_of(a.e, a.count, blockIdx.x)];
    const int mp = (int)up64(e.m), np = (int)up64(e.n), ti = mp / 64, tj = np / 64;
    const int at = blockIdx.x - e.first, i0 = at / tj % ti * 64, j0 = at % tj * 64;
    const int64_t b = at / (ti * tj);
    double sq = 0;
    for (int k = threadIdx.x; k < e.chunks; k += 256) sq += e.part[b * e.chunks + k];
    const double inv = a.scale / (sqrt(group_sum<256>(sq, lds)) + a.r.eps);
    const bool by_row = e.s.gj == 1 || e.s.gi != 1;
#pragma unroll 4
    for (int k = threadIdx.x; k < 64 * 64; k += 256) {
        const int i = by_row ? k / 64 : k % 64, j = by_row ? k % 64 : k / 64;
        double u = 0;
        if (i0 + i < e.m && j0 + j < e.n) u = (double)same_update<T>(e.s, a.r, b, i0 + i, j0 + j) * inv;
        tile[i][j] = (R)u;
    }
    __syncthreads();
    const Layout l = layout_of(mp, np, unit_of(F));
    char* w = e.work + b * l.size;
    for (int k = threadIdx.x; k < 64 * 64; k += 256) {
        put<F>(w + l.x, i0 + k / 64, (int64_t)np * unit_of(F), j0 + k % 64, tile[k / 64][k % 64]);
        put<F>(w + l.xt, j0 + k / 64, (int64_t)mp * unit_of(F), i0 + k % 64, tile[k % 64][k / 64]);
    }
}

// The products: C = L R^T of rows of K values, both with K along the row.
//   GRAM  A = X X^T            (tiles on and below the diagonal, written twice)
//   POLY  B = b A + c A A      (the same)
//   APPLY X = a X + B (X^T)^T, and its transpose
//   LAST  the same, to the caller's matrix
enum Mode { GRAM, POLY, APPLY, LAST };
struct GemmEntry {
    char* work;
    Target t;
    int32_t m, n, first;
};
struct GemmArgs {
    GemmEntry e[ENTRIES];
    Rule r;
    double f0, f1;  // C is stored as f0 * (what it adds to) + f1 * (the sum)
    int32_t count, from;  // from: which X^T is read
};

template <typename T, int MODE, int BT, int WI, int WJ>
__global__ __launch_bounds__(64 * WI * WJ) void k_ortho_gemm(GemmArgs a) {
    constexpr int F = FORMAT<T>, U = unit_of(F), THREADS = 64 * WI * WJ, TI = BT / WI / 16, TJ = BT / WJ / 16;
    using R = Acc<T>;
    using Q = typename Quad<R>::type;
    __shared__ __attribute__((aligned(16))) char sl[BT * 128], sr[BT * 128];
    const GemmEntry& e = a.e[entry_of(a.e, a.count, blockIdx.x)];
    const int mp = (int)up64(e.m), np = (int)up64(e.n);
    const Layout l = layout_of(mp, np, U);
    const int64_t xt_from = l.xt + a.from * (l.a - l.xt) / 2, xt_to = l.xt + (1 - a.from) * (l.a - l.xt) / 2;
    const int mt = (mp + BT - 1) / BT, nt = (np + BT - 1) / BT;
    const int tiles = MODE <= POLY ? mt * (mt + 1) / 2 : mt * nt;
    const int t = (blockIdx.x - e.first) % tiles;
    const int64_t b = (blockIdx.x - e.first) / tiles;
    char* w = e.work + b * l.size;
    int ti, tj;
    if (MODE <= POLY) {
        ti = (int)((sqrtf(8.0f * t + 1) - 1) / 2);
        while (ti * (ti + 1) / 2 > t) ti--;
        while ((ti + 1) * (ti + 2) / 2 <= t) ti++;
        tj = t - ti * (ti + 1) / 2;
    } else {
        ti = t % mt, tj = t / mt;
    }
    const char* left = w + (MODE == GRAM ? l.x : MODE == POLY ? l.a : l.b);
    const char* right = w + (MODE == GRAM ? l.x : MODE == POLY ? l.a : xt_from);
    const int left_rows = mp, right_rows = MODE >= APPLY ? np : mp;
    const int64_t ld = (int64_t)(MODE == GRAM ? np : mp) * U;  // bytes of an operand's row

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave / WJ, wj = wave % WJ;
    const int row = lane % 16, part = lane / 16;
    Q acc[TI][TJ] = {};
    for (int64_t k = 0; k < ld; k += 128) {
        __syncthreads();
#pragma unroll
        for (int c = 0; c < BT * 8 / THREADS; c++) {
            const int id = c * THREADS + threadIdx.x, r = id / 8, q = id % 8;
            const int li = min(ti * BT + r, left_rows - 1), ri = min(tj * BT + r, right_rows - 1);
            // chunk q of row r lies at q ^ (r % 8): rows of a column of chunks in different banks
            *(float4v*)(sl + r * 128 + ((q ^ (r & 7)) * 16)) = *(const float4v*)(left + li * ld + k + q * 16);
            *(float4v*)(sr + r * 128 + ((q ^ (r & 7)) * 16)) = *(const float4v*)(right + ri * ld + k + q * 16);
        }
        __syncthreads();
        if constexpr (F == DOUBLE) {
#pragma unroll
            for (int s = 0; s < 4; s++) {
                double p[TI], q[TJ];
                const int at = s * 2 + part / 2, in = part % 2 * 8;  // value 4 s + part of the row
#pragma unroll
                for (int i = 0; i < TI; i++) {
                    const int r = wi * TI * 16 + i * 16 + row;
                    p[i] = *(const double*)(sl + r * 128 + ((at ^ (r & 7)) * 16) + in);
                }
#pragma unroll
                for (int j = 0; j < TJ; j++) {
                    const int r = wj * TJ * 16 + j * 16 + row;
                    q[j] = *(const double*)(sr + r * 128 + ((at ^ (r & 7)) * 16) + in);
                }
#pragma unroll
                for (int i = 0; i < TI; i++)
#pragma unroll
                    for (int j = 0; j < TJ; j++) acc[i][j] = mma4(q[j], p[i], acc[i][j]);
            }
        } else {
            half8 p[TI][2], q[TJ][2];
#pragma unroll
            for (int s = 0; s < 2; s++) {
                const int at = s * 4 + part;
#pragma unroll
                for (int i = 0; i < TI; i++) {
                    const int r = wi * TI * 16 + i * 16 + row;
                    p[i][s] = *(const half8*)(sl + r * 128 + ((at ^ (r & 7)) * 16));
                }
#pragma unroll
                for (int j = 0; j < TJ; j++) {
                    const int r = wj * TJ * 16 + j * 16 + row;
                    q[j][s] = *(const half8*)(sr + r * 128 + ((at ^ (r & 7)) * 16));
                }
            }
#pragma unroll
            for (int i = 0; i < TI; i++)
#pragma unroll
                for (int j = 0; j < TJ; j++) {
                    if constexpr (F == ONE) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[j][0], p[i][0], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[j][1], p[i][1], acc[i][j], 0, 0, 0);
                    } else {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[j][1], p[i][0], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[j][0], p[i][1], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[j][0], p[i][0], acc[i][j], 0, 0, 0);
                    }
                }
        }
    }
    const int64_t lda = (int64_t)mp * U, ldx = (int64_t)np * U;
#pragma unroll
    for (int i = 0; i < TI; i++)
#pragma unroll
        for (int j = 0; j < TJ; j++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const int gi = ti * BT + (wi * TI + i) * 16 + row, gj = tj * BT + (wj * TJ + j) * 16 + mma_row<R>(lane, r);
                if (gi >= left_rows || gj >= right_rows) continue;
                R v = (R)a.f1 * acc[i][j][r];
                if constexpr (MODE == GRAM) {
                    put<F>(w + l.a, gi, lda, gj, v);
                    if (ti != tj) put<F>(w + l.a, gj, lda, gi, v);
                } else if constexpr (MODE == POLY) {
                    v += (R)a.f0 * get<F>(w + l.a, gi, lda, gj);
                    put<F>(w + l.b, gi, lda, gj, v);
                    if (ti != tj) put<F>(w + l.b, gj, lda, gi, v);
                } else {
                    v += (R)a.f0 * get<F>(w + l.x, gi, ldx, gj);
                    if constexpr (MODE == APPLY) {
                        put<F>(w + l.x, gi, ldx, gj, v);
                        put<F>(w + xt_to, gj, lda, gi, v);
                    } else if (gi < e.m && gj < e.n) {
                        write_out<T>(e.t, a.r, b, gi, gj, v);
                    }
                }
            }
}

// ---------------------------------------------------------------------------
// Host side.

struct Shape {
    int m, n;
    bool turned;
};
Shape shape_of(const ql_matrix& q) {
    const bool turned = q.rows > q.cols;
    return {(int)(turned ? q.cols : q.rows), (int)(turned ? q.rows : q.cols), turned};
}

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

bool is_small(int type, const Shape& s) {
    return s.m <= SMALL_M && small_lds(s.m, s.n, type == E_F64 ? 8 : 4) <= SMALL_LDS;
}

int chunks_of(const Shape& s) {
    return (int)std::min<int64_t>(std::min(s.m, 256), std::max<int64_t>(1, (int64_t)s.m * s.n / 8192));
}

int format_of(int type) { return type == E_BF16 ? ONE : type == E_F64 ? DOUBLE : TWO; }

// Workspace of a matrix of the large route: X, A and B, then the norm's sums.
int64_t large_bytes(int type, const Shape& s) {
    return layout_of((int)up64(s.m), (int)up64(s.n), unit_of(format_of(type))).size;
}
int64_t norm_bytes(const Shape& s) { return (chunks_of(s) * 8 + 255) / 256 * 256; }

bool all_small(int type, const ql_matrix* mats, int count) {
    for (int k = 0; k < count; k++)
        if (mats[k].batch > 0 && !is_small(type, shape_of(mats[k]))) return false;
    return true;
}

template <typename T> hipError_t run_small(const OrthoCall& c, const Rule& rule, hipStream_t s) {
    for (int at = 0; at < c.count;) {
        SmallArgs a{};
        a.r = rule, a.a = c.a, a.b = c.b, a.c = c.c, a.steps = c.steps;
        size_t lds = 0;
        int64_t blocks = 0;
        for (; at < c.count && a.count < ENTRIES; at++) {
            const ql_matrix& q = c.mats[at];
            if (q.batch == 0) continue;
            const Shape sh = shape_of(q);
            if (blocks + q.batch > INT32_MAX) break;
            a.e[a.count++] = {source_of(q, c.muon), target_of(q, c), sh.m, sh.n, (int32_t)blocks, (int32_t)q.batch};
            blocks += q.batch;
            lds = std::max(lds, small_lds(sh.m, sh.n, sizeof(Acc<T>)));
        }
        if (!blocks) continue;
        // past 64 KiB the runtime wants the kernel's limit set, once on each device
        static std::atomic<uint64_t> ready{0};
        int dev = 0;
        if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
        if (dev >= 64 || !(ready.load(std::memory_order_acquire) >> dev & 1)) {
            const hipError_t e = hipFuncSetAttribute((const void*)k_ortho_small<T>, hipFuncAttributeMaxDynamicSharedMemorySize, SMALL_LDS);
            if (e != hipSuccess) return e;
            if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_release);
        }
        k_ortho_small<T><<<(unsigned)blocks, SMALL_THREADS, lds, s>>>(a);
        if (hipError_t f = hipGetLastError(); f != hipSuccess) return f;
    }
    return hipSuccess;
}

static_assert(sizeof(SmallArgs) <= 4096 && sizeof(PackArgs) <= 4096 && sizeof(GemmArgs) <= 4096, "kernel arguments");

template <typename T, int MODE, int BT> hipError_t gemm(GemmArgs a, const int64_t* batch, hipStream_t s) {
    int64_t blocks = 0;
    for (int k = 0; k < a.count; k++) {
        const int64_t mt = (up64(a.e[k].m) + BT - 1) / BT, nt = (up64(a.e[k].n) + BT - 1) / BT;
        a.e[k].first = (int32_t)blocks;
        blocks += batch[k] * (MODE <= POLY ? mt * (mt + 1) / 2 : mt * nt);
    }
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    k_ortho_gemm<T, MODE, BT, 2, 2><<<(unsigned)blocks, 256, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int BT>
hipError_t run_steps(const OrthoCall& c, GemmArgs g, const int64_t* batch, double sx, double sa, double sb, hipStream_t s) {
    hipError_t e = hipSuccess;
    for (int step = 0; step < c.steps && e == hipSuccess; step++) {
        g.from = step & 1;
        g.f0 = 0, g.f1 = sa / (sx * sx);
        e = gemm<T, GRAM, BT>(g, batch, s);
        if (e != hipSuccess) break;
        g.f0 = c.b * sb / sa, g.f1 = c.c * sb / (sa * sa);
        e = gemm<T, POLY, BT>(g, batch, s);
        if (e != hipSuccess) break;
        if (step + 1 < c.steps) {
            g.f0 = c.a, g.f1 = 1 / sb;
            e = gemm<T, APPLY, BT>(g, batch, s);
        } else {
            g.f0 = c.a / sx, g.f1 = 1 / (sb * sx);
            e = gemm<T, LAST, BT>(g, batch, s);
        }
    }
    return e;
}

template <typename T> hipError_t run_large(const OrthoCall& c, const Rule& rule, char* ws, hipStream_t s) {
    // powers of two that bring the largest possible values to at most 2^15
    double sx = 1, sa = 1, sb = 1;
    if (FORMAT<T> != DOUBLE) {
        double most_x = 1, most_q = 1;
        ortho_bounds(c.a, c.b, c.c, c.steps, most_x, most_q);
        sx = std::exp2(std::floor(std::log2(32768 / most_x)));
        sa = std::exp2(std::floor(std::log2(32768 / (most_x * most_x))));
        sb = std::exp2(std::floor(std::log2(32768 / std::max(most_q, 1e-3))));
    }
    for (int at = 0; at < c.count;) {
        PackArgs p{};
        GemmArgs g{};
        int64_t batch[ENTRIES], norm_blocks = 0, tiles128 = 0;
        p.r = g.r = rule, p.scale = sx;
        for (; at < c.count && p.count < ENTRIES; at++) {
            const ql_matrix& q = c.mats[at];
            if (q.batch == 0) continue;
            const Shape sh = shape_of(q);
            PackEntry& e = p.e[p.count];
            e.s = source_of(q, c.muon), e.work = ws, e.m = sh.m, e.n = sh.n, e.chunks = chunks_of(sh);
            ws += q.batch * large_bytes(c.type, sh);
            e.part = (double*)ws;
            ws += q.batch * norm_bytes(sh);
            e.first = (int32_t)norm_blocks;
            norm_blocks += q.batch * e.chunks;
            g.e[p.count] = {e.work, target_of(q, c), sh.m, sh.n, 0};
            batch[p.count++] = q.batch;
            tiles128 += q.batch * ((sh.m + 127) / 128) * ((sh.n + 127) / 128);
        }
        if (!p.count) continue;
        g.count = p.count;
        if (norm_blocks > INT32_MAX) return hipErrorInvalidValue;
        k_ortho_norm<T><<<(unsigned)norm_blocks, 256, 0, s>>>(p);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        int64_t pack_blocks = 0;
        for (int k = 0; k < p.count; k++) {
            p.e[k].first = (int32_t)pack_blocks;
            pack_blocks += batch[k] * (up64(p.e[k].m) / 64) * (up64(p.e[k].n) / 64);
        }
        if (pack_blocks > INT32_MAX) return hipErrorInvalidValue;
        k_ortho_pack<T><<<(unsigned)pack_blocks, 256, 0, s>>>(p);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        hipError_t e;
        if constexpr (FORMAT<T> == DOUBLE) e = run_steps<T, 64>(c, g, batch, sx, sa, sb, s);
        else e = tiles128 >= 256 ? run_steps<T, 128>(c, g, batch, sx, sa, sb, s) : run_steps<T, 64>(c, g, batch, sx, sa, sb, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T> hipError_t run(const OrthoCall& c, void* ws, hipStream_t s) {
    Rule r{};
    r.momentum = c.momentum, r.keep = c.keep, r.eps = c.eps, r.muon = c.muon, r.nesterov = c.nesterov;
    return all_small(c.type, c.mats, c.count) ? run_small<T>(c, r, s) : run_large<T>(c, r, (char*)ws, s);
}

}  // namespace

bool ortho_bounds(double a, double b, double c, int steps, double& most_x, double& most_q) {
    most_x = 1, most_q = 0;
    double reach = 1;  // singular values lie in [0, reach]
    for (int s = 0; s < steps; s++) {
        double next = 0;
        for (int k = 0; k <= 1024; k++) {  // a margin of 1/256 covers what lies between two values
            const double x = reach * k / 1024, q = x * x * (b + c * x * x), v = std::fabs(x * (a + q));
            if (!(v <= 1e6) || !(std::fabs(q) <= 1e5)) return false;
            next = std::max(next, v);
            most_q = std::max(most_q, std::fabs(q));
        }
        if (s + 1 == steps) break;  // what the last step gives is not held
        reach = next * (1 + 1.0 / 256);
        most_x = std::max(most_x, reach);
        if (reach > 64) return false;
    }
    return true;
}

size_t ortho_workspace(int type, const ql_matrix* mats, int count) {
    if (all_small(type, mats, count)) return 0;
    int64_t bytes = 0;
    for (int k = 0; k < count; k++) {
        const Shape s = shape_of(mats[k]);
        bytes += mats[k].batch * (large_bytes(type, s) + norm_bytes(s));
    }
    return (size_t)bytes;
}

hipError_t launch_ortho(const OrthoCall& c, void* ws, hipStream_t s) {
    switch (c.type) {
        case E_F64: return run<double>(c, ws, s);
        case E_BF16: return run<bf16>(c, ws, s);
        case E_F16: return run<_Float16>(c, ws, s);
        default: return run<float>(c, ws, s);
    }
}

}  // namespace qlayer
