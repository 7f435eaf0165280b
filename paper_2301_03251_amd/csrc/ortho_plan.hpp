// ortho_plan.hpp -- how ortho.hip's kernels split a call's matrices: which run in one
// workgroup's LDS, the workspace and formats of the others, tile sizes and
// splits. Plain C++ (ortho_plan.cpp); the kernels share the layouts.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "ortho.hpp"

namespace qlayer {

constexpr int ENTRIES = 24;  // of a launch's table, which is a kernel argument (4 KiB at most)

struct Shape {
    int m, n;
    bool turned;
};
inline Shape shape_of(const ql_matrix& q) {
    const bool turned = q.rows > q.cols;
    return {(int)(turned ? q.cols : q.rows), (int)(turned ? q.rows : q.cols), turned};
}

// ---------------------------------------------------------------------------
// Small matrices: X, A and B in the LDS of one workgroup.
constexpr int SMALL_M = 64, SMALL_THREADS = 512;

constexpr int up16(int v) { return (v + 15) / 16 * 16; }
// Leading dimensions: four words past a multiple of 16, so that the 16 rows of
// an operand start in different banks.
inline size_t small_lds(int m, int n, size_t size) {
    return size * ((size_t)up16(m) * (up16(n) + 4) + 2 * (size_t)up16(m) * (up16(m) + 4));
}
constexpr int SMALL_LDS = 160 * 1024 - SMALL_THREADS / 64 * 8;  // with the norm's sums

constexpr int up32(int v) { return (v + 31) / 32 * 32; }
constexpr int PITCH = 8;  // values behind a row, so that 16 rows start in different banks
constexpr int TINY_LDS = 160 * 1024 - 1024 / 64 * 8;
inline size_t tiny_lds(int m, int n) {
    const size_t mp = up32(m), np = up32(n);
    return 4 * (mp * (np + PITCH) + np * (mp + PITCH) + mp * (mp + PITCH));
}

// Whether one workgroup's LDS holds the matrix; all of the call's.
bool is_small(int type, const Shape& s);
bool all_small(int type, const ql_matrix* mats, int count);
// Matrices of a launch: a launch's threads number less than 2^32, of 1024 at most each.
constexpr int64_t MOST_SMALL = (1 << 22) - 1;

// ---------------------------------------------------------------------------
// Large matrices in the workspace. Formats of X, A and B: two fp16 parts (32
// columns of hi, then the same 32 of lo), or fp64 for QL_F64. A row of K values
// is K * unit bytes, and 128 bytes of it are one step of a product's main loop.
//
// One part (11 bits) would serve no type: where an update has a few directions
// and little beside them, as gradients do, what a product rounds off lands in
// the small directions and is raised by 3.4 a step. bfloat16 results came out
// 12 (1500x1500) to 16 times (900x600) their own rounding off, in two parts once.
enum Format { TWO = 2, DOUBLE = 3 };
constexpr int unit_of(int format) { return format == TWO ? 4 : 8; }

// Padded sides: multiples of 64 hold whole main-loop steps of every format.
// Padding is zero: zero rows and columns of X stay zero.
constexpr int64_t up64(int64_t v) { return (v + 63) / 64 * 64; }

struct Layout {  // of one matrix's part of the workspace
    int64_t x, xt, a, b, size;  // two X^T: one is read while the other is written
};
constexpr Layout layout_of(int mp, int np, int unit) {
    const int64_t x = (int64_t)mp * np * unit, s = (int64_t)mp * mp * unit;
    return {0, x, 3 * x, 3 * x + s, 3 * x + 2 * s};
}

// Workspace of a matrix: X, A and B, then the norm's sums and X's exponent.
int64_t large_bytes(int format, const Shape& s);
int64_t norm_bytes(const Shape& s);
// Workgroups of the norm: each takes at least 4096 elements, and whole lines.
int chunks_of(const Shape& s);

struct Scales {  // powers of two that bring the largest possible values to at most 2^15
    double sx = 1, sa = 1, sb = 1;
    double growth = 0;  // log2 of what a step multiplies a singular value by at most
};
Scales scales_of(const OrthoCall& c);

// The products: C = L R^T of rows of K values, both with K along the row.
//   GRAM  A = X X^T            (tiles on and below the diagonal, written twice)
//   POLY  B = b A + c A A      (the same)
//   APPLY X = a X + B (X^T)^T, and its transpose
//   LAST  the same, to the caller's matrix
enum Mode { GRAM, POLY, APPLY, LAST };

constexpr int TILES[] = {64, 128, 192, 256};
constexpr int FOLDED = 512;  // values after which a Gram product's sums are put aside, in tiles up to 128
int64_t tiles_of(int mode, int64_t bt, int m, int n);

// The entries of a table and their batches, as the costs go by them.
struct Chunk {
    Shape shape[ENTRIES];
    int64_t batch[ENTRIES];
    int count = 0;
};

// The tile size of a launch, and for GRAM with its short sides the split of K.
struct Choice {
    int which = 0, splits = 1;
    int64_t bytes = 0;  // of the parts
};
Choice choose(int format, int mode, const Chunk& c);

// The next entries that a table holds, from `at` on; empty ones are left out.
int next_chunk(const ql_matrix* mats, int count, int at, Chunk& c, const ql_matrix** entry);

}  // namespace qlayer
