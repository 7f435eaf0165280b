// scan.hip -- gated linear recurrence over the steps of sequences, forward,
// backward and one step.
//
//   a_t = 1 / (1 + exp(-z_t)),  h_t = a_t h_{t-1} + (1 - a_t) x_t
//   G_t = g_t + a_{t+1} G_{t+1},  dx_t = (1 - a_t) G_t,
//   dz_t = G_t (h_{t-1} - x_t) a_t (1 - a_t),  dh_{-1} = a_0 G_0
//
// Where a sequence starts, h_{t-1} is 0 and nothing of G_t goes back past it. It is
// chosen, not multiplied by 0: what another sequence held (infinities, NaN) does not come in.
//
// A step is the map h -> a h + b, and a row of steps one such map again: (A, B) then
// (a, b) is (a A, a B + b). So the steps go in blocks of 16, one a wavefront, with a
// column (sequence and feature) a lane: a wavefront reads its block into registers and
// makes its map, the workgroup's wavefronts exchange maps through LDS, and each runs
// its block again from the state before it. Arrays are read once. Where there are
// fewer columns than fill the chip, the steps are split into segments: a launch
// makes the segments' maps, which reads what they need a second time, and the main
// launch begins each segment with the maps before it.
//
// Backward the maps run from the end, of what comes back to a step, and the states
// h_{t-1} are computed again from the one that the forward call kept before each
// block (in fp32: 1/16 of an array's elements).
//
// HBM bounds long calls; about 25 operations an element forward and 45 backward
// come next.
#include <algorithm>
#include <type_traits>

#include "elem.hpp"
#include "scan.hpp"

namespace qlayer {
namespace {

constexpr int L = SCAN_BLOCK;

// The wavefront's number, known to be the same in its lanes.
__device__ __forceinline__ int wavefront() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// a = sigmoid(z) and 1 - a, neither as a difference from 1.
__device__ __forceinline__ void gates(float z, float& a, float& rest) {
    const float e = __builtin_amdgcn_exp2f(-1.44269504f * fabsf(z)), r = __builtin_amdgcn_rcpf(1 + e);
    a = z >= 0 ? r : e * r, rest = z >= 0 ? e * r : r;
}
__device__ __forceinline__ void gates(double z, double& a, double& rest) {
    const double e = exp(-fabs(z)), r = 1 / (1 + e);
    a = z >= 0 ? r : e * r, rest = z >= 0 ? e * r : r;
}

// The map of a row of steps. Where sequences may start in it, A < 0 is a cut: the
// state is B whatever it was before.
template <typename R, bool STARTS> struct Map {
    R A, B;
    __device__ __forceinline__ R operator()(R h) const { return STARTS && A < 0 ? B : A * h + B; }
    // this one, then m
    __device__ __forceinline__ void then(const Map& m) {
        B = m(B);
        A = STARTS && (m.A < 0 || A < 0) ? (R)-1 : A * m.A;
    }
};

// A lane's column. The workgroup's first sequence gives the address that all lanes
// share, and a lane adds the bytes from there to its own column (OFF: 32 bits where
// they fit, which leaves one register and one instruction to an access).
struct Column {
    bool live;
    int64_t at, batch, first, d;  // among all columns; its sequence, the workgroup's first one, its feature
    __device__ __forceinline__ Column(const ScanArgs& a) {
        const int64_t c0 = (int64_t)blockIdx.x * 64, c = c0 + (threadIdx.x & 63), n = a.batch * a.D;
        live = c < n, at = min(c, n - 1), first = c0 / a.D;
        batch = first, d = at - first * a.D;
        if (d >= a.D) batch = at / a.D, d = at % a.D;
    }
};

// An array's column. Rows (steps) are walked with an address in scalar registers,
// which the compiler must not fold into the lanes' own: an access then is that
// address and the lane's bytes.
typedef __attribute__((address_space(1))) char* Row;

template <typename T, typename OFF> struct Lane {
    Row base;
    int64_t step;  // bytes
    OFF off;
    __device__ __forceinline__ Lane(const Column& c, const Strided& s) : Lane(c, s.p, s.batch, s.step) {}
    __device__ __forceinline__ Lane(const Column& c, const void* p, int64_t batch, int64_t step_)
        : base((Row)p + c.first * batch * (int64_t)sizeof(T)),
          step(step_ * (int64_t)sizeof(T)),
          off((OFF)(((c.batch - c.first) * batch + c.d) * (int64_t)sizeof(T))) {}
    __device__ __forceinline__ Row row(int t) const { return base + t * step; }
    // the lane's bytes as the compiler finds them anew where a block's accesses begin
    __device__ __forceinline__ OFF here() const {
        OFF o = off;
        asm("" : "+v"(o));
        return o;
    }
    using Bits = std::conditional_t<sizeof(T) == 2, uint16_t, std::conditional_t<sizeof(T) == 4, uint32_t, uint64_t>>;
    using Place = __attribute__((address_space(1))) Bits*;
    __device__ __forceinline__ T load(Row row, OFF o) const {
        asm("" : "+s"(row));
        return __builtin_bit_cast(T, *(Place)(row + o));
    }
    __device__ __forceinline__ void store(Row row, OFF o, T v) const {
        asm("" : "+s"(row));
        *(Place)(row + o) = __builtin_bit_cast(Bits, v);
    }
};

// The steps of block k that start a sequence, as bits.
template <bool STARTS> __device__ __forceinline__ uint32_t starts_of(const ScanArgs& a, const Column& c, int k, int steps) {
    uint32_t bits = 0;
    if constexpr (STARTS) {
        const uint8_t* s = a.starts + c.batch * a.steps;
#pragma unroll
        for (int j = 0; j < L; j++) {
            const int t = k * L + j;
            bits |= (uint32_t)(s[min(t, steps - 1)] != 0 && t < steps) << j;
        }
    }
    return bits;
}

// Block k's elements of a column; past the end the last step's, which the caller leaves out.
template <typename T, typename OFF>
__device__ __forceinline__ void load_block(T (&v)[L], const Lane<T, OFF>& p, int k, int steps) {
    const OFF o = p.here();
    if (steps - k * L >= L) {
        Row row = p.row(k * L);
#pragma unroll
        for (int j = 0; j < L; j++, row += p.step) v[j] = p.load(row, o);
    } else {
#pragma unroll
        for (int j = 0; j < L; j++) v[j] = p.load(p.row(min(k * L + j, steps - 1)), o);
        asm volatile("");  // the two ways stay apart: their addresses would not fit the scalar registers
    }
}

// Steps past the end leave the state as it is.
template <typename R> __device__ __forceinline__ void leave_out(int left, R (&f)[L], R (&b)[L]) {
    if (left >= L) return;
#pragma unroll
    for (int j = 0; j < L; j++)
        if (j >= left) f[j] = 1, b[j] = 0;
}

// The map of a forward block, and its factors.
template <typename T, bool STARTS, typename R>
__device__ __forceinline__ Map<R, STARTS> forward_map(const T (&x)[L], const T (&z)[L], uint32_t starts, int left, R (&f)[L], R (&b)[L]) {
    Map<R, STARTS> m{1, 0};
    bool cut = false;
#pragma unroll
    for (int j = 0; j < L; j++) {
        R rest;
        gates(up(z[j]), f[j], rest);
        b[j] = rest * up(x[j]);
    }
    leave_out(left, f, b);
#pragma unroll
    for (int j = 0; j < L; j++) {
        if (STARTS && ((starts >> j) & 1)) m.B = b[j], cut = true;
        else m.B = f[j] * m.B + b[j];
        m.A *= f[j];
    }
    if (cut) m.A = -1;
    return m;
}

// The map of a backward block, last step first, of what comes back to a step.
template <bool STARTS, typename R>
__device__ __forceinline__ Map<R, STARTS> backward_map(const R (&f)[L], const R (&g)[L], uint32_t starts) {
    Map<R, STARTS> m{1, 0};
    bool cut = false;
#pragma unroll
    for (int j = L - 1; j >= 0; j--) {
        if (STARTS && ((starts >> j) & 1)) m.B = 0, cut = true;
        else m.B = f[j] * (m.B + g[j]);
        m.A *= f[j];
    }
    if (cut) m.A = -1;
    return m;
}

// Where the segment begins: the maps of the segments that come before it, each
// wavefront a share of them, on the state that the row begins with.
template <int W, bool STARTS, typename R>
__device__ __forceinline__ R begin_segment(R state, const R* maps, int64_t columns, int64_t column, int first, int count, int dir, R (&A)[W][64], R (&B)[W][64]) {
    const int wave = wavefront(), lane = threadIdx.x & 63, each = (count + W - 1) / W;
    Map<R, STARTS> m{1, 0};
#pragma unroll 4
    for (int i = wave * each; i < min(count, (wave + 1) * each); i++) {
        const R* p = maps + (int64_t)(first + dir * i) * 2 * columns + column;
        m.then(Map<R, STARTS>{p[0], p[columns]});
    }
    A[wave][lane] = m.A, B[wave][lane] = m.B;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; w++) state = Map<R, STARTS>{A[w][lane], B[w][lane]}(state);
    __syncthreads();
    return state;
}

template <typename T, typename OFF, int W, bool STARTS> __global__ __launch_bounds__(64 * W) void k_scan_fwd(ScanArgs a, int blocks, int each) {
    using R = Acc<T>;
    __shared__ R A[2][W][64], B[2][W][64];
    const int wave = wavefront(), lane = threadIdx.x & 63;
    const Column c(a);
    const Lane<T, OFF> x(c, a.x), z(c, a.gate), out(c, a.h, a.steps * a.D, a.D);
    const Lane<R, OFF> kept(c, a.states, blocks * a.D, a.D);
    const int steps = (int)a.steps, k0 = blockIdx.y * each, k1 = min(k0 + each, blocks);
    R state = a.initial ? ((const R*)a.initial)[c.at] : 0;
    if (blockIdx.y > 0) state = begin_segment<W, STARTS, R>(state, (const R*)a.ws, a.batch * a.D, c.at, 0, blockIdx.y, 1, A[0], B[0]);
    int turn = 0;
    T vx[L], vz[L];
    if (k0 < k1) load_block(vx, x, k0 + wave, steps), load_block(vz, z, k0 + wave, steps);
    for (int base = k0; base < k1; base += W, turn ^= 1) {
        const int k = base + wave, left = k < k1 ? steps - k * L : 0;
        const uint32_t starts = left > 0 ? starts_of<STARTS>(a, c, k, steps) : 0;
        R f[L], b[L];
        const Map<R, STARTS> m = forward_map<T, STARTS, R>(vx, vz, starts, left, f, b);
        // the next block is under way while this one is finished
        if (base + W < k1) load_block(vx, x, k + W, steps), load_block(vz, z, k + W, steps);
        A[turn][wave][lane] = m.A, B[turn][wave][lane] = m.B;
        __syncthreads();
        R h = state;
#pragma unroll
        for (int w = 0; w < W; w++) {
            if (w == wave) h = state;
            state = Map<R, STARTS>{A[turn][w][lane], B[turn][w][lane]}(state);
        }
        if (left <= 0 || !c.live) continue;
        if (a.states) kept.store(kept.row(k), kept.here(), h);
        auto apply = [&](auto whole) {
            Row row = out.row(k * L);
            const OFF o = out.here();
#pragma unroll
            for (int j = 0; j < L; j++, row += out.step) {
                h = STARTS && ((starts >> j) & 1) ? b[j] : f[j] * h + b[j];
                if (decltype(whole)::value || j < left) out.store(row, o, down<T>(h));
            }
        };
        if (left >= L) apply(std::true_type{});
        else apply(std::false_type{});
    }
    if (a.last && k1 == blocks && wave == 0 && c.live) ((R*)a.last)[c.at] = state;
}

// ws[segment][2][columns]: the segments' maps, forward or backward.
template <typename T, typename OFF, int W, bool STARTS, bool BACK>
__global__ __launch_bounds__(64 * W) void k_scan_maps(ScanArgs a, int blocks, int each) {
    using R = Acc<T>;
    __shared__ R A[W][64], B[W][64];
    const int wave = wavefront(), lane = threadIdx.x & 63;
    const Column c(a);
    const Lane<T, OFF> v(c, BACK ? a.grad : a.x), z(c, a.gate);
    const int steps = (int)a.steps, k0 = blockIdx.y * each, k1 = min(k0 + each, blocks), share = (each + W - 1) / W;
    // wavefront 0 has the blocks that come first in the maps' direction
    const int n = k1 - k0, i0 = min(wave * share, n), i1 = min(i0 + share, n);
    Map<R, STARTS> m{1, 0};
    for (int i = i0; i < i1; i++) {
        const int k = BACK ? k1 - 1 - i : k0 + i, left = steps - k * L;
        T vv[L], vz[L];
        load_block(vv, v, k, steps);
        load_block(vz, z, k, steps);
        const uint32_t starts = starts_of<STARTS>(a, c, k, steps);
        R f[L], b[L];
        if constexpr (BACK) {
#pragma unroll
            for (int j = 0; j < L; j++) {
                R rest;
                gates(up(vz[j]), f[j], rest);
                b[j] = up(vv[j]);
            }
            leave_out(left, f, b);
            m.then(backward_map<STARTS, R>(f, b, starts));
        } else {
            m.then(forward_map<T, STARTS, R>(vv, vz, starts, left, f, b));
        }
    }
    A[wave][lane] = m.A, B[wave][lane] = m.B;
    __syncthreads();
    if (wave > 0 || !c.live) return;
#pragma unroll
    for (int w = 1; w < W; w++) m.then(Map<R, STARTS>{A[w][lane], B[w][lane]});
    R* out = (R*)a.ws + (int64_t)blockIdx.y * 2 * a.batch * a.D + c.at;
    out[0] = m.A, out[a.batch * a.D] = m.B;
}

template <typename T, typename OFF, int W, bool STARTS> __global__ __launch_bounds__(64 * W) void k_scan_bwd(ScanArgs a, int blocks, int each) {
    using R = Acc<T>;
    __shared__ R A[2][W][64], B[2][W][64];
    const int wave = wavefront(), lane = threadIdx.x & 63;
    const Column c(a);
    const Lane<T, OFF> x(c, a.x), z(c, a.gate), g(c, a.grad);
    const Lane<T, OFF> dx(c, a.grad_x, a.steps * a.D, a.D), dz(c, a.grad_gate, a.steps * a.D, a.D);
    const Lane<R, OFF> kept(c, a.states, blocks * a.D, a.D);
    const int steps = (int)a.steps, k0 = blockIdx.y * each, k1 = min(k0 + each, blocks);
    const int behind = gridDim.y - 1 - blockIdx.y;
    R back = a.grad_last ? ((const R*)a.grad_last)[c.at] : 0;
    if (behind > 0) back = begin_segment<W, STARTS, R>(back, (const R*)a.ws, a.batch * a.D, c.at, gridDim.y - 1, behind, -1, A[0], B[0]);
    int turn = 0;
    T vx[L], vz[L], vg[L];
    R nh = 0;
    auto fetch = [&](int top) {
        const int k = max(top - 1 - wave, k0);
        load_block(vx, x, k, steps);
        load_block(vz, z, k, steps);
        load_block(vg, g, k, steps);
        nh = kept.load(kept.row(k), kept.here());
    };
    // fp64 has no registers for a second block
    constexpr bool AHEAD = sizeof(T) < 8;
    if (AHEAD && k1 > k0) fetch(k1);
    for (int top = k1; top > k0; top -= W, turn ^= 1) {
        const int k = max(top - 1 - wave, k0), left = top - 1 - wave >= k0 ? steps - k * L : 0;
        if constexpr (!AHEAD) fetch(top);
        R h = nh;
        const uint32_t starts = left > 0 ? starts_of<STARTS>(a, c, k, steps) : 0;
        // f = a, r = 1 - a, q = dz / G, b = g
        R f[L], r[L], q[L], b[L];
        // one after the other, which keeps to the registers of four wavefronts a SIMD
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < L; j++) {
            gates(up(vz[j]), f[j], r[j]);
            if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int j = 0; j < L; j++) {
            const R v = up(vx[j]), before = STARTS && ((starts >> j) & 1) ? 0 : h;
            q[j] = (before - v) * (f[j] * r[j]);
            h = f[j] * before + r[j] * v;
            b[j] = up(vg[j]);
        }
        leave_out(left, f, b);
        const Map<R, STARTS> m = backward_map<STARTS, R>(f, b, starts);
        // the next block is under way while this one is finished
        if (AHEAD && top - W > k0) fetch(top - W);
        A[turn][wave][lane] = m.A, B[turn][wave][lane] = m.B;
        __syncthreads();
        R s = back;
#pragma unroll 4  // all eight at once: 153 us for 149 at 8x4096x2048 bfloat16, 17.7 for 19.0 at 64x256x256 float32
        for (int w = 0; w < W; w++) {
            if (w == wave) s = back;
            back = Map<R, STARTS>{A[turn][w][lane], B[turn][w][lane]}(back);
        }
        if (left <= 0 || !c.live) continue;
        auto apply = [&](auto whole) {
            Row row_x = dx.row(k * L + L - 1), row_z = dz.row(k * L + L - 1);
            const OFF o = dx.here();
#pragma unroll
            for (int j = L - 1; j >= 0; j--, row_x -= dx.step, row_z -= dz.step) {
                const R G = b[j] + s;
                s = STARTS && ((starts >> j) & 1) ? 0 : f[j] * G;
                if (decltype(whole)::value || j < left) {
                    dx.store(row_x, o, down<T>(r[j] * G));
                    dz.store(row_z, o, down<T>(q[j] * G));
                }
            }
        };
        if (left >= L) apply(std::true_type{});
        else apply(std::false_type{});
    }
    if (a.grad_initial && k0 == 0 && wave == 0 && c.live) ((R*)a.grad_initial)[c.at] = back;
}

// One step: V elements a thread.
template <typename T, int V> __global__ __launch_bounds__(256) void k_scan_step(ScanArgs a, void* state) {
    using R = Acc<T>;
    const int64_t per = a.D / V, n = a.batch * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t b = i / per, d = (i % per) * V;
        const Vec<T, V> x = load_vec<T, V>((const T*)a.x.p + b * a.x.batch + d);
        const Vec<T, V> z = load_vec<T, V>((const T*)a.gate.p + b * a.gate.batch + d);
        Vec<R, V> s = load_vec<R, V>((const R*)state + b * a.D + d);
        const bool start = a.starts && a.starts[b];
        Vec<T, V> h;
#pragma unroll
        for (int e = 0; e < V; e++) {
            R f, rest;
            gates(up(z.v[e]), f, rest);
            const R in = rest * up(x.v[e]);
            s.v[e] = start ? in : f * s.v[e] + in;
            h.v[e] = down<T>(s.v[e]);
        }
        store_vec<R, V>((R*)state + b * a.D + d, s);
        store_vec<T, V>((T*)a.h + b * a.D + d, h);
    }
}

// How a call is split: wavefronts of a workgroup, blocks of a segment, segments.
struct Split {
    int waves;
    int64_t groups, blocks, each, segments;
};
// Wavefronts of a workgroup, which leave a block its registers and the next one's (of
// 16 they are as fast forward: 97 us for 94 at 8x4096x2048 bfloat16, 20.4 for 22.6
// at 1x65536x64 float32; backward there is no room for the next block, 161 for 144).
constexpr int WAVES = 8;

Split split_of(int64_t batch, int64_t steps, int64_t D) {
    Split p{};
    p.groups = (batch * D + 63) / 64;
    p.blocks = (steps + L - 1) / L;
    p.waves = p.blocks <= 1 ? 1 : p.blocks <= 4 ? 4 : WAVES;
    const int64_t turns = std::max<int64_t>(1, (p.blocks + p.waves - 1) / p.waves);
    // segments of whole turns, at most 256 workgroups, one a compute unit: the maps
    // read x and gate (gate and grad) once more, so no more (8x4096x2048 bfloat16, 256
    // groups: 94 and 144 us in one segment, 155 and 204 in two; 1x65536x64 float32, one
    // group: 47 us forward and backward in 256 segments, 58 in 512). Between those two
    // the rule is not measured: 129 to 255 groups have one segment
    const int64_t want = std::min<int64_t>(turns, std::max<int64_t>(1, 256 / p.groups));
    p.each = (turns + want - 1) / want * p.waves;
    p.segments = std::max<int64_t>(1, (p.blocks + p.each - 1) / p.each);
    return p;
}

template <typename T, typename OFF, int W, bool STARTS, bool BACK> hipError_t run(const ScanArgs& a, const Split& p, hipStream_t s) {
    const dim3 grid((unsigned)p.groups, (unsigned)p.segments);
    const int blocks = (int)p.blocks, each = (int)p.each;
    if (p.segments > 1) k_scan_maps<T, OFF, W, STARTS, BACK><<<grid, 64 * W, 0, s>>>(a, blocks, each);
    if constexpr (BACK) k_scan_bwd<T, OFF, W, STARTS><<<grid, 64 * W, 0, s>>>(a, blocks, each);
    else k_scan_fwd<T, OFF, W, STARTS><<<grid, 64 * W, 0, s>>>(a, blocks, each);
    return hipGetLastError();
}

// Whether the bytes from a workgroup's first sequence to any of its columns fit 32 bits.
bool near_by(const ScanArgs& a, int size, int wide) {
    const int64_t most = ((int64_t)1 << 32) - 1, sequences = std::min(a.batch - 1, 63 / a.D + 1);
    auto fits = [&](int64_t batch, int bytes) { return batch <= (most / bytes - a.D) / std::max<int64_t>(sequences, 1); };
    return fits(a.x.batch, size) && fits(a.gate.batch, size) && fits(a.grad.batch, size) && fits(a.steps * a.D, size) &&
           fits((a.steps + L - 1) / L * a.D, wide);
}

template <typename T, bool STARTS, bool BACK> hipError_t run(const ScanArgs& a, const Split& p, hipStream_t s) {
    if (!near_by(a, sizeof(T), sizeof(Acc<T>))) {
        switch (p.waves) {
            case 1: return run<T, uint64_t, 1, STARTS, BACK>(a, p, s);
            case 4: return run<T, uint64_t, 4, STARTS, BACK>(a, p, s);
            default: return run<T, uint64_t, WAVES, STARTS, BACK>(a, p, s);
        }
    }
    switch (p.waves) {
        case 1: return run<T, uint32_t, 1, STARTS, BACK>(a, p, s);
        case 4: return run<T, uint32_t, 4, STARTS, BACK>(a, p, s);
        default: return run<T, uint32_t, WAVES, STARTS, BACK>(a, p, s);
    }
}

// Vectors where no step passes a row's end: the state changes in place, so no two
// lanes may share an element.
template <typename T> hipError_t step(const ScanArgs& a, void* state, hipStream_t s) {
    constexpr int V = 16 / (int)sizeof(T);
    const bool whole = a.D % V == 0;
    const int64_t n = a.batch * (whole ? a.D / V : a.D);
    const unsigned grid = (unsigned)std::min<int64_t>((n + 255) / 256, 1 << 20);
    if (whole) k_scan_step<T, V><<<grid, 256, 0, s>>>(a, state);
    else k_scan_step<T, 1><<<grid, 256, 0, s>>>(a, state);
    return hipGetLastError();
}

template <typename F> hipError_t by_type(int type, F f) {
    switch (type) {
        case E_F64: return f(double{});
        case E_BF16: return f(bf16{});
        case E_F16: return f(_Float16{});
        default: return f(float{});
    }
}

hipError_t launch(int type, const ScanArgs& a, bool back, hipStream_t s) {
    if (a.batch == 0) return hipSuccess;
    const Split p = split_of(a.batch, a.steps, a.D);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        if (back) return a.starts ? run<T, true, true>(a, p, s) : run<T, false, true>(a, p, s);
        return a.starts ? run<T, true, false>(a, p, s) : run<T, false, false>(a, p, s);
    });
}

}  // namespace

size_t scan_workspace(int type, int64_t batch, int64_t steps, int64_t D) {
    if (batch == 0) return 0;
    const int64_t segments = split_of(batch, steps, D).segments;
    return segments > 1 ? (size_t)(segments * 2 * batch * D) * (type == E_F64 ? 8 : 4) : 0;
}

hipError_t launch_scan_forward(int type, const ScanArgs& a, hipStream_t s) { return launch(type, a, false, s); }
hipError_t launch_scan_backward(int type, const ScanArgs& a, hipStream_t s) { return launch(type, a, true, s); }

hipError_t launch_scan_step(int type, const ScanArgs& a, void* state, hipStream_t s) {
    if (a.batch == 0) return hipSuccess;
    return by_type(type, [&](auto t) { return step<decltype(t)>(a, state, s); });
}

}  // namespace qlayer
