// embed.hip -- rows of a table for tokens, times a scale, and the table's gradient.
//
//   y_i = scale W[t_i],   dW[v] = scale sum over i with t_i = v of g_i
//
// Tokens that are the padding have a row of zeros and no gradient. One outside the
// table has a row of NaN, as nothing on the host sees it, and no gradient.
//
// How the gradient's sums are put together follows from the call's tokens, not from the
// grid: places are sorted by token (a stable radix sort), and a wavefront sums the
// rows of a chunk of sorted places, token by token, in the order of their places. A
// token whose rows end in the chunk or the next is done there; of one that goes on
// further the parts are joined in a second launch, every fourth by one wavefront and
// then the four. Chunks are cut from the whole list: with other tokens in the call a
// token's rows may be split elsewhere, and its sum rounded otherwise. Rows without
// tokens are zeros, written beside the sort. HBM bounds large calls (N rows of g read,
// the table written), launches the others.
#include <algorithm>

#include "elem.hpp"
#include "embed.hpp"

namespace qlayer {
namespace {

template <typename T> constexpr int VEC = 16 / (int)sizeof(T);

__device__ __forceinline__ int64_t token_at(const EmbedArgs& a, int64_t i) {
    return a.wide ? ((const int64_t*)a.tokens)[i] : (int64_t)((const int32_t*)a.tokens)[i];
}

// A group of G lanes copies K vectors a lane of token after token's row (a tile of
// it where it is longer): the next row's loads and the token behind it are under way
// while a row is written.
template <typename T, int V, int G, int K> __global__ __launch_bounds__(256) void k_embed_fwd(EmbedArgs a) {
    using R = Acc<T>;
    constexpr int GROUPS = 256 / G;
    const int lane = threadIdx.x % G, D = (int)a.D, tiles = (D + G * V * K - 1) / (G * V * K);
    const R scale = (R)a.scale;
    const int64_t stride = (int64_t)gridDim.x * GROUPS, count = a.n * tiles;
    int64_t w = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G;
    if (w >= count) return;
    auto token = [&](int64_t w) { return token_at(a, min(w, count - 1) / tiles); };
    auto column = [&](int64_t w, int k) { return min(((int)(w % tiles) * G * K + k * G + lane) * V, D - V); };
    Vec<T, V> next[K];
    auto fetch = [&](int64_t w, int64_t t) {
        const T* src = (const T*)a.weight + (t >= 0 && t < a.rows ? t : 0) * a.weight_stride;
#pragma unroll
        for (int k = 0; k < K; k++) next[k] = load_vec<T, V>(src + column(w, k));
    };
    int64_t t = token(w), ahead = token(w + stride);
    fetch(w, t);
    for (; w < count; w += stride) {
        Vec<T, V> v[K];
#pragma unroll
        for (int k = 0; k < K; k++) v[k] = next[k];
        if (w + stride < count) fetch(w + stride, ahead);
        const bool pad = a.padded && t == a.padding, in = t >= 0 && t < a.rows;
        T* dst = (T*)a.y + w / tiles * a.D;
#pragma unroll
        for (int k = 0; k < K; k++) {
#pragma unroll
            for (int e = 0; e < V; e++)
                v[k].v[e] = down<T>(pad ? (R)0 : in ? up(v[k].v[e]) * scale : (R)__builtin_nanf(""));
            store_vec<T, V>(dst + column(w, k), v[k]);
        }
        t = ahead, ahead = token(w + 2 * stride);
    }
}

// ---------------------------------------------------------------------------
// The sort: keys (the token; `rows` for what has no gradient) with their places.

__device__ __forceinline__ uint32_t key_at(const EmbedArgs& a, int64_t i) {
    const int64_t t = token_at(a, i);
    return t < 0 || t >= a.rows || (a.padded && t == a.padding) ? (uint32_t)a.rows : (uint32_t)t;
}

// Zeros for the whole table: share `part` of `parts`.
template <typename T> __device__ void clear_table(const EmbedArgs& a, int64_t part, int64_t parts) {
    constexpr int V = VEC<T>;
    const int64_t n = a.rows * a.D, vectors = n / V, each = (vectors + parts - 1) / parts;
    const int64_t end = min(vectors, (part + 1) * each);
    T* out = (T*)a.grad_weight;
    Vec<T, V> zero;
#pragma unroll
    for (int e = 0; e < V; e++) zero.v[e] = down<T>((Acc<T>)0);
    for (int64_t i = part * each + threadIdx.x; i < end; i += blockDim.x) store_vec<T, V>(out + i * V, zero);
    if (part == 0 && threadIdx.x < n % V) out[vectors * V + threadIdx.x] = zero.v[0];
}

// The lanes of the wavefront with the same digit, of those that take part.
__device__ __forceinline__ uint64_t lanes_alike(uint32_t digit, int bits, bool takes_part) {
    uint64_t m = __ballot(takes_part);
    for (int b = 0; b < bits; b++) {
        const uint64_t has = __ballot((digit >> b) & 1);
        m &= (digit >> b) & 1 ? has : ~has;
    }
    return m;
}

// Where an element comes among its wavefront's with its digit, which `counts` counts on.
__device__ __forceinline__ uint32_t rank_of(uint32_t digit, int bits, bool takes_part, uint32_t* counts) {
    const int lane = threadIdx.x & 63;
    const uint64_t alike = lanes_alike(digit, bits, takes_part);
    const int first = takes_part ? __ffsll((unsigned long long)alike) - 1 : lane;
    uint32_t before = 0;
    if (takes_part && lane == first) before = atomicAdd(&counts[digit], (uint32_t)__popcll(alike));
    before = __shfl(before, first, 64);
    return before + (uint32_t)__popcll(alike & ((1ull << lane) - 1));
}

// Sum of the values before the thread's own over a workgroup of T threads.
template <int T> __device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t* lds) {
    const int lane = threadIdx.x & 63;
    uint32_t s = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t t = __shfl_up(s, d, 64);
        if (lane >= d) s += t;
    }
    if (lane == 63) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    uint32_t base = 0;
#pragma unroll
    for (int w = 0; w < T / 64; w++) base += w < (int)(threadIdx.x >> 6) ? lds[w] : 0;
    __syncthreads();
    return base + s - v;
}

// Up to 8192 places: one launch, in which every place counts what comes before it (16
// lanes a place, all keys in each workgroup's LDS), while further workgroups clear the
// table. 4096 places take 9.1 us (10.5 by digits in one workgroup's LDS); the work
// goes with the square of their number, and at 16384 would take what the launches below do.
constexpr int SMALL = 8192;

template <typename T>
__global__ __launch_bounds__(256) void k_embed_rank(EmbedArgs a, int ranking, uint32_t* keys, uint32_t* places) {
    if ((int)blockIdx.x >= ranking) {
        clear_table<T>(a, blockIdx.x - ranking, gridDim.x - ranking);
        return;
    }
    __shared__ uint4 key4[SMALL / 4];
    uint32_t* key = (uint32_t*)key4;
    const int n = (int)a.n, padded = (n + 63) / 64 * 64;
    for (int i0 = threadIdx.x; i0 < padded; i0 += 256 * 8) {
        uint32_t k[8];
#pragma unroll
        for (int e = 0; e < 8; e++) k[e] = key_at(a, min(i0 + 256 * e, n - 1));
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (i0 + 256 * e < padded) key[i0 + 256 * e] = i0 + 256 * e < n ? k[e] : ~0u;  // after every key
    }
    __syncthreads();
    const int i = blockIdx.x * 16 + threadIdx.x / 16, lane = threadIdx.x % 16;
    const uint32_t own = key[min(i, n - 1)];
    uint32_t before = 0;
#pragma unroll 4
    for (int j = lane * 4; j < padded; j += 64) {
        const uint4 k = key4[j / 4];
        // equal keys come in the order of their places
        before += k.x < own + (j < i);
        before += k.y < own + (j + 1 < i);
        before += k.z < own + (j + 2 < i);
        before += k.w < own + (j + 3 < i);
    }
#pragma unroll
    for (int d = 1; d < 16; d *= 2) before += __shfl_xor((int)before, d, 16);
    if (lane == 0 && i < n) keys[before] = own, places[before] = i;
}

// More: digits of up to 10 bits, each in three launches over tiles of 1024
// places: the tiles' counts of the digit's values, their sums over the tiles before,
// and the move. Pass 0 reads the tokens. The launches are too short to fill the chip:
// further workgroups of theirs clear the table, a share in each launch.
constexpr int TILE = 1024, MOST_VALUES = 1024;

struct SortPass {
    const uint32_t *keys, *places;  // null: the tokens
    uint32_t *to_keys, *to_places;
    uint32_t* counts;  // [tiles][values], then the sums over the tiles before
    uint32_t* totals;  // [values]
    int shift, width;
    int64_t tiles;
    int64_t clear_first, clear_parts;  // shares of the table that this launch begins with, of all
};

template <typename T> __global__ __launch_bounds__(256) void k_embed_count(EmbedArgs a, SortPass p) {
    if (blockIdx.x >= p.tiles) {
        clear_table<T>(a, p.clear_first + blockIdx.x - p.tiles, p.clear_parts);
        return;
    }
    __shared__ uint32_t counts[MOST_VALUES];
    const int values = 1 << p.width;
    for (int v = threadIdx.x; v < values; v += 256) counts[v] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * TILE;
#pragma unroll
    for (int j = 0; j < TILE / 256; j++) {
        const int64_t i = first + j * 256 + threadIdx.x;
        if (i < a.n) atomicAdd(&counts[((p.keys ? p.keys[i] : key_at(a, i)) >> p.shift) & (values - 1)], 1u);
    }
    __syncthreads();
    for (int v = threadIdx.x; v < values; v += 256) p.counts[(int64_t)blockIdx.x * values + v] = counts[v];
}

// 16 values a workgroup, 64 threads for each value's tiles.
__global__ __launch_bounds__(1024) void k_embed_sum_tiles(SortPass p) {
    __shared__ uint32_t parts[64][17];
    const int values = 1 << p.width, v = blockIdx.x * 16 + threadIdx.x % 16, g = threadIdx.x / 16;
    const int64_t each = (p.tiles + 63) / 64, t0 = min(g * each, p.tiles), t1 = min(t0 + each, p.tiles);
    uint32_t sum = 0;
    if (v < values)
#pragma unroll 8
        for (int64_t t = t0; t < t1; t++) sum += p.counts[t * values + v];
    parts[g][threadIdx.x % 16] = sum;
    __syncthreads();
    if (v >= values) return;
    uint32_t before = 0;
    for (int h = 0; h < g; h++) before += parts[h][threadIdx.x % 16];
    if (g == 63) p.totals[v] = before + sum;
#pragma unroll 8
    for (int64_t t = t0; t < t1; t++) {
        const uint32_t c = p.counts[t * values + v];
        p.counts[t * values + v] = before;
        before += c;
    }
}

template <typename T> __global__ __launch_bounds__(256) void k_embed_move(EmbedArgs a, SortPass p) {
    if (blockIdx.x >= p.tiles) {
        clear_table<T>(a, p.clear_first + blockIdx.x - p.tiles, p.clear_parts);
        return;
    }
    constexpr int ITEMS = TILE / 256, EACH = MOST_VALUES / 256;
    __shared__ uint32_t counts[4][MOST_VALUES];
    __shared__ uint32_t base[MOST_VALUES];
    __shared__ uint32_t sums[4];
    const int values = 1 << p.width, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t first = (int64_t)blockIdx.x * TILE + wave * (TILE / 4);
    uint32_t key[ITEMS], place[ITEMS], rank[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; j++) {
        const int64_t i = first + j * 64 + lane;
        key[j] = i < a.n ? p.keys ? p.keys[i] : key_at(a, i) : 0;
        place[j] = i < a.n && p.places ? p.places[i] : (uint32_t)i;
    }
    for (int w = 0; w < 4; w++)
        for (int v = threadIdx.x; v < values; v += 256) counts[w][v] = 0;
    // thread t: values EACH t ... EACH t + EACH - 1
    uint32_t total[EACH], sum = 0;
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        const int v = threadIdx.x * EACH + e;
        total[e] = v < values ? p.totals[v] : 0;
        sum += total[e];
    }
    uint32_t before = sum_before<256>(sum, sums);
#pragma unroll
    for (int e = 0; e < EACH; e++) {
        const int v = threadIdx.x * EACH + e;
        if (v < values) base[v] = before + p.counts[(int64_t)blockIdx.x * values + v];
        before += total[e];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; j++)
        rank[j] = rank_of((key[j] >> p.shift) & (values - 1), p.width, first + j * 64 + lane < a.n, counts[wave]);
    __syncthreads();
    for (int v = threadIdx.x; v < values; v += 256) {
        uint32_t t = base[v];
#pragma unroll
        for (int w = 0; w < 4; w++) {
            const uint32_t c = counts[w][v];
            counts[w][v] = t;
            t += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; j++)
        if (first + j * 64 + lane < a.n) {
            const uint32_t to = counts[wave][(key[j] >> p.shift) & (values - 1)] + rank[j];
            p.to_keys[to] = key[j], p.to_places[to] = place[j];
        }
}

// ---------------------------------------------------------------------------
// The sums.

// Places of a chunk, whose rows one group of lanes sums: 64 where that is enough of
// them, down to 8 for the few tokens of a small call (4096 of 1000x64 float32: 14 us of
// sums in 64 chunks, 7 in 512). It goes by the number of tokens alone.
constexpr int CHUNK = 64, AHEAD = 8;
int chunk_of(int64_t n) { return (int)std::max<int64_t>(AHEAD, std::min<int64_t>(CHUNK, n / 2048 / AHEAD * AHEAD)); }

struct Sums {
    const uint32_t *keys, *places;
    void* parts;  // [chunks][2][D]: of the token that goes on from the chunk before, and on to the next
    int64_t chunks;
    int chunk;
};

// Whether the token at place i has the whole chunk of places from `first` on.
__device__ __forceinline__ bool fills(const Sums& q, int64_t n, uint32_t key, int64_t first) {
    return first + q.chunk <= n && q.keys[first] == key && q.keys[first + q.chunk - 1] == key;
}

// A group of G lanes takes the tokens that begin in a chunk, in a tile of G V columns. One
// that goes on past the chunk is finished here too, unless it fills the next chunk:
// then every chunk that it reaches leaves its part for k_embed_join. Eight
// rows are under way while eight are summed, and the lanes hold the keys and places of
// a chunk between them. Rows are loaded past the caches' usual order, as none is met
// again: 131072 of 1024 bfloat16 for 50000 tokens take 69 us (345 MB at 5.0 TB/s), 97
// by plain loads, however many are under way; 16384 rows take the same either way.
template <typename T, int V, int G> __global__ __launch_bounds__(256) void k_embed_sums(EmbedArgs a, Sums q) {
    using R = Acc<T>;
    constexpr int GROUPS = 256 / G, HELD = CHUNK / G;
    const int lane = threadIdx.x % G, D = (int)a.D;
    const R scale = (R)a.scale;
    const uint32_t none = (uint32_t)a.rows;
    const int tiles = (D + G * V - 1) / (G * V);
    const int group = G == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : threadIdx.x / G;
    for (int64_t w = (int64_t)blockIdx.x * GROUPS + group; w < q.chunks * tiles; w += (int64_t)gridDim.x * GROUPS) {
        // a chunk's tiles side by side: they read the same rows
        const int64_t chunk = w / tiles, lo = chunk * q.chunk, hi = min(lo + q.chunk, a.n);
        const int c = ((int)(w % tiles) * G + lane) * V, at = max(0, min(c, D - V));
        const T* g = (const T*)a.grad + at;
        uint32_t keys[HELD], places[HELD];
        auto hold = [&](int64_t first, int count) {
#pragma unroll
            for (int h = 0; h < HELD; h++) {
                const int64_t k = first + min(h * G + lane, count - 1);
                keys[h] = q.keys[k], places[h] = q.places[k];
            }
        };
        auto held = [&](const uint32_t (&v)[HELD], int i) {  // place i's, in all lanes of the group
            if constexpr (G == 64) {
                return (uint32_t)__builtin_amdgcn_readlane(v[0], i);
            } else {
                uint32_t r = v[0];
#pragma unroll
                for (int h = 1; h < HELD; h++) r = i / G == h ? v[h] : r;
                return (uint32_t)__shfl((int)r, i % G, G);
            }
        };
        R sum[V] = {};
        uint32_t current = none;
        // where the sum of the current token goes: 0 the table, 1 or 2 the chunk's first or second part, 3 nowhere
        int to = 3;
        auto finish = [&] {
            if (current == none || to == 3 || c >= D) return;
            if (to) {
                Vec<R, V> r;
#pragma unroll
                for (int e = 0; e < V; e++) r.v[e] = sum[e];
                store_vec<R, V>((R*)q.parts + (2 * chunk + to - 1) * a.D + at, r);
            } else {
                Vec<T, V> r;
#pragma unroll
                for (int e = 0; e < V; e++) r.v[e] = down<T>(sum[e] * scale);
                store_vec<T, V>((T*)a.grad_weight + (int64_t)current * a.D + at, r);
            }
        };
        // adds the rows of places [skip, count) that are held, up to the first key that `stops`
        auto add = [&](int skip, int count, auto stops) {
            Vec<T, V> next[AHEAD];
            auto fetch = [&](int i) {
#pragma unroll
                for (int j = 0; j < AHEAD; j++)
                    next[j] = load_once<T, V>(g + (int64_t)held(places, min(i + j, count - 1)) * a.grad_stride);
            };
            fetch(skip);
            for (int i = skip; i < count && !stops(held(keys, i)); i += AHEAD) {
                Vec<T, V> row[AHEAD];
#pragma unroll
                for (int j = 0; j < AHEAD; j++) row[j] = next[j];
                if (i + AHEAD < count) fetch(i + AHEAD);
#pragma unroll
                for (int j = 0; j < AHEAD; j++) {
                    const uint32_t key = held(keys, min(i + j, count - 1));
                    if (i + j >= count || stops(key)) break;
                    if (key != current) {
                        finish();
                        current = key, to = 0;
#pragma unroll
                        for (int e = 0; e < V; e++) sum[e] = 0;
                    }
#pragma unroll
                    for (int e = 0; e < V; e++) sum[e] += up(row[j].v[e]);
                }
            }
        };
        const int count = (int)(hi - lo);
        hold(lo, count);
        const uint32_t first = held(keys, 0), last = held(keys, count - 1);
        if (first == none) continue;
        int skip = 0;
        if (lo > 0 && q.keys[lo - 1] == first) {
            // one that began before: it leaves a part if it fills this chunk, or filled
            // the chunk before and began before that; else the chunk where it began adds it
            const bool part = fills(q, a.n, first, lo) || (lo > q.chunk && q.keys[lo - q.chunk - 1] == first);
            current = first, to = part ? 1 : 3;
            if (!part) {
#pragma unroll
                for (int h = 0; h < HELD; h++) {
                    const uint64_t same = __ballot(keys[h] == first && h * G + lane < count);
                    skip += __popcll(G == 64 ? same : (same >> (threadIdx.x % 64 / G * G)) & ((1ull << (G % 64)) - 1));
                }
            }
            if (skip == count) continue;
        }
        add(skip, count, [&](uint32_t key) { return key == none; });
        if (hi < a.n && last != none && current == last && to == 0 && q.keys[hi] == last) {
            if (fills(q, a.n, last, hi)) {
                to = 2;
            } else {
                const int more = (int)min((int64_t)q.chunk, a.n - hi);
                hold(hi, more);
                add(0, more, [&](uint32_t key) { return key != last; });
            }
        }
        finish();
    }
}

// The parts of a token that begins in a chunk and fills the next, in fp64: the
// workgroup's wavefronts take every fourth and meet in LDS.
template <typename T, int V> __global__ __launch_bounds__(256) void k_embed_join(EmbedArgs a, Sums q) {
    using R = Acc<T>;
    __shared__ double lds[4][64 * V];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = (int)a.D;
    for (int64_t chunk = blockIdx.x; chunk < q.chunks - 1; chunk += gridDim.x) {
        const int64_t lo = chunk * q.chunk, hi = lo + q.chunk;
        const uint32_t key = q.keys[hi - 1];
        if (key == (uint32_t)a.rows || !fills(q, a.n, key, hi) || (lo > 0 && q.keys[lo] == key && q.keys[lo - 1] == key)) continue;
        // the last chunk that begins with the token
        int64_t last = chunk + 1;
        for (;;) {
            const int64_t j = last + 1 + lane;
            const uint64_t other = ~__ballot(j < q.chunks && q.keys[min(j, q.chunks - 1) * q.chunk] == key);
            const int alike = other ? __ffsll((unsigned long long)other) - 1 : 64;
            last += alike;
            if (alike < 64) break;
        }
        const int c = (blockIdx.y * 64 + lane) * V, at = max(0, min(c, D - V));
        double sum[V] = {};
        const R* parts = (const R*)q.parts + at;
        for (int64_t j0 = chunk + wave; j0 <= last; j0 += 4 * AHEAD) {
            Vec<R, V> r[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; i++) {
                const int64_t j = min(j0 + 4 * i, last);
                r[i] = load_vec<R, V>(parts + (2 * j + (j == chunk ? 1 : 0)) * a.D);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; i++)
                if (j0 + 4 * i <= last)
#pragma unroll
                    for (int e = 0; e < V; e++) sum[e] += (double)r[i].v[e];
        }
#pragma unroll
        for (int e = 0; e < V; e++) lds[wave][lane * V + e] = sum[e];
        __syncthreads();
        if (wave == 0 && c < D) {
            Vec<T, V> out;
#pragma unroll
            for (int e = 0; e < V; e++) {
                double t = 0;
#pragma unroll
                for (int w = 0; w < 4; w++) t += lds[w][lane * V + e];
                out.v[e] = down<T>((R)(t * a.scale));
            }
            store_vec<T, V>((T*)a.grad_weight + (int64_t)key * a.D + at, out);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------

int bits_of(int64_t rows) { return 64 - __builtin_clzll((unsigned long long)rows); }  // of keys 0 ... rows

struct Layout {
    size_t keys[2], places[2], counts, totals, parts, bytes;
    int64_t tiles, chunks;
    int bits, passes, width, chunk;
};
Layout layout_of(int type, int64_t n, int64_t rows, int64_t D) {
    Layout l{};
    auto take = [&](size_t bytes) {
        const size_t at = l.bytes;
        l.bytes += (bytes + 255) & ~(size_t)255;
        return at;
    };
    l.bits = bits_of(rows);
    l.chunk = chunk_of(n), l.chunks = (n + l.chunk - 1) / l.chunk;
    const bool small = n <= SMALL;
    for (int k = 0; k < (small ? 1 : 2); k++) l.keys[k] = take((size_t)n * 4), l.places[k] = take((size_t)n * 4);
    if (!small) {
        l.tiles = (n + TILE - 1) / TILE;
        l.passes = (l.bits + 9) / 10;
        l.width = (l.bits + l.passes - 1) / l.passes;
        l.counts = take((size_t)l.tiles * 4 << l.width);
        l.totals = take((size_t)4 << l.width);
    }
    l.parts = take((size_t)l.chunks * 2 * (size_t)D * (type == E_F64 ? 8 : 4));
    return l;
}

// Workgroups of 256 threads: 2^22 of them stay below a launch's 2^32 threads.
unsigned grid_x(int64_t groups, int64_t y) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(groups, ((int64_t)1 << 22) / y)); }

template <typename T, int V, int G> void sums(const EmbedArgs& a, const Sums& q, hipStream_t s) {
    const int64_t tiles = (a.D + G * V - 1) / (G * V), wide = (a.D + 64 * V - 1) / (64 * V);
    k_embed_sums<T, V, G><<<grid_x((q.chunks * tiles * G + 255) / 256, 1), 256, 0, s>>>(a, q);
    if (q.chunks > 1) k_embed_join<T, V><<<dim3(grid_x(q.chunks - 1, wide), (unsigned)wide), 256, 0, s>>>(a, q);
}

template <typename T> hipError_t backward(int type, const EmbedArgs& a, void* ws, hipStream_t s) {
    const Layout l = layout_of(type, a.n, a.rows, a.D);
    char* base = (char*)ws;
    uint32_t *keys[2], *places[2];
    for (int k = 0; k < 2; k++) keys[k] = (uint32_t*)(base + l.keys[k]), places[k] = (uint32_t*)(base + l.places[k]);
    // a workgroup clears 16 KB or more
    const int64_t clearing = std::max<int64_t>(1, std::min<int64_t>(2048, a.rows * a.D * (int64_t)sizeof(T) >> 14));
    int at = 0;
    if (a.n <= SMALL) {
        const int ranking = (int)(a.n + 15) / 16;
        k_embed_rank<T><<<(unsigned)(ranking + clearing), 256, 0, s>>>(a, ranking, keys[0], places[0]);
        if (a.n == 0) return hipGetLastError();
    } else {
        for (int k = 0; k < l.passes; k++, at ^= 1) {
            SortPass p{};
            if (k > 0) p.keys = keys[at ^ 1], p.places = places[at ^ 1];
            p.to_keys = keys[at], p.to_places = places[at];
            p.counts = (uint32_t*)(base + l.counts), p.totals = (uint32_t*)(base + l.totals);
            p.shift = k * l.width, p.width = std::min(l.width, l.bits - p.shift), p.tiles = l.tiles;
            const int64_t share = (clearing + 2 * l.passes - 1) / (2 * l.passes);
            p.clear_parts = share * 2 * l.passes, p.clear_first = share * 2 * k;
            k_embed_count<T><<<(unsigned)(l.tiles + share), 256, 0, s>>>(a, p);
            k_embed_sum_tiles<<<((1 << p.width) + 15) / 16, 1024, 0, s>>>(p);
            p.clear_first += share;
            k_embed_move<T><<<(unsigned)(l.tiles + share), 256, 0, s>>>(a, p);
        }
        at ^= 1;
    }
    const Sums q{keys[at], places[at], base + l.parts, l.chunks, l.chunk};
    if (a.D < VEC<T>) sums<T, 1, 16>(a, q, s);
    else if (a.D <= 16 * VEC<T>) sums<T, VEC<T>, 16>(a, q, s);
    else sums<T, VEC<T>, 64>(a, q, s);
    return hipGetLastError();
}

template <typename T, int V, int G, int K> hipError_t rows_of(const EmbedArgs& a, hipStream_t s) {
    constexpr int GROUPS = 256 / G;
    const int64_t count = a.n * ((a.D + G * V * K - 1) / (G * V * K));
    k_embed_fwd<T, V, G, K><<<(unsigned)std::min<int64_t>((count + GROUPS - 1) / GROUPS, 4096), 256, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T> hipError_t forward(const EmbedArgs& a, hipStream_t s) {
    constexpr int V = VEC<T>;
    if (a.D < V) return rows_of<T, 1, 16, 1>(a, s);
    if (a.D <= 16 * V) return rows_of<T, V, 16, 1>(a, s);
    if (a.D <= 64 * V) return rows_of<T, V, 64, 1>(a, s);
    return rows_of<T, V, 64, 2>(a, s);
}

template <typename F> hipError_t by_type(int type, F f) {
    switch (type) {
        case E_F64: return f(double{});
        case E_BF16: return f(bf16{});
        case E_F16: return f(_Float16{});
        default: return f(float{});
    }
}

}  // namespace

size_t embed_workspace(int type, int64_t n, int64_t rows, int64_t D) { return layout_of(type, n, rows, D).bytes; }

hipError_t launch_embed_forward(int type, const EmbedArgs& a, hipStream_t s) {
    if (a.n == 0) return hipSuccess;
    return by_type(type, [&](auto t) { return forward<decltype(t)>(a, s); });
}

hipError_t launch_embed_backward(int type, const EmbedArgs& a, void* ws, hipStream_t s) {
    return by_type(type, [&](auto t) { return backward<decltype(t)>(type, a, ws, s); });
}

}  // namespace qlayer
