// Sums of embedding vectors over a row's ids, and their gradient by sorted ids, on gfx950.
//
//     out[r] = scale * sum_t table[id(r, t) + offset[t]]
//     grad_table[v] = scale * sum of grad[r] over all (r, t) whose vector is v
//
// Forward: a vector of `dim` values is read by a group of lanes, a piece of up to 16 bytes each; groups that share a row
// (a wavefront's, or a workgroup's where rows are few) take its ids in turn and add up their sums at the end.
//
// Backward: (vector, row) pairs, one for each id, are sorted by vector with a stable radix sort, up to 10 bits a pass: counts
// of each digit by tile, sums over the tiles, then each tile moves its pairs to their places.  The sorted list is cut into
// chunks of equal length whatever vectors they hold, so that a vector that every row has costs no more than others; a group
// of lanes adds up a chunk, run after run of equal vectors.  A run inside a chunk is a vector's gradient.  Of runs that cross
// chunks the parts go to the workspace, and a second kernel adds up the parts of each.  No atomics on values: the order
// of every sum is fixed by the ids alone.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "head_device.hpp"

namespace head_impl {
namespace {

constexpr int THREADS = 256;
constexpr int64_t MAX_GRID = 1 << 22;  // workgroups of a launch: 2^30 threads, a grid's axis has room for 2^32

struct Ids {
    const int32_t *id;
    const int64_t *offset;
    int64_t stride, n_vectors;
    int64_t n_ids;
};

// The vector that id t of a row stands for; -1: none.
__device__ __forceinline__ int64_t vector_of(const Ids &s, const int32_t *row, int64_t t)
{
    const int32_t id = row[t];
    const uint64_t v = static_cast<uint64_t>(id) + static_cast<uint64_t>(s.offset ? s.offset[t] : 0);  // below 0: far above all vectors
    return id >= 0 && v < static_cast<uint64_t>(s.n_vectors) ? static_cast<int64_t>(v) : -1;
}

// A piece of V values as the machine word it is read as.  A value that is to count for nothing is masked there, by all ones or
// none: as a choice between values it would be a branch for the compiler, and the loads of a loop would not be on their way together.
template <class T, int V>
using Word = typename WordOf<sizeof(T) * V>::Type;

__device__ __forceinline__ void add(float (&a)[1], uint16_t w) { a[0] += __uint_as_float(static_cast<uint32_t>(w) << 16); }
__device__ __forceinline__ void add(float (&a)[1], uint32_t w) { a[0] += __uint_as_float(w); }
__device__ __forceinline__ void add(float (&a)[2], uint32_t w)
{
    a[0] += __uint_as_float(w << 16);
    a[1] += __uint_as_float(w & 0xFFFF0000u);
}
template <int V, class W>
__device__ __forceinline__ void add(float (&a)[V], W w)
{
    constexpr int WORDS = sizeof(W) / 4;
#pragma unroll
    for (int k = 0; k < WORDS; ++k) {
        if constexpr (V == WORDS) {
            a[k] += __uint_as_float(w[k]);
        } else {
            a[2 * k] += __uint_as_float(w[k] << 16);
            a[2 * k + 1] += __uint_as_float(w[k] & 0xFFFF0000u);
        }
    }
}

// `lanes` lanes of a group read a vector; `team` groups share a row.  Bound by the way from id to offset and vector in memory: one row of
// 500 ids, 64 float32, 6.8 us; 4,096 rows of 128, 18.
template <class T, int V>
__global__ __launch_bounds__(1024) void embed_kernel(int64_t n_rows, int dim, Ids s, const T *table, int64_t table_stride, float scale,
                                                     T *out, int lanes, int team)
{
    extern __shared__ float sums[];  // [groups][lanes * V], where a row's groups are in several wavefronts
    const int group = threadIdx.x / lanes, lane = threadIdx.x % lanes, groups = blockDim.x / lanes;
    const int rows = groups / team, member = group % team;
    const int c = (blockIdx.y * lanes + lane) * V;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * rows; first < n_rows; first += static_cast<int64_t>(gridDim.x) * rows) {
        const int64_t row = first + group / team;
        float a[V] = {};
        if (row < n_rows && c < dim) {
            const int32_t *ids = s.id + row * s.stride;
            constexpr int AHEAD = 8;  // vectors on their way
            int64_t last = 0;  // read again, and dropped, where an id stands for nothing: a load without a branch around it
            for (int64_t t0 = member; t0 < s.n_ids; t0 += int64_t{AHEAD} * team) {
                int64_t v[AHEAD];
                Word<T, V> p[AHEAD];
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    const int64_t t = t0 + j * team;
                    v[j] = t < s.n_ids ? vector_of(s, ids, t) : -1;
                }
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    last = v[j] >= 0 ? v[j] : last;
                    p[j] = *reinterpret_cast<const Word<T, V> *>(table + last * table_stride + c);
                }
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) add(a, static_cast<Word<T, V>>(p[j] & static_cast<uint32_t>(~(v[j] >> 63))));
            }
        }
        if (team > 1) {
            const int in_wave = std::min(team, 64 / lanes);
            for (int d = lanes; d < lanes * in_wave; d *= 2)
#pragma unroll
                for (int k = 0; k < V; ++k) a[k] += __shfl_xor(a[k], d, 64);
            if (team > in_wave) {
                __syncthreads();  // who still reads the last row's
                if (threadIdx.x % 64 < lanes)
#pragma unroll
                    for (int k = 0; k < V; ++k) sums[(threadIdx.x / 64 * lanes + lane) * V + k] = a[k];
                __syncthreads();
                const int waves = team / in_wave, from = threadIdx.x / 64 / waves * waves;
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    a[k] = 0;
                    for (int w = 0; w < waves; ++w) a[k] += sums[((from + w) * lanes + lane) * V + k];
                }
            }
        }
        if (member == 0 && row < n_rows && c < dim) {
            Pack<T, V> p;
#pragma unroll
            for (int k = 0; k < V; ++k) p.v[k] = narrow<T>(scale * a[k]);
            *reinterpret_cast<Pack<T, V> *>(out + row * dim + c) = p;
        }
    }
}

// Many rows with many ids: a group of G lanes takes ROWS rows at once, and all groups go through the ids in the same order: what those that
// run at the same time read is the vectors of a few ids (trees) rather than of the whole table (33 MB of leaves).  The G lanes read G ids of a row at
// once, and each gets every one of them from its neighbours.
// Bound by what goes from the caches to registers: 103,069 rows of 128 ids, 128 bfloat16, 171 us, 17 TB/s.  Two rows of a group 201 us, eight 244, a
// wavefront for each row 365 to 390.  A launch of no more workgroups than are resident takes as long (a million such rows 2.0 ms either way).
// Rounds are of G ids, there or not, so that ids are at least half of one: 20 ids, 256 float32 (G = 64), 110,000 rows take 217 us here and 203 to 218 in
// the general kernel, 4,500 rows 21 and 15; 40 ids 254 and 371, and 23 and 24.
template <class T, int V, int G, int ROWS>
__global__ __launch_bounds__(THREADS) void sweep_kernel(int64_t n_rows, int dim, Ids s, const T *table, uint32_t stride_bytes, float scale,
                                                        T *out)
{
    const int lane = threadIdx.x % G, c = (blockIdx.y * G + lane) * V;
    const bool in = c < dim;
    const int64_t step = static_cast<int64_t>(gridDim.x) * (THREADS / G) * ROWS;
    for (int64_t row0 = (static_cast<int64_t>(blockIdx.x) * (THREADS / G) + threadIdx.x / G) * ROWS; row0 - threadIdx.x / G * ROWS < n_rows;
         row0 += step) {
        float a[ROWS][V] = {};
        int32_t last[ROWS] = {};  // read again, and dropped, where an id stands for nothing: a load without a branch around it
        const char *from = reinterpret_cast<const char *>(table + (in ? c : 0));
        for (int64_t t0 = 0; t0 < s.n_ids; t0 += G) {
            int32_t v[ROWS];  // of id t0 + lane; -1: none
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                v[r] = row0 + r < n_rows && t0 + lane < s.n_ids ? static_cast<int32_t>(vector_of(s, s.id + (row0 + r) * s.stride, t0 + lane)) : -1;
#pragma unroll 2
            for (int t = 0; t < G; ++t) {
                Word<T, V> p[ROWS];
                uint32_t mask[ROWS];
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const int32_t at = __shfl(v[r], t, G);
                    mask[r] = ~static_cast<uint32_t>(at >> 31);
                    last[r] = at >= 0 ? at : last[r];
                    p[r] = *reinterpret_cast<const Word<T, V> *>(from + static_cast<uint64_t>(static_cast<uint32_t>(last[r])) * stride_bytes);
                }
#pragma unroll
                for (int r = 0; r < ROWS; ++r) add(a[r], p[r] & mask[r]);
            }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            if (in && row0 + r < n_rows) {
                Pack<T, V> p;
#pragma unroll
                for (int k = 0; k < V; ++k) p.v[k] = narrow<T>(scale * a[r][k]);
                *reinterpret_cast<Pack<T, V> *>(out + (row0 + r) * dim + c) = p;
            }
    }
}

// ---- the sort

// A digit has at most MAX_DIGIT bits: as many passes as the largest key needs with that, and as few bits as do with those passes.
constexpr int MAX_DIGIT = 10;
constexpr int LANES = 512, WAVES = LANES / 64;
// Pairs of a lane.  16: a workgroup's tile has at 9 bits 16 of each digit, 128 bytes that are written together.  4 where there are
// few, whose tiles are not many either way, and are sorted faster (8,000 pairs: 6 us a pass, against 15).
constexpr int MANY = 16, FEW = 4;
constexpr uint32_t FEW_PAIRS = 1 << 20;

// of move_kernel: the tile's pairs, and for a digit its place away and a count for each wavefront; at 9 bits two workgroups of a CU
constexpr size_t move_lds(int items, int bits) { return LANES * items * 8 + ((4 + 2 * WAVES) << bits); }

struct Pair {
    uint32_t key, row;
};

// Where pairs come from: the ids of the batch on the first pass, the last pass's output on the others.
struct Pairs {
    Ids s;
    const Pair *pair;              // null on the first pass
    uint32_t n;
    uint32_t n_ids, magic, shift;  // division by n_ids of a number below 2^31
};

// What a pass reads: the last pass's output, or ids, without and with offsets.
enum { LAST_PASS, IDS, IDS_AND_OFFSETS };

// Pair i.  An id that stands for no vector sorts behind all that do.
template <int FROM>
__device__ __forceinline__ Pair pair_of(const Pairs &p, uint32_t i)
{
    if constexpr (FROM == LAST_PASS) return p.pair[i];
    const uint32_t row = p.n_ids == 1 ? i : __umulhi(i, p.magic) >> p.shift, t = i - row * p.n_ids;
    const int32_t id = p.s.id[row * p.s.stride + t];
    const uint64_t v = static_cast<uint64_t>(id) + static_cast<uint64_t>(FROM == IDS_AND_OFFSETS ? p.s.offset[t] : 0), all = p.s.n_vectors;
    return Pair{static_cast<uint32_t>(id >= 0 && v < all ? v : all), row};
}

template <int FROM, int ITEMS>
__global__ __launch_bounds__(LANES) void count_kernel(Pairs p, int bit, int bits, uint32_t n_tiles, uint32_t *counts)
{
    constexpr int TILE = LANES * ITEMS;
    __shared__ uint32_t count[1 << MAX_DIGIT];
    const int digits = 1 << bits;
    for (int d = threadIdx.x; d < digits; d += LANES) count[d] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * TILE + threadIdx.x;
    uint32_t key[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) key[k] = pair_of<FROM>(p, std::min(first + k * LANES, p.n - 1)).key;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
        if (first + k * LANES < p.n) atomicAdd(&count[key[k] >> bit & (digits - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += LANES) counts[static_cast<uint32_t>(d) * n_tiles + blockIdx.x] = count[d];
}

// Sum of v over the lanes before this one of the workgroup; `all`: over the whole workgroup.
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t &all, uint32_t *lds)
{
    uint32_t s = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(s, d, 64);
        if (static_cast<int>(threadIdx.x % 64) >= d) s += o;
    }
    __syncthreads();
    if (threadIdx.x % 64 == 63) lds[threadIdx.x / 64] = s;
    __syncthreads();
    uint32_t before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < static_cast<int>(threadIdx.x / 64)) before += lds[w];
        all += lds[w];
    }
    return before + s - v;
}

// A workgroup for each digit: its counts become sums over the tiles before, and the digit's total goes behind them.
__global__ __launch_bounds__(LANES) void tiles_kernel(uint32_t n_tiles, uint32_t *counts, uint32_t *totals)
{
    __shared__ uint32_t lds[WAVES];
    uint32_t *row = counts + static_cast<int64_t>(blockIdx.x) * n_tiles, sum = 0;
    for (uint32_t first = 0; first < n_tiles; first += LANES) {
        const uint32_t i = first + threadIdx.x;
        uint32_t all;
        const uint32_t before = sum_before(i < n_tiles ? row[i] : 0, all, lds);
        if (i < n_tiles) row[i] = sum + before;
        sum += all;
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = sum;
}

// A wavefront's LDS accesses before are made before its accesses after, its lanes' of each other's words too.
__device__ __forceinline__ void in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A tile is sorted by the digit in LDS and then goes out in that order, so that neighbours write neighbouring places.  10 million pairs and
// 9 bits: 60 us a pass, of which half is the traffic; straight to their places from registers, at 8 bits, 112.
template <int FROM, int ITEMS>
__global__ __launch_bounds__(LANES, 4) void move_kernel(Pairs p, int bit, int bits, uint32_t n_tiles, const uint32_t *counts,
                                                        const uint32_t *totals, Pair *out)
{
    constexpr int TILE = LANES * ITEMS;
    extern __shared__ __align__(16) char shared[];  // [TILE] pairs, [digits] differences, [WAVES][digits] counts
    __shared__ uint32_t lds[WAVES];
    const int digits = 1 << bits, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    Pair *sorted = reinterpret_cast<Pair *>(shared);
    uint32_t *away = reinterpret_cast<uint32_t *>(sorted + TILE);  // a digit's place in the output less its place in the tile
    uint16_t *place = reinterpret_cast<uint16_t *>(away + digits);  // where a wavefront's next pair of a digit goes in the tile
    for (int d = threadIdx.x; d < WAVES * digits; d += LANES) place[d] = 0;
    __syncthreads();
    // A wavefront has ITEMS * 64 adjacent pairs, 64 at a time.
    const uint32_t first = blockIdx.x * TILE + wave * (ITEMS * 64) + lane;
    uint16_t *own = place + wave * digits;
    Pair pair[ITEMS];
    uint16_t before[ITEMS];  // pairs of the same digit that the wavefront had before
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) pair[k] = pair_of<FROM>(p, std::min(first + k * 64, p.n - 1));
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const bool here = first + k * 64 < p.n;
        const uint32_t digit = pair[k].key >> bit & (digits - 1);
        const uint64_t all = __ballot(here);
        uint32_t low = static_cast<uint32_t>(all), high = static_cast<uint32_t>(all >> 32);  // lanes that have this lane's digit
#pragma unroll 2
        for (int j = 0; j < bits; ++j) {
            const int32_t own_bit = static_cast<int32_t>(digit << (31 - j)) >> 31;  // all ones or none
            const uint64_t set = __ballot(own_bit < 0);
            low &= ~(static_cast<uint32_t>(set) ^ own_bit);
            high &= ~(static_cast<uint32_t>(set >> 32) ^ own_bit);
        }
        const int ahead = __builtin_amdgcn_mbcnt_hi(high, __builtin_amdgcn_mbcnt_lo(low, 0));
        uint32_t had = 0;
        if (here) had = own[digit];
        in_order();  // all have read before the first lane of each digit writes
        if (here && ahead == 0) own[digit] = static_cast<uint16_t>(had + __popc(low) + __popc(high));
        in_order();
        before[k] = static_cast<uint16_t>(had + ahead);
    }
    __syncthreads();
    // Lanes are digits: places in the output from the digits' totals and the tiles before, places in the tile from its own counts.
    uint32_t in_all = 0, in_tile = 0;
    for (int d0 = 0; d0 < digits; d0 += LANES) {
        const int d = d0 + threadIdx.x;
        uint32_t sum = 0, all;
        if (d < digits)
            for (int w = 0; w < WAVES; ++w) sum += place[w * digits + d];
        const uint32_t to = in_all + sum_before(d < digits ? totals[d] : 0, all, lds);
        in_all += all;
        uint32_t at = in_tile + sum_before(sum, all, lds);
        in_tile += all;
        if (d < digits) {
            away[d] = to + counts[static_cast<uint32_t>(d) * n_tiles + blockIdx.x] - at;
            for (int w = 0; w < WAVES; ++w) {
                const uint32_t had = place[w * digits + d];
                place[w * digits + d] = static_cast<uint16_t>(at);
                at += had;
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
        if (first + k * 64 < p.n) sorted[own[pair[k].key >> bit & (digits - 1)] + before[k]] = pair[k];
    __syncthreads();
    const uint32_t some = std::min<uint32_t>(TILE, p.n - blockIdx.x * TILE);
    auto write = [&](uint32_t i) {
        const Pair o = sorted[i];
        out[away[o.key >> bit & (digits - 1)] + i] = o;
    };
    if (some == TILE) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) write(k * LANES + threadIdx.x);
    } else {
        for (uint32_t i = threadIdx.x; i < some; i += LANES) write(i);
    }
}

// ---- the sums

template <class T>
__global__ __launch_bounds__(THREADS) void zero_kernel(T *to, int64_t n)
{
    constexpr int V = 16 / sizeof(T);
    const int64_t lanes = static_cast<int64_t>(gridDim.x) * THREADS, lane = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x;
    const int64_t head = std::min<int64_t>(n, (16 - reinterpret_cast<uintptr_t>(to) % 16) % 16 / sizeof(T));
    const int64_t whole = (n - head) / V;
    for (int64_t i = lane; i < whole; i += lanes) reinterpret_cast<Pack<T, V> *>(to + head)[i] = Pack<T, V>{};
    if (lane < head) to[lane] = T(0);
    if (lane < n - head - whole * V) to[head + whole * V + lane] = T(0);
}

struct Sorted {
    const Pair *pair;
    uint32_t n, n_vectors;  // pairs whose key is n_vectors stand for nothing
    uint32_t chunk, n_chunks;
};

// A group of `lanes` lanes adds up a chunk.  Bound by the L2s: 10 million rows of 64 float32, 192 us, 13 TB/s; the batch's 5 MB are a
// fifth more than an L2 holds.  4 or 16 rows on their way instead of 8: 193 and 207.  parts: [2 * chunk's number][dim], the part of the run that it begins in the
// midst of, then the part of the run that it ends in the midst of.
template <class T, int V>
__global__ __launch_bounds__(THREADS) void sum_kernel(Sorted s, int dim, const T *grad, int64_t grad_stride, float scale, T *out,
                                                      float *parts, int lanes)
{
    const uint32_t group = (blockIdx.x * THREADS + threadIdx.x) / lanes;
    const int c = (blockIdx.y * lanes + threadIdx.x % lanes) * V;
    if (group >= s.n_chunks || c >= dim) return;
    const uint32_t first = group * s.chunk, end = std::min(s.n, first + s.chunk);
    uint32_t key = s.pair[first].key;
    if (key >= s.n_vectors) return;
    bool begun = first > 0 && s.pair[first - 1].key == key;  // before this chunk
    float a[V] = {};
    auto store = [&](bool ends) {
        if (begun || !ends) {
            float *to = parts + (2 * static_cast<int64_t>(group) + (begun ? 0 : 1)) * dim + c;
            Pack<float, V> p;
#pragma unroll
            for (int k = 0; k < V; ++k) p.v[k] = a[k];
#pragma unroll
            for (int k = 0; k < V; ++k) to[k] = p.v[k];
        } else {
            Pack<T, V> p;
#pragma unroll
            for (int k = 0; k < V; ++k) p.v[k] = narrow<T>(scale * a[k]);
            *reinterpret_cast<Pack<T, V> *>(out + static_cast<int64_t>(key) * dim + c) = p;
        }
    };
    constexpr int AHEAD = 8;
    for (uint32_t i = first; i < end; i += AHEAD) {
        uint32_t keys[AHEAD];
        Pack<T, V> p[AHEAD];
        Pair pair[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) pair[j] = s.pair[std::min(i + j, end - 1)];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            keys[j] = i + j < end ? pair[j].key : s.n_vectors;
            p[j] = *reinterpret_cast<const Pack<T, V> *>(grad + pair[j].row * grad_stride + c);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (keys[j] >= s.n_vectors) break;
            if (keys[j] != key) {
                store(true);
                key = keys[j];
                begun = false;
#pragma unroll
                for (int k = 0; k < V; ++k) a[k] = 0;
            }
#pragma unroll
            for (int k = 0; k < V; ++k) a[k] += widen(p[j].v[k]);
        }
    }
    store(end == s.n || s.pair[end].key != key);
}

// A group of lanes for each chunk: if a run begins in the chunk and goes on, all its parts.  The parts of a long run (a vector
// that very many rows have) are added by the wavefront's groups together, each in turn and several on their way at a time.
template <class T, int V>
__global__ __launch_bounds__(THREADS) void join_kernel(Sorted s, int dim, const float *parts, float scale, T *out, int lanes)
{
    constexpr uint32_t AHEAD = 8;
    const uint32_t group = (blockIdx.x * THREADS + threadIdx.x) / lanes;
    const int c = (blockIdx.y * lanes + threadIdx.x % lanes) * V, at = c < dim ? c : 0;
    uint32_t key = 0;
    bool joins = group + 1 < s.n_chunks;  // no run goes on from the last chunk
    if (joins) {
        const uint32_t first = group * s.chunk, end = first + s.chunk;
        key = s.pair[end - 1].key;
        joins = key < s.n_vectors && s.pair[end].key == key && !(s.pair[first].key == key && first > 0 && s.pair[first - 1].key == key);
    }
    float a[V] = {};
    // Parts first, first + step, ...: AHEAD of them, as many as are of the run; false if the run ends with them.
    auto add = [&](uint32_t first, uint32_t step, uint32_t of) {
        uint32_t keys[AHEAD];
        float p[AHEAD][V];
#pragma unroll
        for (uint32_t j = 0; j < AHEAD; ++j) {
            const uint32_t g = std::min(first + j * step, s.n_chunks - 1);
            keys[j] = s.pair[g * s.chunk].key;
#pragma unroll
            for (int k = 0; k < V; ++k) p[j][k] = parts[2 * static_cast<int64_t>(g) * dim + at + k];
        }
#pragma unroll
        for (uint32_t j = 0; j < AHEAD; ++j) {
            if (first + j * step >= s.n_chunks || keys[j] != of) return false;
#pragma unroll
            for (int k = 0; k < V; ++k) a[k] += p[j][k];
        }
        return true;
    };
    bool more = false;
    if (joins) {
#pragma unroll
        for (int k = 0; k < V; ++k) a[k] = parts[(2 * static_cast<int64_t>(group) + 1) * dim + at + k];
        more = add(group + 1, 1, key);
    }
    const int own = threadIdx.x % 64 / lanes, groups = 64 / lanes;
    for (int g = 0; g < groups; ++g) {
        if (!__shfl(static_cast<int>(more), g * lanes, 64)) continue;  // the same for the whole wavefront
        const uint32_t of = __shfl(key, g * lanes, 64);
        float before[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            before[k] = a[k];
            a[k] = 0;
        }
        uint32_t next = group - own + g + 1 + AHEAD + own;
        while (add(next, groups, of)) next += AHEAD * groups;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            for (int d = lanes; d < 64; d *= 2) a[k] += __shfl_xor(a[k], d, 64);
            a[k] = own == g ? before[k] + a[k] : before[k];
        }
    }
    if (joins && c < dim) {
        Pack<T, V> p;
#pragma unroll
        for (int k = 0; k < V; ++k) p.v[k] = narrow<T>(scale * a[k]);
        *reinterpret_cast<Pack<T, V> *>(out + static_cast<int64_t>(key) * dim + c) = p;
    }
}

// ---- what a call launches

template <class T, class F>
hipError_t by_piece(int wide, F f)
{
    switch (wide) {
        case 1: return f(std::integral_constant<int, 1>());
        case 2: return f(std::integral_constant<int, 2>());
        case 4: return f(std::integral_constant<int, 4>());
        default:
            if constexpr (sizeof(T) == 2) return f(std::integral_constant<int, 8>());
            return hipErrorInvalidValue;
    }
}

template <class F>
hipError_t by_lanes(int lanes, F f)
{
    switch (lanes) {
        case 4: return f(std::integral_constant<int, 4>());
        case 8: return f(std::integral_constant<int, 8>());
        case 16: return f(std::integral_constant<int, 16>());
        case 32: return f(std::integral_constant<int, 32>());
        case 64: return f(std::integral_constant<int, 64>());
        default: return hipErrorInvalidValue;
    }
}

int power_at_least(int64_t n, int most)
{
    int p = 1;
    while (p < n && p < most) p *= 2;
    return p;
}

template <class T>
hipError_t embed(const head_ids &ids, int64_t dim, const T *table, int64_t table_stride, float scale, T *out, hipStream_t stream)
{
    const uint64_t bits = address(table) | address(out) | static_cast<uint64_t>(table_stride * sizeof(T)) | static_cast<uint64_t>(dim * sizeof(T));
    // an id without a vector may read vector 0: where there are no vectors there are no ids
    const Ids s{ids.ids, ids.offset, ids.ids_stride, ids.n_vectors, ids.n_vectors ? ids.n_ids : 0};
    return by_piece<T>(piece(bits, sizeof(T)), [&](auto V) {
        const int lanes = power_at_least(ceil_div(dim, V()), 64), in_wave = 64 / lanes;
        constexpr int ROWS = 4;
        if constexpr (V() * sizeof(T) == 16)
            if (lanes >= 4 && ids.n_ids >= std::max(16, lanes / 2) && ids.n_rows >= int64_t{1024} * ROWS * in_wave && table_stride * sizeof(T) <= UINT32_MAX)
                return by_lanes(lanes, [&](auto G) {
                    const dim3 grid(static_cast<uint32_t>(std::min(ceil_div(ids.n_rows, ROWS * (THREADS / G())), MAX_GRID)),
                                    static_cast<uint32_t>(ceil_div(dim, G() * V())));
                    hipLaunchKernelGGL((sweep_kernel<T, V(), G(), ROWS>), grid, dim3(THREADS), 0, stream, ids.n_rows, static_cast<int>(dim), s,
                                       table, static_cast<uint32_t>(table_stride * sizeof(T)), scale, out);
                    return hipGetLastError();
                });
        // a group for each row, a wavefront's groups, or a workgroup's
        const bool few = ids.n_rows <= 1024 && ids.n_ids >= 4 * in_wave;
        const int threads = few ? 1024 : THREADS;
        const int team = few ? threads / lanes : ids.n_ids >= 4 * in_wave ? in_wave : 1;
        const int64_t rows = threads / lanes / team;
        const size_t bytes = team > in_wave ? static_cast<size_t>(threads / 64) * lanes * V() * sizeof(float) : 0;
        const dim3 grid(static_cast<uint32_t>(std::min(ceil_div(ids.n_rows, rows), MAX_GRID / (threads / THREADS))),
                        static_cast<uint32_t>(ceil_div(dim, static_cast<int64_t>(lanes) * V())));
        hipLaunchKernelGGL((embed_kernel<T, V()>), grid, dim3(threads), bytes, stream, ids.n_rows, static_cast<int>(dim), s, table,
                           table_stride, scale, out, lanes, team);
        return hipGetLastError();
    });
}

// The parts of the workspace of the backward pass, in bytes from its start.
struct GradPlan {
    uint32_t n, n_tiles, chunk, n_chunks;
    int items, passes, bits;
    int64_t pair[2], counts, totals, parts, bytes;
};

GradPlan plan_grad(const head_ids &ids, int64_t dim)
{
    GradPlan p{};
    p.n = static_cast<uint32_t>(ids.n_rows * ids.n_ids);
    p.items = p.n < FEW_PAIRS ? FEW : MANY;
    p.n_tiles = static_cast<uint32_t>(ceil_div(p.n, LANES * p.items));
    int bits = 1;
    while (ids.n_vectors >> bits) ++bits;
    p.passes = static_cast<int>(ceil_div(bits, MAX_DIGIT));
    p.bits = static_cast<int>(ceil_div(bits, p.passes));
    // long chunks have fewer runs that cross them (64 instead of 128: 20 us more for 10 million pairs), short ones fill the device
    p.chunk = 8;
    while (p.chunk < 128 && p.n / (2 * p.chunk) >= 16384) p.chunk *= 2;
    p.n_chunks = static_cast<uint32_t>(ceil_div(p.n, p.chunk));
    int64_t at = 0;
    auto part = [&](int64_t bytes) {
        const int64_t from = at;
        at += round_up(bytes, 256);
        return from;
    };
    for (int64_t &pair : p.pair) pair = part(int64_t{sizeof(Pair)} * p.n);
    p.counts = part((int64_t{4} << p.bits) * p.n_tiles);
    p.totals = part(int64_t{4} << p.bits);
    p.parts = part(int64_t{8} * p.n_chunks * dim);
    p.bytes = p.n ? at : 0;
    return p;
}

template <class T>
hipError_t embed_grad(const head_ids &ids, int64_t dim, const T *grad, int64_t grad_stride, float scale, T *out, char *workspace,
                      hipStream_t stream)
{
    const int64_t values = ids.n_vectors * dim;
    hipLaunchKernelGGL((zero_kernel<T>), dim3(static_cast<uint32_t>(std::min<int64_t>(ceil_div(values, THREADS * 16), 8192))), dim3(THREADS), 0,
                       stream, out, values);
    if (const hipError_t e = hipGetLastError()) return e;
    const GradPlan plan = plan_grad(ids, dim);
    if (plan.n == 0) return hipSuccess;
    auto words = [&](int64_t at) { return reinterpret_cast<uint32_t *>(workspace + at); };
    Pairs p{};
    p.s = Ids{ids.ids, ids.offset, ids.ids_stride, ids.n_vectors, ids.n_ids};
    p.n = plan.n;
    p.n_ids = static_cast<uint32_t>(ids.n_ids);
    if (p.n_ids > 1) {  // 2^(31 + k) / n_ids, rounded up, is exact for numbers below 2^31 where 2^k >= n_ids
        int k = 0;
        while ((uint64_t{1} << k) < p.n_ids) ++k;
        p.magic = static_cast<uint32_t>((uint64_t{1} << (31 + k)) / p.n_ids + 1);
        p.shift = static_cast<uint32_t>(k - 1);
    }
    auto pairs = [&](int which) { return reinterpret_cast<Pair *>(workspace + plan.pair[which]); };
    auto pass = [&](auto FROM, auto ITEMS, int k) {
        if (const hipError_t e = allow_lds<move_kernel<FROM(), ITEMS()>>(move_lds(ITEMS(), MAX_DIGIT))) return e;
        const int bit = k * plan.bits;
        hipLaunchKernelGGL((count_kernel<FROM(), ITEMS()>), dim3(plan.n_tiles), dim3(LANES), 0, stream, p, bit, plan.bits, plan.n_tiles,
                           words(plan.counts));
        hipLaunchKernelGGL(tiles_kernel, dim3(1u << plan.bits), dim3(LANES), 0, stream, plan.n_tiles, words(plan.counts), words(plan.totals));
        hipLaunchKernelGGL((move_kernel<FROM(), ITEMS()>), dim3(plan.n_tiles), dim3(LANES), move_lds(ITEMS(), plan.bits), stream, p, bit,
                           plan.bits, plan.n_tiles, words(plan.counts), words(plan.totals), pairs(k % 2));
        p.pair = pairs(k % 2);
        return hipGetLastError();
    };
    auto sort = [&](auto ITEMS) {
        hipError_t e = ids.offset ? pass(std::integral_constant<int, IDS_AND_OFFSETS>(), ITEMS, 0) : pass(std::integral_constant<int, IDS>(), ITEMS, 0);
        for (int k = 1; k < plan.passes && e == hipSuccess; ++k) e = pass(std::integral_constant<int, LAST_PASS>(), ITEMS, k);
        return e;
    };
    if (const hipError_t e = plan.items == FEW ? sort(std::integral_constant<int, FEW>()) : sort(std::integral_constant<int, MANY>())) return e;
    const Sorted s{pairs((plan.passes - 1) % 2), plan.n, static_cast<uint32_t>(ids.n_vectors), plan.chunk, plan.n_chunks};
    float *parts = reinterpret_cast<float *>(workspace + plan.parts);
    const uint64_t bits = address(grad) | address(out) | static_cast<uint64_t>(grad_stride * sizeof(T)) | static_cast<uint64_t>(dim * sizeof(T));
    return by_piece<T>(piece(bits, sizeof(T)), [&](auto V) {
        const int lanes = power_at_least(ceil_div(dim, V()), 64);
        const dim3 grid(static_cast<uint32_t>(ceil_div(static_cast<int64_t>(plan.n_chunks) * lanes, THREADS)),
                        static_cast<uint32_t>(ceil_div(dim, static_cast<int64_t>(lanes) * V())));
        hipLaunchKernelGGL((sum_kernel<T, V()>), grid, dim3(THREADS), 0, stream, s, static_cast<int>(dim), grad, grad_stride, scale, out,
                           parts, lanes);
        hipLaunchKernelGGL((join_kernel<T, V()>), grid, dim3(THREADS), 0, stream, s, static_cast<int>(dim), parts, scale, out, lanes);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_embed(const head_ids &ids, int32_t dtype, int64_t dim, const void *table, int64_t table_stride, float scale,
                        void *out, hipStream_t stream)
{
    if (dtype == HEAD_BF16)
        return embed(ids, dim, static_cast<const bf16 *>(table), table_stride, scale, static_cast<bf16 *>(out), stream);
    return embed(ids, dim, static_cast<const float *>(table), table_stride, scale, static_cast<float *>(out), stream);
}

int64_t embed_grad_bytes(const head_ids &ids, int32_t, int64_t dim) { return plan_grad(ids, dim).bytes; }

hipError_t launch_embed_grad(const head_ids &ids, int32_t dtype, int64_t dim, const void *grad, int64_t grad_stride, float scale,
                             void *grad_table, void *workspace, hipStream_t stream)
{
    if (dtype == HEAD_BF16)
        return embed_grad(ids, dim, static_cast<const bf16 *>(grad), grad_stride, scale, static_cast<bf16 *>(grad_table),
                          static_cast<char *>(workspace), stream);
    return embed_grad(ids, dim, static_cast<const float *>(grad), grad_stride, scale, static_cast<float *>(grad_table),
                      static_cast<char *>(workspace), stream);
}

}  // namespace head_impl
