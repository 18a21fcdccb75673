// Softmax cross entropy of a linear model over many classes, on gfx950, without keeping the logits.
//
//     logit = hidden weight^T + bias;  lse = log sum exp(logit);  loss = lse - logit[target]
//     p = grad_loss * (exp(logit - lse) - [class is target])
//     grad_hidden = p weight;  grad_weight = p^T hidden;  grad_bias = sum over rows of p
//
// Four matrix products, forward one (the logits go no further than the registers of the workgroup that makes them: a
// tile's largest value and sum of exponentials for each row is all it writes), backward three: the logits again, as p of a
// piece of the classes in the workspace, then p times weight and p^T times hidden.  All four run on one body: a workgroup's
// tile of C = A B, A and B in tiles of 128 bytes of the sum's axis, brought to LDS by the loads that bypass registers while
// the matrix core works on the tiles before.  An operand lies in memory with the sum's axis along its rows (hidden and weight
// in the logits, p in the first gradient) or across them (weight, p and hidden in the gradients).
//
// bfloat16 products run on the 32x32x16 matrix instruction, float32 ones on the 32x32x2 float32 one, whose rate, a
// sixteenth, then bounds them; both accumulate in float32.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "head_device.hpp"

namespace head_impl {
namespace {

constexpr int STEP = 128;                       // bytes of the sum's axis in a tile
constexpr int64_t PIECE_BYTES = int64_t{1} << 30;  // of p in the workspace, where rows are not too many for that

using Acc = float __attribute__((ext_vector_type(16)));
using Bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using Chunk = float __attribute__((ext_vector_type(4)));  // 16 bytes of either type

__device__ const Chunk g_zeros[1] = {};

using GlobalChunk = const __attribute__((address_space(1))) void *;
using LdsChunk = __attribute__((address_space(3))) void *;
using Half = short __attribute__((ext_vector_type(4)));  // of a chunk
using LdsHalf = __attribute__((address_space(3))) Half *;

// An operand: `rows` along the result's axis, `depth` along the sum's.  has: a bit for each row of the batch, or null, where those are one
// of the axes; a row without its bit counts for nothing, whatever it holds.
template <class T>
struct Operand {
    const T *at;
    int64_t stride;
    int64_t rows, depth;
    const uint64_t *has = nullptr;
};

// A word of the bits.  Those are written by a kernel before, which the compiler cannot know: a scalar load has to be asked for.
template <class W>
__device__ __forceinline__ W bits_of(const uint64_t *has, int64_t word)
{
    return reinterpret_cast<const __attribute__((address_space(4))) W *>(reinterpret_cast<uintptr_t>(has))[word];
}

// Tiles of ROWS x 128 bytes of an operand, brought to LDS by THREADS lanes, 16 bytes each at a time.
// ALONG: the sum's axis lies along memory.  Row r of the tile is STEP bytes, its chunk c of 16 bytes in slot c ^ key(r): the
// 16 lanes that are served at once read the same chunk of 16 rows, which so lie in 16 different groups of four banks.  Rows are
// those of memory in another order where a lane of a matrix instruction is to have NT adjacent ones: row nt * 32 + l of every
// NT * 32 is the one NT * l + nt in memory.
// Otherwise a row of the tile holds the ROWS values of one index of the sum, its chunk c in slot c ^ key(index): bfloat16 values
// are read by the instruction that transposes 4 x 16 of them, 16 lanes 32 bytes of each of 4 rows, and 32 lanes are served at
// once; float32 ones one by one, 32 adjacent ones of each of two rows.
template <class T, bool ALONG, int ROWS, int THREADS, int NT>
struct Tile {
    static constexpr int VALUES = 16 / sizeof(T), DEPTH = STEP / sizeof(T), BYTES = ROWS * STEP;
    static constexpr int LOADS = BYTES / (THREADS * 16), WAVES = THREADS / 64;
    static constexpr int CHUNKS = ROWS / VALUES;  // of a row of the tile that lies across
    static constexpr int SLOTS = STEP / 16;       // of a row of one that lies along

    static __device__ __forceinline__ int key(int r)
    {
        if constexpr (ALONG) return r / (256 / STEP) % SLOTS;
        if constexpr (sizeof(T) == 4) return r / 4 % 2 * 8;
        return ROWS >= 128 ? r % 4 * 4 : r / 2 % 2 * 4;  // rows of 256 bytes or more lie in the same banks, of 128 every other
    }

    const T *from[LOADS];  // this lane's chunks at depth 0; rows past the end are the last one again, of whose results nobody reads
    int at[LOADS];         // their indexes of the sum, in the tile

    __device__ __forceinline__ void aim(const Operand<T> &o, int64_t row0)
    {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int part = j * WAVES + wave;  // 1024 bytes of the tile
            if constexpr (ALONG) {
                const int r = part * (64 / SLOTS) + lane / SLOTS, in = r % (NT * 32);
                const int64_t row = row0 + r - in + in % 32 * NT + in / 32;
                at[j] = ((lane % SLOTS) ^ key(r)) * VALUES;
                from[j] = o.at + std::min(row, o.rows - 1) * o.stride + at[j];
            } else {
                at[j] = (part * 64 + lane) / CHUNKS;
                const int64_t row = row0 + ((part * 64 + lane) % CHUNKS ^ key(at[j])) * VALUES;
                from[j] = o.at + at[j] * o.stride + std::min(row, (o.rows - 1) / VALUES * VALUES);
            }
        }
    }

    __device__ __forceinline__ void load(const Operand<T> &o, int64_t depth, char *lds) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const int64_t ahead = ALONG ? depth : depth * o.stride;
        auto chunk = [&](int j, const void *p) {
            __builtin_amdgcn_global_load_lds((GlobalChunk)(p), (LdsChunk)(lds + (j * WAVES + wave) * 1024), 16, 0, 0);
        };
        // Zeros past the end of the sum, and in place of rows of the batch that count for nothing: their values, finite or not, would be
        // multiplied by the zeros of p.
        if constexpr (ALONG) {
            const int left = static_cast<int>(std::min<int64_t>(DEPTH, o.depth - depth));
            if (left == DEPTH) {
#pragma unroll
                for (int j = 0; j < LOADS; ++j) chunk(j, from[j] + ahead);
            } else {
#pragma unroll
                for (int j = 0; j < LOADS; ++j) chunk(j, at[j] < left ? static_cast<const void *>(from[j] + ahead) : g_zeros);
            }
        } else {
            using Bits = std::conditional_t<DEPTH == 64, uint64_t, uint32_t>;  // of a step's indexes, aligned in the words of `has`
            static_assert(DEPTH == 8 * sizeof(Bits), "a step is a word of the bits");
            constexpr Bits ALL = ~Bits{0};
            Bits some = depth + DEPTH <= o.depth ? ALL : ALL >> (depth + DEPTH - o.depth);
            if (o.has) some &= bits_of<Bits>(o.has, depth / DEPTH);
            if (some == ALL) {
#pragma unroll
                for (int j = 0; j < LOADS; ++j) chunk(j, from[j] + ahead);
            } else {
#pragma unroll
                for (int j = 0; j < LOADS; ++j) chunk(j, some >> at[j] & 1 ? static_cast<const void *>(from[j] + ahead) : g_zeros);
            }
        }
    }

    // What a lane holds of 32 rows in a matrix instruction: of row r (the first of them + lane % 32) the values of chunk
    // 2 * kk + lane / 32.
    static __device__ __forceinline__ Chunk read(const char *lds, int r, int kk)
    {
        const int chunk = 2 * kk + threadIdx.x % 64 / 32;
        if constexpr (ALONG) {
            return *reinterpret_cast<const Chunk *>(lds + r * STEP + ((chunk ^ key(r)) * 16));
        } else if constexpr (sizeof(T) == 2) {
            // lane i of 16 reads 4 values of row i / 4 and gets those of column i, of 4 rows
            const int i = threadIdx.x % 16, depth = chunk * VALUES + i / 4;
            const int in = r / 32 * 32 + threadIdx.x % 32 / 16 * 16 + i % 4 * 4;
            const char *at = lds + depth * (ROWS * 2) + (in / VALUES ^ key(depth)) * 16 + in % VALUES * 2;
            Half h[2];
            h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsHalf)(at));
            h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsHalf)(at + 4 * ROWS * 2));
            return *reinterpret_cast<Chunk *>(h);
        } else {
            Chunk p;
#pragma unroll
            for (int j = 0; j < VALUES; ++j) {
                const int depth = chunk * VALUES + j;
                p[j] = reinterpret_cast<const float *>(lds)[depth * ROWS + (r / VALUES ^ key(depth)) * VALUES + r % VALUES];
            }
            return p;
        }
    }
};

__device__ __forceinline__ void multiply(Chunk a, Chunk b, Acc &c, bf16)
{
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<Bf16x8 *>(&a), *reinterpret_cast<Bf16x8 *>(&b), c, 0, 0, 0);
}
__device__ __forceinline__ void multiply(Chunk a, Chunk b, Acc &c, float)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
}

// How a workgroup's tile is dealt to its wavefronts.  NEXT: a lane's columns of the result are adjacent.
template <int M_, int N_, int WAVES_M_, int WAVES_N_, bool NEXT_>
struct Shape {
    static constexpr int M = M_, N = N_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, THREADS = 64 * WAVES_M * WAVES_N;
    static constexpr int MT = M / WAVES_M / 32, NT = N / WAVES_N / 32;  // 32 x 32 results of a wavefront
    static constexpr bool NEXT = NEXT_;

    static __device__ __forceinline__ int wave_m() { return threadIdx.x / 64 / WAVES_N; }
    static __device__ __forceinline__ int wave_n() { return threadIdx.x / 64 % WAVES_N; }
    // A lane's result i of 16 is row(mt, i), column(nt).
    static __device__ __forceinline__ int row(int mt, int i)
    {
        return wave_m() * (MT * 32) + mt * 32 + i / 4 * 8 + threadIdx.x % 64 / 32 * 4 + i % 4;
    }
    static __device__ __forceinline__ int column(int nt)
    {
        const int lane = threadIdx.x % 32;
        return wave_n() * (NT * 32) + (NEXT ? lane * NT + nt : nt * 32 + lane);
    }
};

// The products of a workgroup's tiles, one after the other: tile of C = A[row0.., depth0..depth1) B[.., column0..).  While the
// matrix core works on one step's tiles of A and B the next step's are on their way to the other half of LDS, the next
// tile's first ones while it works on a tile's last ones and while that tile is finished.
template <class T, class S, bool A_ALONG, bool B_ALONG>
struct Products {
    using A = Tile<T, A_ALONG, S::M, S::THREADS, 1>;
    using B = Tile<T, B_ALONG, S::N, S::THREADS, S::NEXT ? S::NT : 1>;
    static_assert(B_ALONG || !S::NEXT, "rows of a tile that lies across stay in order");
    static constexpr int BYTES = A::BYTES + B::BYTES;  // of a step; LDS holds two

    const Operand<T> &a, &b;
    char *lds;
    A ta;
    B tb;
    int64_t depth0;
    int steps = 0, step = 0, half = 0;

    __device__ __forceinline__ Products(const Operand<T> &a_, const Operand<T> &b_, char *lds_) : a(a_), b(b_), lds(lds_) {}

    __device__ __forceinline__ void load() const
    {
        const int64_t depth = depth0 + step * int64_t{A::DEPTH};
        ta.load(a, depth, lds + half * BYTES);
        tb.load(b, depth, lds + half * BYTES + A::BYTES);
    }

    // Begins a tile.  Tiles begin at different steps (turn), so that workgroups side by side, whose rows may lie a power of
    // two apart, do not ask for the same few of the memory's channels at the same time.
    // `plane`: A's values begin so many further on.
    __device__ __forceinline__ void aim(int64_t row0, int64_t column0, int64_t from, int64_t to, uint32_t turn, int64_t plane = 0)
    {
        ta.aim(Operand<T>{a.at + plane, a.stride, a.rows, a.depth, nullptr}, row0);
        tb.aim(b, column0);
        depth0 = from;
        steps = from < to ? static_cast<int>((to - from + A::DEPTH - 1) / A::DEPTH) : 0;
        step = steps ? static_cast<int>(turn % static_cast<uint32_t>(steps)) : 0;
        if (steps) load();
    }

    static __device__ __forceinline__ void clear(Acc (&c)[S::MT][S::NT])
    {
#pragma unroll
        for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < S::NT; ++nt) c[mt][nt] = Acc{};
    }

    // Adds the product that aim() began; next() is called once, to begin the one after it.
    template <class Next>
    __device__ __forceinline__ void run(Acc (&c)[S::MT][S::NT], Next next)
    {
        if (steps == 0) return next();
        const int count = steps;
        for (int done = 1; done <= count; ++done) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();  // this step's tiles are there, and nobody reads the other half any more
            const char *la = lds + half * BYTES, *lb = la + A::BYTES;
            half ^= 1;
            if (done < count) {
                step = step + 1 < count ? step + 1 : 0;
                load();
            } else next();
            // the next 32 bytes of the sum's axis are read while the matrix core has the last ones; more would fill the registers
            Chunk x[2][S::MT], y[2][S::NT];
            auto read = [&](int kk) {
#pragma unroll
                for (int mt = 0; mt < S::MT; ++mt) x[kk % 2][mt] = A::read(la, S::wave_m() * (S::MT * 32) + mt * 32 + threadIdx.x % 32, kk);
#pragma unroll
                for (int nt = 0; nt < S::NT; ++nt) y[kk % 2][nt] = B::read(lb, S::wave_n() * (S::NT * 32) + nt * 32 + threadIdx.x % 32, kk);
            };
            read(0);
#pragma unroll
            for (int kk = 0; kk < STEP / 32; ++kk) {
                if (kk + 1 < STEP / 32) read(kk + 1);
#pragma unroll
                for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
                    for (int nt = 0; nt < S::NT; ++nt) multiply(x[kk % 2][mt], y[kk % 2][nt], c[mt][nt], T());
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
};

// exp(x - from), finite or not: the difference first, which no finite x and from >= x take out of range.  The product with
// log2(e) is rounded, by x - from times 2^-24 of the result.  Where results are float32 it is taken in two parts, to a rounding or
// two of the result; the exponentials are then still nothing next to the float32 matrix instructions.
template <class T>
__device__ __forceinline__ float exp_from(float x, float from)
{
    constexpr float LOG2E = 1.44269502162933349609375f, REST = 1.925963033500011079e-08f;
    const float d = x - from, t = d * LOG2E, e = __builtin_amdgcn_exp2f(t);
    if constexpr (sizeof(T) == 2) return e;
    const float rest = fmaf(d, LOG2E, -t) + d * REST;
    return fabsf(rest) < 1 ? fmaf(e, rest * 0.693147180559945f, e) : e;  // d infinite: no rest
}

// Workgroup `id` of `rows` x `columns` tiles: workgroups go to the 8 XCDs in turn, so each XCD gets a range of the tiles, in
// which GROUP rows of tiles go together, column after column: what an XCD works on at a time is a block of tiles of some 8 x 8,
// whose operands its L2 holds.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t rows, uint32_t columns, uint32_t &row, uint32_t &column)
{
    constexpr uint32_t XCDS = 8, GROUP = 8;
    const uint32_t tiles = rows * columns, each = tiles / XCDS, more = tiles % XCDS, xcd = id % XCDS;
    const uint32_t i = xcd * each + std::min(xcd, more) + id / XCDS;
    const uint32_t first = i / (GROUP * columns) * GROUP, in = std::min(GROUP, rows - first), k = i - first * columns;
    row = first + k % in;
    column = k / in;
}

template <class T>
struct Model {
    Operand<T> hidden, weight;  // [n_rows][dim], [n_classes][dim], whole in 16 bytes
    const float *bias;
    const int32_t *target;
};

// ---- forward

// Rows of C are classes and its columns rows of the batch, so that a lane has the values of one row in its registers.  16,384 x 65,536 logits
// over 512 bfloat16: 1.23 to 1.32 ms, 833 to 894 TFLOP/s; bound by LDS and matrix core in turn, and by the exponentials at a tile's end, 15 vector
// instructions for each logit in all.  4,099 x 20,011 over 128 float32: 260 us, 81 TFLOP/s.
template <class T, class S>
__global__ __launch_bounds__(S::THREADS, 2) void lse_kernel(Model<T> m, uint32_t row_tiles, uint32_t class_tiles, float2 *parts, float *target_logit)
{
    extern __shared__ char lds[];
    float *numbers = reinterpret_cast<float *>(lds + 2 * Products<T, S, true, true>::BYTES);
    float2 *most = reinterpret_cast<float2 *>(numbers);  // [WAVES_M][N]
    float *bias = numbers + 2 * S::WAVES_M * S::N;       // [2][M], for tiles in turn
    Products<T, S, true, true> products(m.weight, m.hidden, lds);
    const uint32_t tiles = row_tiles * class_tiles;
    uint32_t class_tile = 0, row_tile = 0;
    auto aim = [&](uint32_t tile) {
        if (tile >= tiles) return;
        tile_of(tile, row_tiles, class_tiles, row_tile, class_tile);
        products.aim(int64_t{S::M} * class_tile, int64_t{S::N} * row_tile, 0, m.hidden.depth, row_tile + class_tile);
    };
    aim(blockIdx.x);
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint32_t this_class_tile = class_tile;
        const int64_t class0 = int64_t{S::M} * class_tile, row0 = int64_t{S::N} * row_tile;
        // What the end needs is read before the product, whose barriers come between.
        int targets[S::NT];  // among this lane's classes of each column, in the order of its results; -1: not there
#pragma unroll
        for (int nt = 0; nt < S::NT; ++nt) {
            const int64_t row = row0 + S::column(nt), target = row < m.hidden.rows ? m.target[row] : -1;
            const int64_t in = target < m.weight.rows ? target - class0 - S::row(0, 0) : -1;
            targets[nt] = in >= 0 && in < S::MT * 32 && in % 8 < 4 ? static_cast<int>(in / 8 * 4 + in % 4) : -1;
        }
        for (int i = threadIdx.x; i < S::M; i += S::THREADS)
            bias[i] = class0 + i < m.weight.rows ? (m.bias ? m.bias[class0 + i] : 0.0f) : -INFINITY;
        Acc c[S::MT][S::NT];
        products.clear(c);
        products.run(c, [&] { aim(tile + gridDim.x); });
        const float *own_bias = bias + S::row(0, 0);
#pragma unroll
        for (int nt = 0; nt < S::NT; ++nt) {
            float top = -INFINITY;
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const Chunk b = *reinterpret_cast<const Chunk *>(own_bias + mt * 32 + i * 2);
#pragma unroll
                    for (int k = 0; k < 4; ++k) top = fmaxf(top, c[mt][nt][i + k] += b[k]);
                }
            int target = targets[nt];
            if (__any(target >= 0)) {  // few wavefronts have a target among their classes
                asm volatile("" : "+v"(target));  // nor are the comparisons made ahead of the branch
                float v = 0;
#pragma unroll
                for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) v = target == mt * 16 + i ? c[mt][nt][i] : v;
                if (target >= 0) target_logit[row0 + S::column(nt)] = v;
            }
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float from = top > -INFINITY ? top : 0.0f;
            float sum = 0;
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
                for (int i = 0; i < 16; ++i) sum += exp_from<T>(c[mt][nt][i], from);
            sum += __shfl_xor(sum, 32, 64);
            if (threadIdx.x % 64 < 32) most[S::wave_m() * S::N + S::column(nt)] = make_float2(top, sum);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < S::N; i += S::THREADS)
            if (row0 + i < m.hidden.rows) {
                float2 all = most[i];
                for (int w = 1; w < S::WAVES_M; ++w) {
                    const float2 o = most[w * S::N + i];
                    const float top = fmaxf(all.x, o.x), from = top > -INFINITY ? top : 0.0f;
                    all = make_float2(top, all.y * exp_from<float>(all.x, from) + o.y * exp_from<float>(o.x, from));
                }
                parts[this_class_tile * m.hidden.rows + row0 + i] = all;
            }
        bias = numbers + 2 * S::WAVES_M * S::N + (bias == numbers + 2 * S::WAVES_M * S::N) * S::M;
    }
}

// The tiles' largest values and sums of a row become its lse.  ROWS rows of a workgroup, 256 / ROWS lanes on each.
template <int ROWS>
__global__ __launch_bounds__(256) void lse_join_kernel(int64_t n_rows, int64_t n_classes, int64_t class_tiles, const float2 *parts,
                                                       const float *target_logit, const int32_t *target, float *loss, float *lse)
{
    constexpr int LANES = 256 / ROWS;
    __shared__ float2 lds[LANES][ROWS];
    const int lane = threadIdx.x / ROWS, r = threadIdx.x % ROWS;
    for (int64_t row0 = int64_t{ROWS} * blockIdx.x; row0 < n_rows; row0 += int64_t{ROWS} * gridDim.x) {
        const int64_t row = row0 + r;
        float2 all = make_float2(-INFINITY, 0);
        auto add = [&](float2 o) {
            const float top = fmaxf(all.x, o.x), from = top > -INFINITY ? top : 0.0f;
            all = make_float2(top, all.y * exp_from<float>(all.x, from) + o.y * exp_from<float>(o.x, from));
        };
        if (row < n_rows) {
#pragma unroll 4
            for (int64_t t = lane; t < class_tiles; t += LANES) add(parts[t * n_rows + row]);
        }
        __syncthreads();
        lds[lane][r] = all;
        __syncthreads();
        if (lane == 0 && row < n_rows) {
            const int some = static_cast<int>(std::min<int64_t>(LANES, class_tiles));
            for (int i = 1; i < some; ++i) add(lds[i][r]);
            const float log = logf(all.y);
            lse[row] = all.x + log;
            loss[row] = target[row] >= 0 && target[row] < n_classes ? log + (all.x - target_logit[row]) : 0.0f;
        }
    }
}

// ---- backward

// p of the classes from `class0` on, [n_rows][stride]: whole tiles, zero where there is no class.  bias_parts: the sums of
// a tile's rows, [tiles of rows][stride].
// Where p is bfloat16, a row's largest value by far is that of its target, and its rounding, up to 2^-8 of it, would be the rounding of the
// whole gradient.  So p is kept in two planes (TWO), the second one, `plane` values behind the first, being what the first one's
// rounding left; the products with both cost little where there are few logits.  In tiles of 256, so where there are many, p is one plane, and grad_loss is divided
// by its largest magnitude (`scale`) first, and the results are multiplied by it: values are near -1 then, which roundings of
// many rows, of either sign, are right for on average, and not all of one factor times that (in a mean loss 1 / n_rows, say).
// A row without a target has logits of -inf here, so that p is 0 whatever it holds, and no bit in `has_target`, by which the products leave it out.
// 16,384 x 32,768 bfloat16: 732 us, of which the stores alone take about half.
template <class T, class S, bool TWO>
__global__ __launch_bounds__(S::THREADS, 2) void p_kernel(Model<T> m, const float *lse, const float *grad_loss, int64_t first_class,
                                                       uint32_t row_tiles, uint32_t class_tiles, T *p, int64_t stride, int64_t plane,
                                                       const float *scale, float *bias_parts, uint64_t *has_target)
{
    constexpr int ELSEWHERE = -1, NONE = -2;  // where a row's target is no class of the tile, or no class
    extern __shared__ char lds[];
    float *numbers = reinterpret_cast<float *>(lds + 2 * Products<T, S, true, true>::BYTES);
    float *sums = numbers;  // [WAVES_M][N]
    int turn = 0;           // for tiles in turn: [2][3][M]
    Products<T, S, true, true> products(m.hidden, m.weight, lds);
    const uint32_t tiles = row_tiles * class_tiles;
    uint32_t class_tile = 0, row_tile = 0;
    auto aim = [&](uint32_t tile) {
        if (tile >= tiles) return;
        tile_of(tile, row_tiles, class_tiles, row_tile, class_tile);
        products.aim(int64_t{S::M} * row_tile, first_class + int64_t{S::N} * class_tile, 0, m.hidden.depth, row_tile + class_tile);
    };
    aim(blockIdx.x);
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x, turn ^= 1) {
        const uint32_t this_row_tile = row_tile;
        const int64_t class0 = first_class + int64_t{S::N} * class_tile, row0 = int64_t{S::M} * row_tile;
        // What the end needs is read before the product, whose barriers come between.
        float *row_lse = numbers + S::WAVES_M * S::N + turn * 3 * S::M, *row_grad = row_lse + S::M;
        int *row_target = reinterpret_cast<int *>(row_grad + S::M);
        for (int i = threadIdx.x; i < S::M; i += S::THREADS) {
            const int64_t row = row0 + i;
            const int target = row < m.hidden.rows ? m.target[row] : -1;
            const bool has = target >= 0 && target < m.weight.rows;
            row_lse[i] = has ? lse[row] : 0.0f;
            row_grad[i] = has ? (scale ? grad_loss[row] / *scale : grad_loss[row]) : 0.0f;
            row_target[i] = !has ? NONE : target >= class0 && target < class0 + S::N ? static_cast<int>(target - class0) : ELSEWHERE;
            const uint64_t word = __ballot(has);
            if (class0 == 0 && i % 64 == 0) has_target[row / 64] = word;
        }
        float bias[S::NT], sum[S::NT] = {};
#pragma unroll
        for (int nt = 0; nt < S::NT; ++nt) {
            const int64_t k = class0 + S::column(nt);
            bias[nt] = k < m.weight.rows ? (m.bias ? m.bias[k] : 0.0f) : -INFINITY;
        }
        Acc c[S::MT][S::NT];
        products.clear(c);
        products.run(c, [&] { aim(tile + gridDim.x); });
        static_assert(S::NEXT, "a lane's classes are adjacent");
        char *to = reinterpret_cast<char *>(p + (row0 + S::row(0, 0)) * stride + (class0 - first_class) + S::column(0));
        int64_t row_bytes = stride * sizeof(T);
        asm volatile("" : "+s"(row_bytes));  // or its multiples are kept in registers over all tiles
        const int rows = static_cast<int>(std::min<int64_t>(S::M, m.hidden.rows - row0)) - S::row(0, 0);
        const float *own_lse = row_lse + S::row(0, 0), *own_grad = row_grad + S::row(0, 0);
        const int *own_target = row_target + S::row(0, 0);
        // Few rows have their target among a wavefront's classes, and few have none: a bit for each of its rows that does.
        uint64_t targets[(S::MT + 1) / 2];
#pragma unroll
        for (int k = 0; k < (S::MT + 1) / 2; ++k) {
            const int r = k * 64 + threadIdx.x % 64;
            const int target = r < S::MT * 32 ? row_target[S::wave_m() * (S::MT * 32) + r] : ELSEWHERE;
            targets[k] = __ballot(target >= 0 && target / (S::NT * 32) == S::wave_n());
            const uint64_t none = __ballot(target == NONE);
#pragma unroll
            for (int h = 0; h < 2 && k * 2 + h < S::MT; ++h) {
                uint32_t bits = static_cast<uint32_t>(none >> (h * 32));
                if (bits == 0) continue;
                bits >>= threadIdx.x % 64 / 32 * 4;
#pragma unroll
                for (int i = 0; i < 16; ++i)  // a lane's results are of four rows in each eight
#pragma unroll
                    for (int nt = 0; nt < S::NT; ++nt) c[k * 2 + h][nt][i] = bits >> (i / 4 * 8 + i % 4) & 1 ? -INFINITY : c[k * 2 + h][nt][i];
            }
        }
        char *at = to;  // a lane's results are of four rows in every eight
#pragma unroll
        for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
            for (int i = 0; i < 16; i += 4, at += 8 * row_bytes) {
                __builtin_amdgcn_sched_barrier(0);  // the numbers of four rows at a time, or they fill the registers
                const int down = mt * 32 + i * 2;
                const Chunk l = *reinterpret_cast<const Chunk *>(own_lse + down), g = *reinterpret_cast<const Chunk *>(own_grad + down);
                auto rows_of_four = [&](auto TARGETS) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        Pack<T, S::NT> out, rest;
#pragma unroll
                        for (int nt = 0; nt < S::NT; ++nt) {
                            float e = exp_from<T>(c[mt][nt][i + k] + bias[nt], l[k]);
                            if (TARGETS() && own_target[down + k] == S::column(nt)) e -= 1.0f;
                            e *= g[k];
                            sum[nt] += e;
                            out.v[nt] = narrow<T>(e);
                            if constexpr (TWO) rest.v[nt] = narrow<T>(e - widen(out.v[nt]));
                        }
                        if (down + k < rows) {
                            *reinterpret_cast<Pack<T, S::NT> *>(at + k * row_bytes) = out;
                            if constexpr (TWO) *reinterpret_cast<Pack<T, S::NT> *>(at + k * row_bytes + plane * sizeof(T)) = rest;
                        }
                    }
                };
                if (targets[mt / 2] >> (mt % 2 * 32 + i * 2) & 255) rows_of_four(std::true_type());
                else rows_of_four(std::false_type());
            }
        if (bias_parts) {
#pragma unroll
            for (int nt = 0; nt < S::NT; ++nt) {
                sum[nt] += __shfl_xor(sum[nt], 32, 64);
                if (threadIdx.x % 64 < 32) sums[S::wave_m() * S::N + S::column(nt)] = sum[nt];
            }
            __syncthreads();
            for (int i = threadIdx.x; i < S::N; i += S::THREADS) {
                float all = sums[i];
                for (int w = 1; w < S::WAVES_M; ++w) all += sums[w * S::N + i];
                bias_parts[this_row_tile * stride + (class0 - first_class) + i] = all;
            }
        }
    }
}

// C = A B with B across memory.  Each of `splits` parts of the sum's axis goes to a result of its own, [splits][rows][dim]
// float32, added to what is there where `add` says so; or (out) the one part is the result.
// TWO: A has two planes, whose products are added.  Where A lies along memory its rows are the batch's, elsewhere the sum goes over those.
// scale: of the results, or null.  p of 16,384 rows and 32,768
// classes, 512 columns, bfloat16: 706 us for hidden's gradient, 636 for weight's, 778 and 864 TFLOP/s; 4,099 x 20,011, 128 columns, float32:
// 230 and 238 us, 91 and 88, the matrix core busy for 78 %.
template <class T, class S, bool A_ALONG, bool TWO>
__global__ __launch_bounds__(S::THREADS, 2) void product_kernel(Operand<T> a, Operand<T> b, int64_t dim, uint32_t row_tiles,
                                                             uint32_t column_tiles, uint32_t splits, int64_t split_depth, int64_t plane,
                                                             const float *scale, float *parts, bool add, T *out)
{
    extern __shared__ char lds[];
    Products<T, S, A_ALONG, false> products(a, b, lds);
    const uint32_t tiles = row_tiles * column_tiles * splits;
    uint32_t column_tile = 0, row_tile = 0;
    auto aim = [&](uint32_t tile, int64_t from) {
        if (tile >= tiles) return;
        tile_of(tile, row_tiles * splits, column_tiles, row_tile, column_tile);
        const int64_t depth0 = row_tile / row_tiles * split_depth;
        products.aim(int64_t{S::M} * (row_tile % row_tiles), int64_t{S::N} * column_tile, depth0, std::min(a.depth, depth0 + split_depth), 0, from);
    };
    aim(blockIdx.x, 0);
    const float by = scale ? *scale : 1.0f;
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t column0 = int64_t{S::N} * column_tile, row0 = int64_t{S::M} * (row_tile % row_tiles), split = row_tile / row_tiles;
        Acc c[S::MT][S::NT];
        products.clear(c);
        if constexpr (TWO) products.run(c, [&] { aim(tile, plane); });
        products.run(c, [&] { aim(tile + gridDim.x, 0); });
        const int rows = static_cast<int>(std::min<int64_t>(S::M, a.rows - row0)) - S::row(0, 0);
        const int64_t at = (row0 + S::row(0, 0)) * dim + column0 + S::column(0);
        const int wave_m = __builtin_amdgcn_readfirstlane(S::wave_m());
        auto each = [&](auto store) {
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt) {
                // rows of the batch without a target get zeros, whatever the weights are
                uint32_t here = 0;
                if constexpr (A_ALONG) here = bits_of<uint32_t>(a.has, row0 / 32 + wave_m * S::MT + mt) >> (threadIdx.x % 64 / 32 * 4);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int down = mt * 32 + i / 4 * 8 + i % 4;
#pragma unroll
                    for (int nt = 0; nt < S::NT; ++nt)
                        if (down < rows && column0 + S::column(nt) < dim)
                            store(down * dim + nt * 32, !A_ALONG || here >> (i / 4 * 8 + i % 4) & 1 ? c[mt][nt][i] : 0.0f);
                }
            }
        };
        static_assert(!S::NEXT, "a lane's columns are 32 apart");
        if (out) {
            T *to = out + at;
            each([&](int64_t k, float v) { to[k] = narrow<T>(by * v); });
        } else {
            float *to = parts + split * a.rows * dim + at;
            if (add) each([&](int64_t k, float v) { to[k] += by * v; });
            else each([&](int64_t k, float v) { to[k] = by * v; });
        }
    }
}

// The sum of the splits, a lane for each result.
template <class T>
__global__ __launch_bounds__(256) void parts_kernel(const float *parts, int64_t splits, int64_t n, T *out)
{
    for (int64_t i = int64_t{256} * blockIdx.x + threadIdx.x; i < n; i += int64_t{256} * gridDim.x) {
        float s = 0;
#pragma unroll 8
        for (int64_t k = 0; k < splits; ++k) s += parts[k * n + i];
        out[i] = narrow<T>(s);
    }
}

// The same where there are many splits, of few results: 64 of a workgroup, 16 wavefronts on them in turn (512 splits of 512 results: 4 us,
// against 110).
template <class T>
__global__ __launch_bounds__(1024) void many_parts_kernel(const float *parts, int64_t splits, int64_t n, T *out)
{
    __shared__ float lds[16][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    for (int64_t i0 = int64_t{64} * blockIdx.x; i0 < n; i0 += int64_t{64} * gridDim.x) {
        const int64_t i = std::min(i0 + lane, n - 1);
        float s = 0;
#pragma unroll 8
        for (int64_t k = wave; k < splits; k += 16) s += parts[k * n + i];
        __syncthreads();
        lds[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && i0 + lane < n) {
#pragma unroll
            for (int w = 1; w < 16; ++w) s += lds[w][lane];
            out[i] = narrow<T>(s);
        }
    }
}

// The sum of the tiles of rows, of 64 classes a workgroup, 16 wavefronts on them in turn.
__global__ __launch_bounds__(1024) void bias_kernel(const float *parts, int64_t row_tiles, int64_t stride, int64_t n, const float *scale,
                                                    float *grad_bias)
{
    __shared__ float lds[16][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const int64_t k = int64_t{64} * blockIdx.x + lane;
    float s = 0;
#pragma unroll 4
    for (int64_t t = wave; t < row_tiles; t += 16) s += parts[t * stride + std::min(k, n - 1)];
    lds[wave][lane] = s;
    __syncthreads();
    if (wave > 0 || k >= n) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += lds[w][lane];
    grad_bias[k] = scale ? *scale * s : s;
}

// The largest finite magnitude of x over the rows that have a target (TARGETS), a part of it for each workgroup; 1, in
// the last launch, where there is none above 0.
constexpr int SCALE_PARTS = 256;

template <bool TARGETS>
__global__ __launch_bounds__(1024) void scale_kernel(const float *x, const int32_t *target, int64_t n_classes, int64_t n, bool last, float *out)
{
    __shared__ float lds[16];
    float most = 0;
#pragma unroll 4
    for (int64_t i = int64_t{1024} * blockIdx.x + threadIdx.x; i < n; i += int64_t{1024} * gridDim.x) {
        const float v = fabsf(x[i]);
        const int32_t t = TARGETS ? target[i] : 0;
        most = fmaxf(most, ((v < INFINITY) & (t >= 0) & (t < n_classes)) ? v : 0.0f);
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) most = fmaxf(most, __shfl_xor(most, d, 64));
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) most = fmaxf(most, lds[w]);
        out[blockIdx.x] = most > 0 || !last ? most : 1.0f;
    }
}

template <class T>
__global__ __launch_bounds__(256) void zero_kernel(T *to, int64_t n)
{
    for (int64_t i = int64_t{256} * blockIdx.x + threadIdx.x; i < n; i += int64_t{256} * gridDim.x) to[i] = T(0);
}

// Rows that are not whole in 16 bytes, into ones that are, with zeros behind them.
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(const T *from, int64_t stride, int64_t n_rows, int64_t dim, T *to, int64_t packed)
{
    const int64_t n = n_rows * packed;
    for (int64_t i = int64_t{256} * blockIdx.x + threadIdx.x; i < n; i += int64_t{256} * gridDim.x) {
        const int64_t r = i / packed, k = i % packed;
        to[i] = k < dim ? from[r * stride + k] : T(0);
    }
}

// ---- what a call launches

// A workgroup's tile.  Small: 4 wavefronts and 128 x 128, of which a CU has two.  Large: 8 wavefronts and 256 x 256, where bfloat16
// products have enough of them: half the traffic to LDS and a third less from it for as many products (16,384 x 65,536 logits over 512
// values: 1.23 to 1.32 ms, against 1.58).  float32 products are bound by the matrix core and gain nothing (4,099 x 20,011 logits over 128: 257 us, against 255).
// Of fewer than 256 rows or classes it would be empty in part, and its one plane of p would have few of them to be right on average over: 1 row, 70,000
// classes and 64 values take 72 us a step in Small, against 100; 66,001 rows, 10 classes and 512 values 150, against 179; but 255 rows, 66,000
// classes and 512 values 250, with two planes, against 227 with one.
// Tiny: 64 x 64, where there are so few tiles that the time of one counts, or so few rows or classes that most of a larger one
// would be empty; float32 products, whose steps take sixteen times as long, sooner than bfloat16 ones.  Both calls, in us: 1,021 rows
// and 10 classes 31, against 57 in Small; 1 row and 100,000 classes 81, against 130 (both float32); 60 rows and 30,000 classes 50, against 57
// (bfloat16).
struct Tiny {
    static constexpr int TILE = 64, RESIDENT = 512;
    template <bool NEXT>
    using Of = Shape<64, 64, 2, 2, NEXT>;
};
struct Small {
    static constexpr int TILE = 128, RESIDENT = 512;
    template <bool NEXT>
    using Of = Shape<128, 128, 2, 2, NEXT>;
};
struct Large {
    static constexpr int TILE = 256, RESIDENT = 256;
    template <bool NEXT>
    using Of = Shape<256, 256, 2, 4, NEXT>;
};

template <class S>
constexpr size_t lds_bytes()
{
    // two steps' tiles; what tiles are finished with, at most: of the wavefronts [WAVES_M][N] pairs, and twice [3][M] numbers
    return 2 * (S::M + S::N) * STEP + (2 * S::WAVES_M * S::N + 6 * S::M) * sizeof(float);
}

template <class S, auto *KERNEL, class... Args>
hipError_t launch_product(dim3 grid, hipStream_t stream, Args... args)
{
    if (const hipError_t e = allow_lds<KERNEL>(lds_bytes<S>())) return e;
    hipLaunchKernelGGL(KERNEL, grid, dim3(S::THREADS), lds_bytes<S>(), stream, args...);
    return hipGetLastError();
}

dim3 grid_of(int64_t n, int64_t most = 8192) { return dim3(static_cast<uint32_t>(std::max<int64_t>(1, std::min(n, most)))); }

enum { TINY, SMALL, LARGE };

// The parts of a call's workspace, in bytes from its start; and its sizes.
struct Plan {
    int size;                       // and what it is
    int64_t tile, resident;
    int64_t packed;                 // values of a packed row
    int64_t hidden = -1, weight = -1;  // packed operands; -1: used where they are
    int64_t class_tiles, row_tiles;
    int64_t parts, target;          // forward
    int64_t piece, pieces, stride;  // classes of a piece, a multiple of a tile's; values of a row of p
    int64_t plane, scale;           // values of a plane of p, where there are two (else 0); -1: grad_loss as it is
    int64_t has;                    // a bit for each row that has a target, in whole tiles
    int64_t p, bias, hidden_splits, hidden_parts, weight_splits, weight_parts;
    int64_t bytes = 0;

    int64_t part(int64_t n)
    {
        const int64_t at = bytes;
        bytes += round_up(n, 256);
        return at;
    }
};

Plan plan_operands(const head_classes &c)
{
    Plan p{};
    p.hidden = p.weight = -1;
    auto tiles = [&](int64_t tile) { return ceil_div(c.n_rows, tile) * ceil_div(c.n_classes, tile); };
    const bool narrow = c.n_rows <= Tiny::TILE || c.n_classes <= Tiny::TILE;
    const bool tiny = c.dtype == HEAD_F32 ? narrow || tiles(Small::TILE) < Small::RESIDENT : tiles(Small::TILE) < Small::RESIDENT / 2;
    const bool large = c.dtype == HEAD_BF16 && std::min(c.n_rows, c.n_classes) >= Large::TILE && tiles(Large::TILE) >= Large::RESIDENT;
    p.size = large ? LARGE : tiny ? TINY : SMALL;
    p.tile = p.size == LARGE ? Large::TILE : p.size == TINY ? Tiny::TILE : Small::TILE;
    p.resident = p.size == LARGE ? Large::RESIDENT : p.size == TINY ? Tiny::RESIDENT : Small::RESIDENT;
    const int e = value_bytes(c.dtype);
    p.packed = round_up(c.dim, 16 / e);
    auto whole = [&](const void *at, int64_t stride) { return (address(at) | static_cast<uint64_t>(stride * e) | static_cast<uint64_t>(c.dim * e)) % 16 == 0; };
    if (!whole(c.hidden, c.hidden_stride)) p.hidden = p.part(c.n_rows * p.packed * e);
    if (!whole(c.weight, c.weight_stride)) p.weight = p.part(c.n_classes * p.packed * e);
    return p;
}

Plan plan_forward(const head_classes &c)
{
    Plan p = plan_operands(c);
    p.class_tiles = ceil_div(c.n_classes, p.tile);
    p.row_tiles = ceil_div(c.n_rows, p.tile);
    p.parts = p.part(p.class_tiles * c.n_rows * static_cast<int64_t>(sizeof(float2)));
    p.target = p.part(c.n_rows * 4);
    return p;
}

// Parts of a sum of `depth` such that `tiles` tiles of each fill the device, each part having at least 2 steps.
int64_t splits_of(int64_t tiles, int64_t resident, int64_t depth, int64_t step)
{
    return std::max<int64_t>(1, std::min(resident / std::max<int64_t>(1, tiles), ceil_div(depth, 2 * step)));
}

Plan plan_backward(const head_classes &c)
{
    Plan p = plan_operands(c);
    const int e = value_bytes(c.dtype);
    const int64_t step = STEP / e;
    p.piece = std::min(round_up(c.n_classes, p.tile), std::max<int64_t>(1024, PIECE_BYTES / (std::max<int64_t>(1, c.n_rows) * e) / 1024 * 1024));
    p.pieces = ceil_div(c.n_classes, p.piece);
    p.row_tiles = ceil_div(c.n_rows, p.tile);
    // Rows a power of two apart would lie in few of the memory's channels: a row more than a piece by 256 bytes goes through all.
    p.stride = p.piece + 256 / e;
    const bool narrow = c.dtype == HEAD_BF16;
    p.plane = narrow && p.size != LARGE ? c.n_rows * p.stride : 0;
    p.scale = narrow && p.size == LARGE ? p.part(4 * (1 + SCALE_PARTS)) : -1;
    p.has = p.part(p.row_tiles * p.tile / 8);
    p.p = p.part((p.plane ? 2 : 1) * c.n_rows * p.stride * e);
    p.bias = p.part(p.row_tiles * p.stride * 4);
    const int64_t columns = ceil_div(c.dim, p.tile);
    p.hidden_splits = splits_of(p.row_tiles * columns, p.resident, p.piece, step);
    p.hidden_parts = p.hidden_splits * p.pieces > 1 ? p.part(p.hidden_splits * c.n_rows * c.dim * 4) : -1;
    p.weight_splits = splits_of(ceil_div(p.piece, p.tile) * columns, p.resident, c.n_rows, step);
    p.weight_parts = p.weight_splits > 1 ? p.part(p.weight_splits * p.piece * c.dim * 4) : -1;
    return p;
}

template <class T>
Model<T> model_of(const head_classes &c, const Plan &p, char *workspace, hipStream_t stream)
{
    auto operand = [&](const void *at, int64_t stride, int64_t rows, int64_t packed_at) {
        const T *from = static_cast<const T *>(at);
        if (packed_at < 0) return Operand<T>{from, stride, rows, c.dim};
        T *to = reinterpret_cast<T *>(workspace + packed_at);
        hipLaunchKernelGGL((pack_kernel<T>), grid_of(ceil_div(rows * p.packed, 256)), dim3(256), 0, stream, from, stride,
                           rows, c.dim, to, p.packed);
        return Operand<T>{to, p.packed, rows, p.packed};
    };
    return Model<T>{operand(c.hidden, c.hidden_stride, c.n_rows, p.hidden), operand(c.weight, c.weight_stride, c.n_classes, p.weight), c.bias,
                    c.target};
}

template <class T, class Size>
hipError_t forward(const head_classes &c, const Plan &p, float *loss, float *lse, char *workspace, hipStream_t stream)
{
    using Forward = typename Size::template Of<false>;
    const Model<T> m = model_of<T>(c, p, workspace, stream);
    if (const hipError_t e = hipGetLastError()) return e;
    float2 *parts = reinterpret_cast<float2 *>(workspace + p.parts);
    float *target_logit = reinterpret_cast<float *>(workspace + p.target);
    const int64_t tiles = p.class_tiles * p.row_tiles;
    if (const hipError_t e = launch_product<Forward, lse_kernel<T, Forward>>(grid_of(tiles, Size::RESIDENT), stream, m, static_cast<uint32_t>(p.row_tiles),
                                                                                static_cast<uint32_t>(p.class_tiles), parts, target_logit)) return e;
    auto *join = c.n_rows <= 4096 ? lse_join_kernel<4> : lse_join_kernel<32>;
    hipLaunchKernelGGL(join, grid_of(ceil_div(c.n_rows, c.n_rows <= 4096 ? 4 : 32)), dim3(256), 0, stream, c.n_rows, c.n_classes, p.class_tiles,
                       parts, target_logit, c.target, loss, lse);
    return hipGetLastError();
}

template <class T>
void add_parts(const float *parts, int64_t splits, int64_t n, T *out, hipStream_t stream)
{
    if (splits >= 32) hipLaunchKernelGGL((many_parts_kernel<T>), grid_of(ceil_div(n, 64)), dim3(1024), 0, stream, parts, splits, n, out);
    else hipLaunchKernelGGL((parts_kernel<T>), grid_of(ceil_div(n, 256)), dim3(256), 0, stream, parts, splits, n, out);
}

template <class T, class Size>
hipError_t backward(const head_classes &c, const Plan &plan, const float *lse, const float *grad_loss, T *grad_hidden, T *grad_weight, float *grad_bias,
                    char *workspace, hipStream_t stream)
{
    using Backward = typename Size::template Of<true>;
    using Gradient = typename Size::template Of<false>;
    if (c.n_rows == 0) {
        hipLaunchKernelGGL((zero_kernel<T>), grid_of(ceil_div(c.n_classes * c.dim, 256)), dim3(256), 0, stream,
                           grad_weight, c.n_classes * c.dim);
        if (grad_bias)
            hipLaunchKernelGGL((zero_kernel<float>), grid_of(ceil_div(c.n_classes, 256)), dim3(256), 0, stream, grad_bias,
                               c.n_classes);
        return hipGetLastError();
    }
    const Model<T> m = model_of<T>(c, plan, workspace, stream);
    if (const hipError_t e = hipGetLastError()) return e;
    T *p = reinterpret_cast<T *>(workspace + plan.p);
    uint64_t *has = reinterpret_cast<uint64_t *>(workspace + plan.has);
    float *bias_parts = grad_bias ? reinterpret_cast<float *>(workspace + plan.bias) : nullptr;
    float *hidden_parts = plan.hidden_parts < 0 ? nullptr : reinterpret_cast<float *>(workspace + plan.hidden_parts);
    float *weight_parts = plan.weight_parts < 0 ? nullptr : reinterpret_cast<float *>(workspace + plan.weight_parts);
    float *scale = plan.scale < 0 ? nullptr : reinterpret_cast<float *>(workspace + plan.scale);
    if (scale) {
        const bool one = c.n_rows <= 1 << 16;  // else the parts of many workgroups, behind the scale, first
        if (one) {
            hipLaunchKernelGGL(scale_kernel<true>, dim3(1), dim3(1024), 0, stream, grad_loss, c.target, c.n_classes, c.n_rows, true, scale);
        } else {
            hipLaunchKernelGGL(scale_kernel<true>, dim3(SCALE_PARTS), dim3(1024), 0, stream, grad_loss, c.target, c.n_classes, c.n_rows, false, scale + 1);
            hipLaunchKernelGGL(scale_kernel<false>, dim3(1), dim3(1024), 0, stream, scale + 1, nullptr, c.n_classes, SCALE_PARTS, true, scale);
        }
    }
    constexpr bool TWO = sizeof(T) == 2 && !std::is_same_v<Size, Large>;
    const int64_t step = STEP / sizeof(T);
    const uint32_t columns = static_cast<uint32_t>(ceil_div(c.dim, Gradient::N));
    for (int64_t piece = 0; piece < plan.pieces; ++piece) {
        const int64_t first = piece * plan.piece, classes = std::min(plan.piece, c.n_classes - first);
        const int64_t class_tiles = ceil_div(classes, Backward::N), stride = plan.stride;
        const int64_t p_tiles = class_tiles * plan.row_tiles;
        if (const hipError_t e = launch_product<Backward, p_kernel<T, Backward, TWO>>(grid_of(p_tiles, Size::RESIDENT), stream, m, lse, grad_loss, first,
                                                                                 static_cast<uint32_t>(plan.row_tiles),
                                                                                 static_cast<uint32_t>(class_tiles), p, stride, plan.plane, scale, bias_parts, has))
            return e;
        if (grad_bias)
            hipLaunchKernelGGL(bias_kernel, dim3(static_cast<uint32_t>(ceil_div(classes, 64))), dim3(1024), 0, stream, bias_parts,
                               plan.row_tiles, stride, classes, scale, grad_bias + first);
        // grad_hidden [n_rows][dim] += p [n_rows][classes] weight [classes][dim]
        {
            const uint32_t row_tiles = static_cast<uint32_t>(ceil_div(c.n_rows, Gradient::M));
            const int64_t depth = round_up(ceil_div(classes, plan.hidden_splits), step);
            const Operand<T> a{p, stride, c.n_rows, classes, has}, b{m.weight.at + first * m.weight.stride, m.weight.stride, m.weight.depth, classes};
            const int64_t tiles = int64_t{row_tiles} * columns * plan.hidden_splits;
            if (const hipError_t e = launch_product<Gradient, product_kernel<T, Gradient, true, TWO>>(grid_of(tiles, Size::RESIDENT), stream, a, b, c.dim, row_tiles, columns,
                                                                                                 static_cast<uint32_t>(plan.hidden_splits), depth, plan.plane, scale, hidden_parts,
                                                                                                 piece > 0, hidden_parts ? nullptr : grad_hidden))
                return e;
        }
        // grad_weight [classes][dim] = p^T [classes][n_rows] hidden [n_rows][dim]
        {
            const uint32_t row_tiles = static_cast<uint32_t>(ceil_div(classes, Gradient::M));
            const int64_t depth = round_up(ceil_div(c.n_rows, plan.weight_splits), step);
            const Operand<T> a{p, stride, classes, c.n_rows}, b{m.hidden.at, m.hidden.stride, m.hidden.depth, c.n_rows, has};
            const int64_t tiles = int64_t{row_tiles} * columns * plan.weight_splits;
            T *out = grad_weight + first * c.dim;
            if (const hipError_t e = launch_product<Gradient, product_kernel<T, Gradient, false, TWO>>(grid_of(tiles, Size::RESIDENT), stream, a, b, c.dim, row_tiles, columns,
                                                                                                  static_cast<uint32_t>(plan.weight_splits), depth, plan.plane, scale, weight_parts,
                                                                                                  false, weight_parts ? nullptr : out))
                return e;
            if (weight_parts) add_parts(weight_parts, plan.weight_splits, classes * c.dim, out, stream);
        }
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (hidden_parts) add_parts(hidden_parts, plan.hidden_splits, c.n_rows * c.dim, grad_hidden, stream);
    return hipGetLastError();
}

}  // namespace

int64_t cross_entropy_bytes(const head_classes &c) { return c.n_rows ? plan_forward(c).bytes : 0; }

hipError_t launch_cross_entropy(const head_classes &c, float *loss, float *lse, void *workspace, hipStream_t stream)
{
    char *w = static_cast<char *>(workspace);
    const Plan p = plan_forward(c);
    if (c.dtype == HEAD_F32)
        return p.size == TINY ? forward<float, Tiny>(c, p, loss, lse, w, stream) : forward<float, Small>(c, p, loss, lse, w, stream);
    return p.size == LARGE  ? forward<bf16, Large>(c, p, loss, lse, w, stream)
           : p.size == TINY ? forward<bf16, Tiny>(c, p, loss, lse, w, stream)
                            : forward<bf16, Small>(c, p, loss, lse, w, stream);
}

int64_t cross_entropy_grad_bytes(const head_classes &c) { return c.n_rows ? plan_backward(c).bytes : 0; }

hipError_t launch_cross_entropy_grad(const head_classes &c, const float *lse, const float *grad_loss, void *grad_hidden,
                                     void *grad_weight, float *grad_bias, void *workspace, hipStream_t stream)
{
    char *w = static_cast<char *>(workspace);
    const Plan p = plan_backward(c);
    if (c.dtype == HEAD_F32) {
        float *gh = static_cast<float *>(grad_hidden), *gw = static_cast<float *>(grad_weight);
        return p.size == TINY ? backward<float, Tiny>(c, p, lse, grad_loss, gh, gw, grad_bias, w, stream)
                              : backward<float, Small>(c, p, lse, grad_loss, gh, gw, grad_bias, w, stream);
    }
    bf16 *gh = static_cast<bf16 *>(grad_hidden), *gw = static_cast<bf16 *>(grad_weight);
    return p.size == LARGE  ? backward<bf16, Large>(c, p, lse, grad_loss, gh, gw, grad_bias, w, stream)
           : p.size == TINY ? backward<bf16, Tiny>(c, p, lse, grad_loss, gh, gw, grad_bias, w, stream)
                            : backward<bf16, Small>(c, p, lse, grad_loss, gh, gw, grad_bias, w, stream);
}

}  // namespace head_impl
