// Matrix products C = A B of the trainable head, on gfx950.  What head_loss.hip and head_linear.hip share: operands, the shapes of a workgroup's tile,
// their order over the XCDs, and the kernels that add parts; and the body that head_loss.hip's kernels run on (Tile, Products; that of head_linear.hip is in
// head_flow.hpp).  There a workgroup makes tiles of C one after the other; A and B come to LDS in tiles of 128 bytes of the sum's axis, by the loads that
// bypass registers, while the matrix core works on the tiles before.  An operand lies in memory with the sum's axis along its rows or across
// them.  bfloat16 products run on the 32x32x16 matrix instruction, float32 ones on the 32x32x2 float32 one, whose rate, a sixteenth, then
// bounds them; both accumulate in float32.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "head_device.hpp"

namespace head_impl {
namespace {

constexpr int STEP = 128;                       // bytes of the sum's axis in a tile

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
                at[j] = ((lane % SLOTS) ^ key(r)) * VALUES;
                const int64_t row = row0 + r - in + in % 32 * NT + in / 32;
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

// A workgroup's tile.  Small: 4 wavefronts and 128 x 128, of which a CU has two.  Large: 8 wavefronts and 256 x 256, where bfloat16
// products have enough of them.  Tiny: 64 x 64, where there are so few tiles that the time of one counts.  Who chooses says what it measured.
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

inline dim3 grid_of(int64_t n, int64_t most = 8192) { return dim3(static_cast<uint32_t>(std::max<int64_t>(1, std::min(n, most)))); }

// Parts of a sum of `depth` such that `tiles` tiles of each fill the device, each part having at least 2 steps.
inline int64_t splits_of(int64_t tiles, int64_t resident, int64_t depth, int64_t step)
{
    return std::max<int64_t>(1, std::min(resident / std::max<int64_t>(1, tiles), ceil_div(depth, 2 * step)));
}

template <class T>
void add_parts(const float *parts, int64_t splits, int64_t n, T *out, hipStream_t stream)
{
    if (splits >= 32) hipLaunchKernelGGL((many_parts_kernel<T>), grid_of(ceil_div(n, 64)), dim3(1024), 0, stream, parts, splits, n, out);
    else hipLaunchKernelGGL((parts_kernel<T>), grid_of(ceil_div(n, 256)), dim3(256), 0, stream, parts, splits, n, out);
}

}  // namespace
}  // namespace head_impl
