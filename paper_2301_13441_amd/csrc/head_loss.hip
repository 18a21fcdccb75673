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

#include "head_device.hpp"

namespace head_impl {
namespace {

constexpr int64_t MAX_GRID = 1 << 22;
constexpr int STEP = 128;                       // bytes of the sum's axis in a tile
constexpr int64_t PIECE_BYTES = int64_t{1} << 30;  // of p in the workspace, where rows are not too many for that

using Acc = float __attribute__((ext_vector_type(16)));
using Bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using Chunk = float __attribute__((ext_vector_type(4)));  // 16 bytes of either type

__device__ const Chunk g_zeros[1] = {};

using GlobalChunk = const __attribute__((address_space(1))) void *;
using LdsChunk = __attribute__((address_space(3))) void *;

__device__ __forceinline__ void to_lds(const void *from, char *to)  // 16 bytes a lane, the wavefront's 1024 adjacent
{
    __builtin_amdgcn_global_load_lds((GlobalChunk)(from), (LdsChunk)(to), 16, 0, 0);
}

// An operand: `rows` along the result's axis, `depth` along the sum's.
template <class T>
struct Operand {
    const T *at;
    int64_t stride;
    int64_t rows, depth;
};

// Tiles of ROWS x 128 bytes of an operand.  ALONG: the sum's axis lies along memory; row r's chunk c of 16 bytes is in slot
// c ^ (r / SPREAD % 8), so that the 8 lanes that read the same chunk of 8 rows SPREAD apart meet 8 different bank groups.
// Otherwise a row of the tile holds the ROWS values of one index of the sum.
template <class T, bool ALONG, int ROWS, int THREADS, int SPREAD>
struct Tile {
    static constexpr int VALUES = 16 / sizeof(T), DEPTH = STEP / sizeof(T), BYTES = ROWS * STEP;
    static constexpr int LOADS = BYTES / (THREADS * 16);

    static __device__ __forceinline__ void load(const Operand<T> &o, int64_t row0, int64_t depth0, char *lds)
    {
        const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int part = j * (THREADS / 64) + wave;  // 1024 bytes of the tile
            const void *from = g_zeros;
            if constexpr (ALONG) {
                const int r = part * 8 + lane / 8;
                const int chunk = (lane % 8) ^ (r / SPREAD % 8);
                const int64_t row = std::min(row0 + r, o.rows - 1), k = depth0 + chunk * VALUES;
                if (k < o.depth) from = o.at + row * o.stride + k;
            } else {
                constexpr int CHUNKS = ROWS / VALUES;  // of a row of the tile
                const int64_t k = depth0 + (part * 64 + lane) / CHUNKS, row = row0 + (part * 64 + lane) % CHUNKS * VALUES;
                if (k < o.depth && row < o.rows) from = o.at + k * o.stride + row;
            }
            to_lds(from, lds + part * 1024);
        }
    }

    // What lane `lane` holds of 32 rows in a matrix instruction: of row r (its own, lane % 32's), the values of chunk
    // 2 * kk + lane / 32.
    static __device__ __forceinline__ Chunk read(const char *lds, int r, int kk)
    {
        const int chunk = 2 * kk + threadIdx.x % 64 / 32;
        if constexpr (ALONG) {
            return *reinterpret_cast<const Chunk *>(lds + r * STEP + ((chunk ^ (r / SPREAD % 8)) * 16));
        } else {
            Pack<T, VALUES> p;
#pragma unroll
            for (int j = 0; j < VALUES; ++j) p.v[j] = reinterpret_cast<const T *>(lds)[(chunk * VALUES + j) * ROWS + r];
            return *reinterpret_cast<Chunk *>(&p);
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

// c = A[row0.., depth0..depth1) B[.., column0..): A and B of 2 * (S::M + S::N) * STEP bytes of LDS.
template <class T, class S, bool A_ALONG, bool B_ALONG>
__device__ __forceinline__ void product(const Operand<T> &a, const Operand<T> &b, int64_t row0, int64_t column0, int64_t depth0,
                                        int64_t depth1, char *lds, Acc (&c)[S::MT][S::NT])
{
    using A = Tile<T, A_ALONG, S::M, S::THREADS, 1>;
    using B = Tile<T, B_ALONG, S::N, S::THREADS, S::NEXT ? S::NT : 1>;
    constexpr int BYTES = A::BYTES + B::BYTES;
#pragma unroll
    for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < S::NT; ++nt) c[mt][nt] = Acc{};
    auto load = [&](int64_t depth, int which) {
        A::load(a, row0, depth, lds + which * BYTES);
        B::load(b, column0, depth, lds + which * BYTES + A::BYTES);
    };
    __syncthreads();  // who still reads what LDS held before
    if (depth0 < depth1) load(depth0, 0);
    int which = 0;
    for (int64_t depth = depth0; depth < depth1; depth += A::DEPTH, which ^= 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();  // this step's tiles are there, and nobody reads the other ones any more
        if (depth + A::DEPTH < depth1) load(depth + A::DEPTH, which ^ 1);
        const char *la = lds + which * BYTES, *lb = la + A::BYTES;
#pragma unroll
        for (int kk = 0; kk < STEP / 32; ++kk) {
            Chunk x[S::MT], y[S::NT];
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt) x[mt] = A::read(la, S::wave_m() * (S::MT * 32) + mt * 32 + threadIdx.x % 32, kk);
#pragma unroll
            for (int nt = 0; nt < S::NT; ++nt) y[nt] = B::read(lb, S::column(nt), kk);
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
                for (int nt = 0; nt < S::NT; ++nt) multiply(x[mt], y[nt], c[mt][nt], T());
        }
    }
    __syncthreads();  // LDS is free
}

// exp(x) for x <= 0 or little above, to a rounding or two: the product with log2(e) is taken in two parts, for the rounding
// of one would be multiplied by x.
__device__ __forceinline__ float exp_of(float x)
{
    constexpr float LOG2E = 1.44269502162933349609375f, REST = 1.925963033500011079e-08f;
    const float t = x * LOG2E;
    const float e = __builtin_amdgcn_exp2f(t);
    const float rest = fmaf(x, LOG2E, -t) + x * REST;
    return fabsf(rest) < 1 ? fmaf(e, rest * 0.693147180559945f, e) : e;  // x infinite: no rest
}

template <class T>
struct Model {
    Operand<T> hidden, weight;  // [n_rows][dim], [n_classes][dim], whole in 16 bytes
    const float *bias;
    const int32_t *target;
};

// ---- forward

// Rows of C are classes and its columns rows of the batch, so that a lane has the values of one row in its registers.
template <class T, class S>
__global__ __launch_bounds__(S::THREADS) void lse_kernel(Model<T> m, int64_t class_tiles, int64_t tiles, float2 *parts, float *target_logit)
{
    extern __shared__ char lds[];
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t class0 = tile % class_tiles * S::M, row0 = tile / class_tiles * S::N;
        Acc c[S::MT][S::NT];
        product<T, S, true, true>(m.weight, m.hidden, class0, row0, 0, m.hidden.depth, lds, c);
        float *bias = reinterpret_cast<float *>(lds);
        float2 *most = reinterpret_cast<float2 *>(bias + S::M);  // [WAVES_M][N]
        for (int i = threadIdx.x; i < S::M; i += S::THREADS)
            bias[i] = class0 + i < m.weight.rows ? (m.bias ? m.bias[class0 + i] : 0.0f) : -INFINITY;
        __syncthreads();
#pragma unroll
        for (int nt = 0; nt < S::NT; ++nt) {
            const int64_t row = row0 + S::column(nt);
            const int64_t target = row < m.hidden.rows ? m.target[row] - class0 : -1;
            float top = -INFINITY;
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float v = c[mt][nt][i] += bias[S::row(mt, i)];
                    top = fmaxf(top, v);
                    if (target == S::row(mt, i) && class0 + target < m.weight.rows) target_logit[row] = v;
                }
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float from = top > -INFINITY ? top : 0.0f;
            float sum = 0;
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
                for (int i = 0; i < 16; ++i) sum += exp_of(c[mt][nt][i] - from);
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
                    all = make_float2(top, all.y * exp_of(all.x - from) + o.y * exp_of(o.x - from));
                }
                parts[class0 / S::M * m.hidden.rows + row0 + i] = all;
            }
    }
}

// The tiles' largest values and sums of a row become its lse.  32 rows of a workgroup, 8 lanes on each.
__global__ __launch_bounds__(256) void lse_join_kernel(int64_t n_rows, int64_t n_classes, int64_t class_tiles, const float2 *parts,
                                                       const float *target_logit, const int32_t *target, float *loss, float *lse)
{
    __shared__ float2 lds[8][32];
    const int lane = threadIdx.x / 32, r = threadIdx.x % 32;
    for (int64_t row0 = int64_t{32} * blockIdx.x; row0 < n_rows; row0 += int64_t{32} * gridDim.x) {
        const int64_t row = row0 + r;
        float2 all = make_float2(-INFINITY, 0);
        auto add = [&](float2 o) {
            const float top = fmaxf(all.x, o.x), from = top > -INFINITY ? top : 0.0f;
            all = make_float2(top, all.y * exp_of(all.x - from) + o.y * exp_of(o.x - from));
        };
        if (row < n_rows) {
#pragma unroll 4
            for (int64_t t = lane; t < class_tiles; t += 8) add(parts[t * n_rows + row]);
        }
        __syncthreads();
        lds[lane][r] = all;
        __syncthreads();
        if (lane == 0 && row < n_rows) {
            for (int i = 1; i < 8; ++i) add(lds[i][r]);
            const float log = logf(all.y);
            lse[row] = all.x + log;
            loss[row] = target[row] >= 0 && target[row] < n_classes ? log + (all.x - target_logit[row]) : 0.0f;
        }
    }
}

// ---- backward

// p of the classes from `class0` on, [n_rows][stride]: whole tiles, zero where there is no class.  bias_parts: the sums of
// a tile's rows, [tiles of rows][stride].
template <class T, class S>
__global__ __launch_bounds__(S::THREADS) void p_kernel(Model<T> m, const float *lse, const float *grad_loss, int64_t first_class,
                                                       int64_t class_tiles, int64_t tiles, T *p, int64_t stride, float *bias_parts)
{
    extern __shared__ char lds[];
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t class0 = first_class + tile % class_tiles * S::N, row0 = tile / class_tiles * S::M;
        Acc c[S::MT][S::NT];
        product<T, S, true, true>(m.hidden, m.weight, row0, class0, 0, m.hidden.depth, lds, c);
        float *row_lse = reinterpret_cast<float *>(lds), *row_grad = row_lse + S::M;
        int *row_target = reinterpret_cast<int *>(row_grad + S::M);
        float *sums = reinterpret_cast<float *>(row_target + S::M);  // [WAVES_M][N]
        for (int i = threadIdx.x; i < S::M; i += S::THREADS) {
            const int64_t row = row0 + i;
            const int target = row < m.hidden.rows ? m.target[row] : -1;
            const bool has = target >= 0 && target < m.weight.rows;
            row_lse[i] = has ? lse[row] : 0.0f;
            row_grad[i] = has ? grad_loss[row] : 0.0f;
            row_target[i] = has ? static_cast<int>(std::max<int64_t>(-1, std::min<int64_t>(S::N, target - class0))) : -2;
        }
        __syncthreads();
        float bias[S::NT], sum[S::NT] = {};
        bool is_class[S::NT];
#pragma unroll
        for (int nt = 0; nt < S::NT; ++nt) {
            const int64_t k = class0 + S::column(nt);
            is_class[nt] = k < m.weight.rows;
            bias[nt] = is_class[nt] && m.bias ? m.bias[k] : 0.0f;
        }
        T *to = p + (class0 - first_class) + S::column(0);
#pragma unroll
        for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = S::row(mt, i);
                const float l = row_lse[r], g = row_grad[r];
                const int target = row_target[r];
                Pack<T, S::NT> out;
#pragma unroll
                for (int nt = 0; nt < S::NT; ++nt) {
                    float v = g * (exp_of(c[mt][nt][i] + bias[nt] - l) - (S::column(nt) == target ? 1.0f : 0.0f));
                    if (!is_class[nt] || target == -2) v = 0;
                    sum[nt] += v;
                    out.v[nt] = narrow<T>(v);
                }
                static_assert(S::NEXT, "a lane's classes are adjacent");
                if (row0 + r < m.hidden.rows) *reinterpret_cast<Pack<T, S::NT> *>(to + (row0 + r) * stride) = out;
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
                bias_parts[row0 / S::M * stride + (class0 - first_class) + i] = all;
            }
        }
    }
}

// C = A B with B across memory.  Each of `splits` parts of the sum's axis goes to a result of its own, [splits][rows][dim]
// float32, added to what is there where `add` says so; or (out) the one part is the result.
template <class T, class S, bool A_ALONG>
__global__ __launch_bounds__(S::THREADS) void product_kernel(Operand<T> a, Operand<T> b, int64_t dim, int64_t row_tiles, int64_t column_tiles,
                                                             int64_t split_depth, int64_t tiles, float *parts, bool add, T *out)
{
    extern __shared__ char lds[];
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t column0 = tile % column_tiles * S::N, row0 = tile / column_tiles % row_tiles * S::M;
        const int64_t split = tile / column_tiles / row_tiles, depth0 = split * split_depth;
        Acc c[S::MT][S::NT];
        product<T, S, A_ALONG, false>(a, b, row0, column0, depth0, std::min(a.depth, depth0 + split_depth), lds, c);
#pragma unroll
        for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < S::NT; ++nt) {
                const int64_t column = column0 + S::column(nt);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int64_t row = row0 + S::row(mt, i);
                    if (row >= a.rows || column >= dim) continue;
                    if (out) out[row * dim + column] = narrow<T>(c[mt][nt][i]);
                    else {
                        float *to = parts + (split * a.rows + row) * dim + column;
                        *to = add ? *to + c[mt][nt][i] : c[mt][nt][i];
                    }
                }
            }
    }
}

template <class T>
__global__ __launch_bounds__(256) void parts_kernel(const float *parts, int64_t splits, int64_t n, T *out)
{
    for (int64_t i = int64_t{256} * blockIdx.x + threadIdx.x; i < n; i += int64_t{256} * gridDim.x) {
        float s = parts[i];
        for (int64_t k = 1; k < splits; ++k) s += parts[k * n + i];
        out[i] = narrow<T>(s);
    }
}

__global__ __launch_bounds__(256) void bias_kernel(const float *parts, int64_t row_tiles, int64_t stride, int64_t n, float *grad_bias)
{
    const int64_t k = int64_t{256} * blockIdx.x + threadIdx.x;
    if (k >= n) return;
    float s = 0;
#pragma unroll 8
    for (int64_t t = 0; t < row_tiles; ++t) s += parts[t * stride + k];
    grad_bias[k] = s;
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

using Forward = Shape<128, 128, 2, 2, false>;
using Backward = Shape<128, 128, 2, 2, true>;
using Gradient = Shape<128, 128, 2, 2, false>;

template <class S>
constexpr size_t lds_bytes()
{
    return 2 * (S::M + S::N) * STEP;
}

dim3 grid_of(int64_t n) { return dim3(static_cast<uint32_t>(std::max<int64_t>(1, std::min(n, MAX_GRID)))); }

// The parts of a call's workspace, in bytes from its start; and its sizes.
struct Plan {
    int64_t packed;                 // values of a packed row
    int64_t hidden = -1, weight = -1;  // packed operands; -1: used where they are
    int64_t class_tiles, row_tiles;
    int64_t parts, target;          // forward
    int64_t piece, pieces;          // classes of a piece, a multiple of a tile's
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
    p.class_tiles = ceil_div(c.n_classes, Forward::M);
    p.row_tiles = ceil_div(c.n_rows, Forward::N);
    p.parts = p.part(p.class_tiles * c.n_rows * static_cast<int64_t>(sizeof(float2)));
    p.target = p.part(c.n_rows * 4);
    return p;
}

// Parts of a sum of `depth` such that `tiles` tiles of each fill the device twice over, each part having at least 8 steps.
int64_t splits_of(int64_t tiles, int64_t depth, int64_t step)
{
    return std::max<int64_t>(1, std::min(512 / std::max<int64_t>(1, tiles), ceil_div(depth, 8 * step)));
}

Plan plan_backward(const head_classes &c)
{
    Plan p = plan_operands(c);
    const int e = value_bytes(c.dtype);
    const int64_t step = STEP / e;
    p.piece = std::min(round_up(c.n_classes, Backward::N), std::max<int64_t>(1024, PIECE_BYTES / (std::max<int64_t>(1, c.n_rows) * e) / 1024 * 1024));
    p.pieces = ceil_div(c.n_classes, p.piece);
    p.row_tiles = ceil_div(c.n_rows, Backward::M);
    p.p = p.part(c.n_rows * p.piece * e);
    p.bias = p.part(p.row_tiles * p.piece * 4);
    const int64_t columns = ceil_div(c.dim, Gradient::N);
    p.hidden_splits = splits_of(ceil_div(c.n_rows, Gradient::M) * columns, p.piece, step);
    p.hidden_parts = p.hidden_splits * p.pieces > 1 ? p.part(p.hidden_splits * c.n_rows * c.dim * 4) : -1;
    p.weight_splits = splits_of(ceil_div(p.piece, Gradient::M) * columns, c.n_rows, step);
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
        hipLaunchKernelGGL((pack_kernel<T>), grid_of(std::min<int64_t>(8192, ceil_div(rows * p.packed, 256))), dim3(256), 0, stream, from, stride,
                           rows, c.dim, to, p.packed);
        return Operand<T>{to, p.packed, rows, p.packed};
    };
    return Model<T>{operand(c.hidden, c.hidden_stride, c.n_rows, p.hidden), operand(c.weight, c.weight_stride, c.n_classes, p.weight), c.bias,
                    c.target};
}

template <class T>
hipError_t forward(const head_classes &c, float *loss, float *lse, char *workspace, hipStream_t stream)
{
    const Plan p = plan_forward(c);
    const Model<T> m = model_of<T>(c, p, workspace, stream);
    if (const hipError_t e = hipGetLastError()) return e;
    float2 *parts = reinterpret_cast<float2 *>(workspace + p.parts);
    float *target_logit = reinterpret_cast<float *>(workspace + p.target);
    const int64_t tiles = p.class_tiles * p.row_tiles;
    hipLaunchKernelGGL((lse_kernel<T, Forward>), grid_of(tiles), dim3(Forward::THREADS), lds_bytes<Forward>(), stream, m, p.class_tiles, tiles,
                       parts, target_logit);
    hipLaunchKernelGGL(lse_join_kernel, grid_of(ceil_div(c.n_rows, 32)), dim3(256), 0, stream, c.n_rows, c.n_classes, p.class_tiles, parts,
                       target_logit, c.target, loss, lse);
    return hipGetLastError();
}

template <class T>
hipError_t backward(const head_classes &c, const float *lse, const float *grad_loss, T *grad_hidden, T *grad_weight, float *grad_bias,
                    char *workspace, hipStream_t stream)
{
    if (c.n_rows == 0) {
        hipLaunchKernelGGL((zero_kernel<T>), grid_of(std::min<int64_t>(8192, ceil_div(c.n_classes * c.dim, 256))), dim3(256), 0, stream,
                           grad_weight, c.n_classes * c.dim);
        if (grad_bias)
            hipLaunchKernelGGL((zero_kernel<float>), grid_of(std::min<int64_t>(8192, ceil_div(c.n_classes, 256))), dim3(256), 0, stream, grad_bias,
                               c.n_classes);
        return hipGetLastError();
    }
    const Plan plan = plan_backward(c);
    const Model<T> m = model_of<T>(c, plan, workspace, stream);
    if (const hipError_t e = hipGetLastError()) return e;
    T *p = reinterpret_cast<T *>(workspace + plan.p);
    float *bias_parts = grad_bias ? reinterpret_cast<float *>(workspace + plan.bias) : nullptr;
    float *hidden_parts = plan.hidden_parts < 0 ? nullptr : reinterpret_cast<float *>(workspace + plan.hidden_parts);
    float *weight_parts = plan.weight_parts < 0 ? nullptr : reinterpret_cast<float *>(workspace + plan.weight_parts);
    const int64_t step = STEP / sizeof(T), columns = ceil_div(c.dim, Gradient::N);
    for (int64_t piece = 0; piece < plan.pieces; ++piece) {
        const int64_t first = piece * plan.piece, classes = std::min(plan.piece, c.n_classes - first);
        const int64_t class_tiles = ceil_div(classes, Backward::N), stride = plan.piece;
        const int64_t p_tiles = class_tiles * plan.row_tiles;
        hipLaunchKernelGGL((p_kernel<T, Backward>), grid_of(p_tiles), dim3(Backward::THREADS), lds_bytes<Backward>(), stream, m, lse, grad_loss,
                           first, class_tiles, p_tiles, p, stride, bias_parts);
        if (grad_bias)
            hipLaunchKernelGGL(bias_kernel, dim3(static_cast<uint32_t>(ceil_div(classes, 256))), dim3(256), 0, stream, bias_parts,
                               plan.row_tiles, stride, classes, grad_bias + first);
        // grad_hidden [n_rows][dim] += p [n_rows][classes] weight [classes][dim]
        {
            const int64_t row_tiles = ceil_div(c.n_rows, Gradient::M), depth = round_up(ceil_div(classes, plan.hidden_splits), step);
            const Operand<T> a{p, stride, c.n_rows, classes}, b{m.weight.at + first * m.weight.stride, m.weight.stride, m.weight.depth, classes};
            const int64_t tiles = row_tiles * columns * plan.hidden_splits;
            hipLaunchKernelGGL((product_kernel<T, Gradient, true>), grid_of(tiles), dim3(Gradient::THREADS), lds_bytes<Gradient>(), stream, a, b,
                               c.dim, row_tiles, columns, depth, tiles, hidden_parts, piece > 0, hidden_parts ? nullptr : grad_hidden);
        }
        // grad_weight [classes][dim] = p^T [classes][n_rows] hidden [n_rows][dim]
        {
            const int64_t row_tiles = ceil_div(classes, Gradient::M), depth = round_up(ceil_div(c.n_rows, plan.weight_splits), step);
            const Operand<T> a{p, stride, classes, c.n_rows}, b{m.hidden.at, m.hidden.stride, m.hidden.depth, c.n_rows};
            const int64_t tiles = row_tiles * columns * plan.weight_splits;
            T *out = grad_weight + first * c.dim;
            hipLaunchKernelGGL((product_kernel<T, Gradient, false>), grid_of(tiles), dim3(Gradient::THREADS), lds_bytes<Gradient>(), stream, a, b,
                               c.dim, row_tiles, columns, depth, tiles, weight_parts, false, weight_parts ? nullptr : out);
            if (weight_parts)
                hipLaunchKernelGGL((parts_kernel<T>), grid_of(std::min<int64_t>(8192, ceil_div(classes * c.dim, 256))), dim3(256), 0, stream,
                                   weight_parts, plan.weight_splits, classes * c.dim, out);
        }
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (hidden_parts)
        hipLaunchKernelGGL((parts_kernel<T>), grid_of(std::min<int64_t>(8192, ceil_div(c.n_rows * c.dim, 256))), dim3(256), 0, stream, hidden_parts,
                           plan.hidden_splits, c.n_rows * c.dim, grad_hidden);
    return hipGetLastError();
}

}  // namespace

int64_t cross_entropy_bytes(const head_classes &c) { return c.n_rows ? plan_forward(c).bytes : 0; }

hipError_t launch_cross_entropy(const head_classes &c, float *loss, float *lse, void *workspace, hipStream_t stream)
{
    char *w = static_cast<char *>(workspace);
    return c.dtype == HEAD_BF16 ? forward<bf16>(c, loss, lse, w, stream) : forward<float>(c, loss, lse, w, stream);
}

int64_t cross_entropy_grad_bytes(const head_classes &c) { return c.n_rows ? plan_backward(c).bytes : 0; }

hipError_t launch_cross_entropy_grad(const head_classes &c, const float *lse, const float *grad_loss, void *grad_hidden,
                                     void *grad_weight, float *grad_bias, void *workspace, hipStream_t stream)
{
    char *w = static_cast<char *>(workspace);
    if (c.dtype == HEAD_BF16)
        return backward(c, lse, grad_loss, static_cast<bf16 *>(grad_hidden), static_cast<bf16 *>(grad_weight), grad_bias, w, stream);
    return backward(c, lse, grad_loss, static_cast<float *>(grad_hidden), static_cast<float *>(grad_weight), grad_bias, w, stream);
}

}  // namespace head_impl
