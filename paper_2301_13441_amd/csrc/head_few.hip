// Dense layers of few rows, forward, on gfx950: single records and small batches of a trained head (formulas: head.h).
//
// Bound by reading the weights once, or by the chain of a launch, a load and a sum where they are few.  A workgroup has 16 columns of y
// (with a gated layer, both halves of z for them) and cuts the sum's axis over its wavefronts; a wavefront reads 16 rows of weights
// straight into the registers of the matrix instruction, 64 bytes of each at a time, several ahead, next to the same bytes of the batch's
// rows, 16 to an instruction.  The wavefronts' sums meet in LDS, in a fixed order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "head_layer.hpp"

namespace head_impl {
namespace {

using Sums = float __attribute__((ext_vector_type(4)));
using Bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using Chunk = float __attribute__((ext_vector_type(4)));  // 16 bytes of either type

constexpr int COLUMNS = FEW_COLUMNS;

__device__ __forceinline__ void multiply(Chunk a, Chunk b, Sums &c, bf16)
{
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<Bf16x8 *>(&a), *reinterpret_cast<Bf16x8 *>(&b), c, 0, 0, 0);
}
__device__ __forceinline__ void multiply(Chunk a, Chunk b, Sums &c, float)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
}

// 16 bytes from value k on, those past `dim` zero.  WIDE: all or none are, and they are aligned.
template <class T, bool WIDE>
__device__ __forceinline__ Chunk take(const T *row, int k, int dim)
{
    constexpr int V = 16 / sizeof(T);
    Chunk c = {};
    if constexpr (WIDE) {
        if (k < dim) c = *reinterpret_cast<const Chunk *>(row + k);
    } else {
        Pack<T, V> p;
#pragma unroll
        for (int j = 0; j < V; ++j) p.v[j] = k + j < dim ? row[k + j] : T(0);
        c = *reinterpret_cast<Chunk *>(&p);
    }
    return c;
}

// One row of 256 float32 values to 64: 3.3 us; 5 of 2048 bfloat16 values to 8192 gated ones, 67 MB of weights: 12.4 us (5.4 TB/s).
// parts (or null): where the sums over `each` steps from step `each` * blockIdx.y on go, [gridDim.y][n_rows][columns of z] float32.
template <class T, bool GATED, bool WIDE, int MT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(const T *x, int64_t x_stride, const T *weight, int64_t weight_stride, int dim, int each, End<T> e,
                                                         float *parts)
{
    constexpr int NT = GATED ? 2 : 1, V = 16 / sizeof(T), STEP = 4 * V, AHEAD = 4;
    __shared__ Sums lds[WAVES][NT][MT][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, in = lane % 16, quarter = lane / 16;
    const int64_t column0 = int64_t{COLUMNS} * blockIdx.x, column = std::min(column0 + in, e.outs - 1);
    // rows past the end are the last one again, of whose results nobody reads
    const T *w[NT], *b[MT];
#pragma unroll
    for (int h = 0; h < NT; ++h) w[h] = weight + (column + h * e.outs) * weight_stride;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) b[mt] = x + std::min<int64_t>(mt * 16 + in, e.n_rows - 1) * x_stride;
    Sums c[NT][MT] = {};
    // A wavefront's steps are WAVES apart.  Workgroups begin at different ones: rows may lie a power of two apart, and all would ask for the
    // same few of the memory's channels at the same time.
    const int steps = (dim + STEP - 1) / STEP, first = each * blockIdx.y + wave, last = std::min<int>(steps, each * (blockIdx.y + 1));
    const int own = last > first ? (last - first + WAVES - 1) / WAVES : 0;
    int at = own ? static_cast<int>(blockIdx.x % static_cast<uint32_t>(own)) : 0;
    auto some = [&](auto COUNT) {  // steps whose loads are on their way together
        Chunk p[COUNT()][NT], q[COUNT()][MT];
#pragma unroll
        for (int j = 0; j < COUNT(); ++j) {
            const int k = (first + at * WAVES) * STEP + quarter * V;
            at = at + 1 < own ? at + 1 : 0;
#pragma unroll
            for (int h = 0; h < NT; ++h) p[j][h] = take<T, WIDE>(w[h], k, dim);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) q[j][mt] = take<T, WIDE>(b[mt], k, dim);
        }
#pragma unroll
        for (int j = 0; j < COUNT(); ++j)
#pragma unroll
            for (int h = 0; h < NT; ++h)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) multiply(p[j][h], q[j][mt], c[h][mt], T());
    };
    int left = own;
    for (; left >= AHEAD; left -= AHEAD) some(std::integral_constant<int, AHEAD>());
    for (; left > 0; --left) some(std::integral_constant<int, 1>());
#pragma unroll
    for (int h = 0; h < NT; ++h)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) lds[wave][h][mt][lane] = c[h][mt];
    __syncthreads();
    // A lane for four adjacent columns of a row.
    for (int i = threadIdx.x; i < MT * 64; i += 64 * WAVES) {
        const int mt = i / 64, at = i % 64;
        const int64_t row = mt * 16 + at % 16, first = column0 + at / 16 * 4;
        Sums s[NT];
#pragma unroll
        for (int h = 0; h < NT; ++h) {
            s[h] = lds[0][h][mt][at];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) s[h] += lds[v][h][mt][at];
        }
        if (row >= e.n_rows) continue;
        if (parts) {
#pragma unroll
            for (int h = 0; h < NT; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (first + j < e.outs) parts[((blockIdx.y * e.n_rows + row) * NT + h) * e.outs + first + j] = s[h][j];
            continue;
        }
        with_activation(e.activation, [&](auto ACTIVATION) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t n = first + j;
                if (n >= e.outs) break;
                float z[NT];
#pragma unroll
                for (int h = 0; h < NT; ++h) {
                    z[h] = s[h][j] + (e.bias ? e.bias[h * e.outs + n] : 0.0f);
                    if (e.z) e.z[(row * NT + h) * e.outs + n] = narrow<T>(z[h]);
                }
                float v = Activation<T, ACTIVATION()>(z[0]).value;
                if constexpr (GATED) v *= z[1];
                else v = e.scale * v + (e.residual ? widen(e.residual[row * e.residual_stride + n]) : 0.0f);
                e.y[row * e.outs + n] = narrow<T>(v);
            }
        });
    }
}

}  // namespace

template <class T, bool GATED>
hipError_t launch_few(const head_layer &l, const End<T> &end, int64_t splits, float *parts, hipStream_t stream)
{
    constexpr int WAVES = 8;
    const int each = static_cast<int>(ceil_div(ceil_div(l.dim, 64 / static_cast<int64_t>(sizeof(T))), splits));
    auto run = [&](auto WIDE, auto MT) {
        hipLaunchKernelGGL((few_kernel<T, GATED, WIDE(), MT(), WAVES>), dim3(static_cast<uint32_t>(ceil_div(l.n_outputs, COLUMNS)), static_cast<uint32_t>(splits)),
                           dim3(64 * WAVES), 0, stream, static_cast<const T *>(l.x), l.x_stride, static_cast<const T *>(l.weight), l.weight_stride,
                           static_cast<int>(l.dim), each, end, splits > 1 ? parts : nullptr);
        return hipGetLastError();
    };
    auto rows = [&](auto WIDE) {
        using std::integral_constant;
        return l.n_rows <= 16 ? run(WIDE, integral_constant<int, 1>()) : l.n_rows <= 32 ? run(WIDE, integral_constant<int, 2>()) : run(WIDE, integral_constant<int, 4>());
    };
    return few_wide(l) ? rows(std::true_type()) : rows(std::false_type());
}

template hipError_t launch_few<float, false>(const head_layer &, const End<float> &, int64_t, float *, hipStream_t);
template hipError_t launch_few<float, true>(const head_layer &, const End<float> &, int64_t, float *, hipStream_t);
template hipError_t launch_few<bf16, false>(const head_layer &, const End<bf16> &, int64_t, float *, hipStream_t);
template hipError_t launch_few<bf16, true>(const head_layer &, const End<bf16> &, int64_t, float *, hipStream_t);

}  // namespace head_impl
