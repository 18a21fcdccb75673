// Layer norm on gfx950, forward and backward.
//
//     y = (x - mean) * rstd * w + b
//     dx = rstd * (g w - mean(g w) - unit * mean(g w unit)),  unit = (x - mean) * rstd
//     dw = sum over rows of g unit,  db = sum over rows of g
//
// Bound by memory: x is read and y written once forward, g and x are read and dx written once backward.  A row is held in
// the registers of a team of LANES lanes (a part of a wavefront, or a whole workgroup for long rows), so that the
// variance is taken from the differences to the mean, as its definition has it, without a second read.  Backward, a team goes
// from row to row and keeps its columns' sums of dw and db in registers; the teams' sums meet in LDS and go to the workspace,
// a row for each workgroup, and a second kernel adds those, so no atomics are needed and the order of the sums is fixed.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "head_device.hpp"

namespace head_impl {
namespace {

constexpr int THREADS = 256;
constexpr int MAX_GRID = 1 << 22;       // workgroups of the forward pass: 2^30 threads, a grid's axis has room for 2^32
constexpr int MAX_WORKGROUPS = 1024;  // of the backward pass: rows of its workspace

template <int LANES>
__device__ __forceinline__ float team_sum(float v, float *lds)
{
    if constexpr (LANES <= 64) {
#pragma unroll
        for (int d = LANES / 2; d > 0; d /= 2) v += __shfl_xor(v, d, LANES);
        return v;
    } else {
#pragma unroll
        for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d, 64);
        __syncthreads();  // who still reads the last sum
        if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
        __syncthreads();
        float s = 0;
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) s += lds[i];
        return s;
    }
}

// Column of value 0 of a lane's i-th piece.
template <int V, int LANES>
__device__ __forceinline__ int column(int i)
{
    return (i * LANES + static_cast<int>(threadIdx.x % LANES)) * V;
}

template <class T, int V, int LANES, int N>
__global__ __launch_bounds__(THREADS) void norm_kernel(int64_t n_rows, int dim, const T *x, int64_t x_stride, const float *weight,
                                                       const float *bias, float eps, T *y, float *mean, float *rstd)
{
    __shared__ float lds[THREADS / 64];
    constexpr int TEAMS = THREADS / LANES;
    const int64_t step = static_cast<int64_t>(gridDim.x) * TEAMS;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * TEAMS; first < n_rows; first += step) {
        const int64_t row = first + threadIdx.x / LANES;
        const bool here = row < n_rows;
        const T *from = x + (here ? row : 0) * x_stride;
        float a[N][V];
        float sum = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = column<V, LANES>(i);
            Pack<T, V> p{};
            if (c < dim) p = *reinterpret_cast<const Pack<T, V> *>(from + c);
#pragma unroll
            for (int k = 0; k < V; ++k) sum += a[i][k] = widen(p.v[k]);
        }
        const float m = team_sum<LANES>(sum, lds) / dim;
        float squares = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (column<V, LANES>(i) < dim)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    a[i][k] -= m;
                    squares = fmaf(a[i][k], a[i][k], squares);
                }
        const float r = 1.0f / sqrtf(team_sum<LANES>(squares, lds) / dim + eps);
        if (!here) continue;
        T *to = y + row * dim;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = column<V, LANES>(i);
            if (c < dim) {
                Pack<T, V> p;
#pragma unroll
                for (int k = 0; k < V; ++k) p.v[k] = narrow<T>(fmaf(a[i][k] * r, weight[c + k], bias ? bias[c + k] : 0.0f));
                *reinterpret_cast<Pack<T, V> *>(to + c) = p;
            }
        }
        if (threadIdx.x % LANES == 0) {
            mean[row] = m;
            rstd[row] = r;
        }
    }
}

template <class T, int V, int LANES, int N>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(int64_t n_rows, int dim, const T *grad, int64_t grad_stride, const T *x,
                                                            int64_t x_stride, const float *weight, const float *mean,
                                                            const float *rstd, T *grad_x, float *parts)
{
    __shared__ float lds[THREADS / 64];
    constexpr int TEAMS = THREADS / LANES;
    extern __shared__ float columns[];  // [2][dim], where there are several teams
    float dw[N][V] = {}, db[N][V] = {}, w[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int c = column<V, LANES>(i);
            w[i][k] = c < dim ? weight[c + k] : 0.0f;
        }
    // Every team makes the same number of rounds: the sums of a whole workgroup meet in barriers.
    const int64_t step = static_cast<int64_t>(gridDim.x) * TEAMS;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * TEAMS; first < n_rows; first += step) {
        const int64_t row = first + threadIdx.x / LANES;
        const bool here = row < n_rows;
        const float m = here ? mean[row] : 0.0f, r = here ? rstd[row] : 0.0f;
        float g[N][V], u[N][V], along = 0, across = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = column<V, LANES>(i);
            const bool in = here && c < dim;
            Pack<T, V> pg{}, px{};
            if (in) {
                pg = *reinterpret_cast<const Pack<T, V> *>(grad + row * grad_stride + c);
                px = *reinterpret_cast<const Pack<T, V> *>(x + row * x_stride + c);
            }
#pragma unroll
            for (int k = 0; k < V; ++k) {
                g[i][k] = widen(pg.v[k]);
                u[i][k] = in ? (widen(px.v[k]) - m) * r : 0.0f;
                dw[i][k] = fmaf(g[i][k], u[i][k], dw[i][k]);
                db[i][k] += g[i][k];
                g[i][k] *= w[i][k];
                along += g[i][k];
                across = fmaf(g[i][k], u[i][k], across);
            }
        }
        along = team_sum<LANES>(along, lds) / dim;
        across = team_sum<LANES>(across, lds) / dim;
        if (here)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = column<V, LANES>(i);
                if (c < dim) {
                    Pack<T, V> p;
#pragma unroll
                    for (int k = 0; k < V; ++k) p.v[k] = narrow<T>(r * (g[i][k] - along - u[i][k] * across));
                    *reinterpret_cast<Pack<T, V> *>(grad_x + row * dim + c) = p;
                }
            }
    }
    float *part = parts + static_cast<int64_t>(blockIdx.x) * 2 * dim;
    // The teams add their sums one after the other.
    for (int team = 0; team < TEAMS; ++team) {
        if (static_cast<int>(threadIdx.x) / LANES == team)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = column<V, LANES>(i);
                if (c < dim)
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        float a = dw[i][k], b = db[i][k];
                        if (team > 0) {
                            a += columns[c + k];
                            b += columns[dim + c + k];
                        }
                        if (team + 1 < TEAMS) {
                            columns[c + k] = a;
                            columns[dim + c + k] = b;
                        } else {
                            part[c + k] = a;
                            part[dim + c + k] = b;
                        }
                    }
            }
        if (TEAMS > 1) __syncthreads();
    }
}

// The columns' sums over the workgroups: 16 columns at a time, 16 lanes on each.
__global__ __launch_bounds__(THREADS) void norm_columns_kernel(int n_parts, int dim, const float *parts, float *grad_weight,
                                                               float *grad_bias)
{
    __shared__ float lds[16][17];
    const int c = blockIdx.x * 16 + threadIdx.x % 16, lane = threadIdx.x / 16;
    float s = 0;
    if (c < 2 * dim)
        for (int p = lane; p < n_parts; p += 16) s += parts[static_cast<int64_t>(p) * 2 * dim + c];
    lds[lane][threadIdx.x % 16] = s;
    __syncthreads();
    if (lane == 0 && c < 2 * dim) {
        float all = 0;
        for (int p = 0; p < 16; ++p) all += lds[p][threadIdx.x];
        (c < dim ? grad_weight : grad_bias)[c < dim ? c : c - dim] = all;
    }
}

// Calls f(values in a piece, lanes of a team, pieces of a lane) with constants that hold `dim` values of T.
template <class T, class F>
hipError_t by_shape(int wide, int64_t dim, F f)
{
    auto with = [&](auto V) {
        const int64_t n = ceil_div(dim, V());
        using std::integral_constant;
#define HEAD_TEAM(LANES, N) f(V, integral_constant<int, LANES>(), integral_constant<int, N>())
        if (n <= 4) return HEAD_TEAM(4, 1);
        if (n <= 8) return HEAD_TEAM(8, 1);
        if (n <= 16) return HEAD_TEAM(16, 1);
        if (n <= 32) return HEAD_TEAM(32, 1);
        if (n <= 64) return HEAD_TEAM(64, 1);
        if (n <= 128) return HEAD_TEAM(64, 2);
        if (n <= 256) return HEAD_TEAM(64, 4);
        if (n <= 512) return HEAD_TEAM(256, 2);
        if (n <= 1024) return HEAD_TEAM(256, 4);
        if (n <= 2048) return HEAD_TEAM(256, 8);
        if constexpr (V() <= 4) if (n <= 4096) return HEAD_TEAM(256, 16);
        if constexpr (V() <= 2) if (n <= 8192) return HEAD_TEAM(256, 32);
        if constexpr (V() <= 1) if (n <= 16384) return HEAD_TEAM(256, 64);
#undef HEAD_TEAM
        return hipErrorInvalidValue;
    };
    static_assert(HEAD_MAX_DIM <= 16384, "the longest row that a team holds");
    switch (wide) {
        case 1: return with(std::integral_constant<int, 1>());
        case 2: return with(std::integral_constant<int, 2>());
        case 4: return with(std::integral_constant<int, 4>());
        default:
            if constexpr (sizeof(T) == 2) return with(std::integral_constant<int, 8>());
            return hipErrorInvalidValue;
    }
}

template <class T>
hipError_t norm(int64_t n_rows, int64_t dim, const T *x, int64_t x_stride, const float *weight, const float *bias, float eps, T *y,
                float *mean, float *rstd, hipStream_t stream)
{
    const uint64_t bits = address(x) | address(y) | static_cast<uint64_t>(x_stride * sizeof(T)) | static_cast<uint64_t>(dim * sizeof(T));
    return by_shape<T>(piece(bits, sizeof(T)), dim, [&](auto V, auto LANES, auto N) {
        const int64_t teams = THREADS / LANES();
        hipLaunchKernelGGL((norm_kernel<T, V(), LANES(), N()>), dim3(static_cast<uint32_t>(std::min<int64_t>(ceil_div(n_rows, teams), MAX_GRID))), dim3(THREADS), 0,
                           stream, n_rows, static_cast<int>(dim), x, x_stride, weight, bias, eps, y, mean, rstd);
        return hipGetLastError();
    });
}

int64_t grad_workgroups(int64_t n_rows) { return std::max<int64_t>(1, std::min<int64_t>(n_rows, MAX_WORKGROUPS)); }

template <class T>
hipError_t norm_grad(int64_t n_rows, int64_t dim, const T *grad, int64_t grad_stride, const T *x, int64_t x_stride,
                     const float *weight, const float *mean, const float *rstd, T *grad_x, float *parts, int64_t &n_parts,
                     hipStream_t stream)
{
    const uint64_t bits = address(grad) | address(x) | address(grad_x) | static_cast<uint64_t>(x_stride * sizeof(T)) |
                          static_cast<uint64_t>(grad_stride * sizeof(T)) | static_cast<uint64_t>(dim * sizeof(T));
    return by_shape<T>(piece(bits, sizeof(T)), dim, [&](auto V, auto LANES, auto N) {
        const int64_t teams = THREADS / LANES();
        n_parts = grad_workgroups(ceil_div(n_rows, teams));
        const size_t bytes = teams > 1 ? static_cast<size_t>(2 * dim) * sizeof(float) : 0;
        hipLaunchKernelGGL((norm_grad_kernel<T, V(), LANES(), N()>), dim3(static_cast<uint32_t>(n_parts)), dim3(THREADS), bytes, stream,
                           n_rows, static_cast<int>(dim), grad, grad_stride, x, x_stride, weight, mean, rstd, grad_x, parts);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_layer_norm(int32_t dtype, int64_t n_rows, int64_t dim, const void *x, int64_t x_stride, const float *weight,
                             const float *bias, float eps, void *y, float *mean, float *rstd, hipStream_t stream)
{
    if (dtype == HEAD_BF16)
        return norm(n_rows, dim, static_cast<const bf16 *>(x), x_stride, weight, bias, eps, static_cast<bf16 *>(y), mean, rstd, stream);
    return norm(n_rows, dim, static_cast<const float *>(x), x_stride, weight, bias, eps, static_cast<float *>(y), mean, rstd, stream);
}

int64_t layer_norm_grad_bytes(int32_t, int64_t n_rows, int64_t dim)
{
    return round_up(grad_workgroups(n_rows) * 2 * dim * static_cast<int64_t>(sizeof(float)), 16);
}

hipError_t launch_layer_norm_grad(int32_t dtype, int64_t n_rows, int64_t dim, const void *grad, int64_t grad_stride, const void *x,
                                  int64_t x_stride, const float *weight, const float *mean, const float *rstd, void *grad_x,
                                  float *grad_weight, float *grad_bias, void *workspace, hipStream_t stream)
{
    float *parts = static_cast<float *>(workspace);
    int64_t n_parts = 0;  // no rows: the sums are zero
    if (n_rows > 0) {
        const hipError_t e =
            dtype == HEAD_BF16
                ? norm_grad(n_rows, dim, static_cast<const bf16 *>(grad), grad_stride, static_cast<const bf16 *>(x), x_stride, weight,
                            mean, rstd, static_cast<bf16 *>(grad_x), parts, n_parts, stream)
                : norm_grad(n_rows, dim, static_cast<const float *>(grad), grad_stride, static_cast<const float *>(x), x_stride, weight,
                            mean, rstd, static_cast<float *>(grad_x), parts, n_parts, stream);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(norm_columns_kernel, dim3(static_cast<uint32_t>(ceil_div(2 * dim, 16))), dim3(THREADS), 0, stream,
                       static_cast<int>(n_parts), static_cast<int>(dim), parts, grad_weight, grad_bias);
    return hipGetLastError();
}

}  // namespace head_impl
