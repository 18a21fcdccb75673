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
// A y of so many bytes is no more in the 32 MB of the L2s when it is read: its stores are non-temporal (515,345 x 90 float32: 89 us, 4.2 TB/s,
// against 107).  The backward pass, which reads twice what it writes, gains nothing (295 us, against 296).
constexpr int64_t PAST_BYTES = int64_t{64} << 20;
constexpr int MAX_WORKGROUPS = 768;   // of the backward pass, three for each of 256 CUs: rows of its workspace

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

// A team takes ROWS rows at once where a lane has few values of each: their loads are on their way together.  515,345 rows of 90 float32: 89
// us, 4.2 TB/s; one row at a time 195, eight 118 (both with ordinary stores, as 107).
template <class T, int V, int LANES, int N, int ROWS, bool PAST>
__global__ __launch_bounds__(THREADS) void norm_kernel(int64_t n_rows, int dim, const T *x, int64_t x_stride, const float *weight,
                                                       const float *bias, float eps, T *y, float *mean, float *rstd)
{
    __shared__ float lds[THREADS / 64];
    constexpr int TEAMS = THREADS / LANES;
    const int64_t step = static_cast<int64_t>(gridDim.x) * TEAMS * ROWS;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * TEAMS * ROWS; first < n_rows; first += step) {
        const int64_t row0 = first + threadIdx.x / LANES;  // and every TEAMS rows from there
        float a[ROWS][N][V], m[ROWS], r[ROWS];
        Pack<T, V> p[ROWS][N];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const T *from = x + std::min(row0 + k * TEAMS, n_rows - 1) * x_stride;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = column<V, LANES>(i);
                p[k][i] = *reinterpret_cast<const Pack<T, V> *>(from + (c < dim ? c : 0));
            }
        }
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            float sum = 0;
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) sum += a[k][i][j] = column<V, LANES>(i) < dim ? widen(p[k][i].v[j]) : 0.0f;
            m[k] = team_sum<LANES>(sum, lds) / dim;
        }
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            float squares = 0;
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    a[k][i][j] -= m[k];
                    squares = column<V, LANES>(i) < dim ? fmaf(a[k][i][j], a[k][i][j], squares) : squares;
                }
            r[k] = 1.0f / sqrtf(team_sum<LANES>(squares, lds) / dim + eps);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = column<V, LANES>(i);
            if (c < dim) {
                float w[V], b[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    w[j] = weight[c + j];
                    b[j] = bias ? bias[c + j] : 0.0f;
                }
#pragma unroll
                for (int k = 0; k < ROWS; ++k) {
                    Pack<T, V> o;
#pragma unroll
                    for (int j = 0; j < V; ++j) o.v[j] = narrow<T>(fmaf(a[k][i][j] * r[k], w[j], b[j]));
                    const int64_t row = row0 + k * TEAMS;
                    if (row >= n_rows) continue;
                    if constexpr (PAST) store_past(y + row * dim + c, o);
                    else *reinterpret_cast<Pack<T, V> *>(y + row * dim + c) = o;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int64_t row = row0 + k * TEAMS;
            if (threadIdx.x % LANES == 0 && row < n_rows) {
                mean[row] = m[k];
                rstd[row] = r[k];
            }
        }
    }
}

// 262,147 rows of 1024 bfloat16: 302 us, 5.3 TB/s; two rows at a time, of 16 values a lane, 323.
template <class T, int V, int LANES, int N, int ROWS>
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
        for (int j = 0; j < V; ++j) {
            const int c = column<V, LANES>(i);
            w[i][j] = c < dim ? weight[c + j] : 0.0f;
        }
    // Every team makes the same number of rounds: the sums of a whole workgroup meet in barriers.
    const int64_t step = static_cast<int64_t>(gridDim.x) * TEAMS * ROWS;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * TEAMS * ROWS; first < n_rows; first += step) {
        const int64_t row0 = first + threadIdx.x / LANES;  // and every TEAMS rows from there
        Pack<T, V> pg[ROWS][N], px[ROWS][N];
        float m[ROWS], r[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int64_t row = row0 + k * TEAMS;
            const bool here = row < n_rows;
            m[k] = here ? mean[row] : 0.0f;
            r[k] = here ? rstd[row] : 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = column<V, LANES>(i);
                pg[k][i] = px[k][i] = Pack<T, V>{};  // nothing is added where g is 0
                if (here && c < dim) {
                    pg[k][i] = *reinterpret_cast<const Pack<T, V> *>(grad + row * grad_stride + c);
                    px[k][i] = *reinterpret_cast<const Pack<T, V> *>(x + row * x_stride + c);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int64_t row = row0 + k * TEAMS;
            float g[N][V], u[N][V], along = 0, across = 0;
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    g[i][j] = widen(pg[k][i].v[j]);
                    u[i][j] = (widen(px[k][i].v[j]) - m[k]) * r[k];
                    dw[i][j] = fmaf(g[i][j], u[i][j], dw[i][j]);
                    db[i][j] += g[i][j];
                    g[i][j] *= w[i][j];
                    along += g[i][j];
                    across = fmaf(g[i][j], u[i][j], across);
                }
            along = team_sum<LANES>(along, lds) / dim;
            across = team_sum<LANES>(across, lds) / dim;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = column<V, LANES>(i);
                Pack<T, V> o;
#pragma unroll
                for (int j = 0; j < V; ++j) o.v[j] = narrow<T>(r[k] * (g[i][j] - along - u[i][j] * across));
                if (row < n_rows && c < dim) *reinterpret_cast<Pack<T, V> *>(grad_x + row * dim + c) = o;
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
                    for (int j = 0; j < V; ++j) {
                        float a = dw[i][j], b = db[i][j];
                        if (team > 0) {
                            a += columns[c + j];
                            b += columns[dim + c + j];
                        }
                        if (team + 1 < TEAMS) {
                            columns[c + j] = a;
                            columns[dim + c + j] = b;
                        } else {
                            part[c + j] = a;
                            part[dim + c + j] = b;
                        }
                    }
            }
        if (TEAMS > 1) __syncthreads();
    }
}

// The columns' sums over the workgroups: 16 columns at a time, 64 lanes on each.
__global__ __launch_bounds__(1024) void norm_columns_kernel(int n_parts, int dim, const float *parts, float *grad_weight, float *grad_bias)
{
    __shared__ float lds[64][17];
    const int c = blockIdx.x * 16 + threadIdx.x % 16, lane = threadIdx.x / 16;
    float s = 0;
    if (c < 2 * dim) {
#pragma unroll 8
        for (int p = lane; p < n_parts; p += 64) s += parts[static_cast<int64_t>(p) * 2 * dim + c];
    }
    lds[lane][threadIdx.x % 16] = s;
    __syncthreads();
    if (lane == 0 && c < 2 * dim) {
        float all = 0;
#pragma unroll
        for (int p = 0; p < 64; ++p) all += lds[p][threadIdx.x];
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
        constexpr int ROWS = V() * N() <= 8 ? 4 : V() * N() <= 16 ? 2 : 1;
        const int64_t rows = THREADS / LANES() * ROWS;
        // two kernels: of a branch between the two kinds of store the compiler makes one of the ordinary kind
        auto *kernel = n_rows * dim * static_cast<int64_t>(sizeof(T)) >= PAST_BYTES ? norm_kernel<T, V(), LANES(), N(), ROWS, true>
                                                                                     : norm_kernel<T, V(), LANES(), N(), ROWS, false>;
        hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(std::min<int64_t>(ceil_div(n_rows, rows), MAX_GRID))), dim3(THREADS), 0, stream,
                           n_rows, static_cast<int>(dim), x, x_stride, weight, bias, eps, y, mean, rstd);
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
        constexpr int ROWS = V() * N() <= 4 ? 4 : V() * N() <= 8 ? 2 : 1;
        n_parts = grad_workgroups(ceil_div(n_rows, teams * ROWS));
        const size_t bytes = teams > 1 ? static_cast<size_t>(2 * dim) * sizeof(float) : 0;
        hipLaunchKernelGGL((norm_grad_kernel<T, V(), LANES(), N(), ROWS>), dim3(static_cast<uint32_t>(n_parts)), dim3(THREADS), bytes, stream,
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
    hipLaunchKernelGGL(norm_columns_kernel, dim3(static_cast<uint32_t>(ceil_div(2 * dim, 16))), dim3(1024), 0, stream,
                       static_cast<int>(n_parts), static_cast<int>(dim), parts, grad_weight, grad_bias);
    return hipGetLastError();
}

}  // namespace head_impl
