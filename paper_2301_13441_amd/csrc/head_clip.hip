// The 2-norm over many tensors and their clipping to a limit, on gfx950 (head.h).
//
//     norm = sqrt(sum of squares over all values of all tensors);  out = grad * min(1, max_norm / norm)
//
// Bound by memory: every value is read for the norm, and read and written once more where it is scaled.  Two launches for each TENSORS
// tensors, whose addresses go by value with the arguments; every workgroup adds its squares in float64 and leaves one number, and the
// second launch's workgroups add those numbers again, each for itself, in the same order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "head_device.hpp"

namespace head_impl {
namespace {

constexpr int THREADS = 256;
constexpr int BYTES = 16384;        // of a block: four times 16 bytes of each lane
constexpr int TENSORS = 64;         // tensors of a launch
constexpr int64_t MAX_GRID = 2048;  // workgroups of a launch
constexpr int64_t MAX_PARTS = 4096; // numbers that every workgroup of the second launch adds; more are added by one workgroup before

struct Tensor {
    const void *grad;
    void *out;
    int64_t n;
    int32_t dtype;
    int32_t wide;  // addresses are whole in 16 bytes
};
struct Batch {
    Tensor tensor[TENSORS];
    int64_t first[TENSORS + 1];  // first block of a tensor; the last entry: the number of blocks
    int32_t count;
};

// The sum over a workgroup, in every lane.
__device__ __forceinline__ double workgroup_sum(double s)
{
    __shared__ double lds[THREADS / 64];
#pragma unroll
    for (int d = 32; d > 0; d /= 2) s += __shfl_xor(s, d, 64);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = s;
    __syncthreads();
    s = lds[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) s += lds[w];
    return s;
}

// f(tensor, values type, first value, values that exist) for this lane's pieces of every block of this workgroup.
template <class F>
__device__ __forceinline__ void over_blocks(const Batch &b, F f)
{
    const int64_t blocks = b.first[b.count];
    for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        int t = 0, end = b.count;  // the last tensor that begins at the block or before
        while (end - t > 1) {
            const int mid = (t + end) / 2;
            if (b.first[mid] <= block) t = mid;
            else end = mid;
        }
        const Tensor &s = b.tensor[t];
        if (s.dtype == HEAD_BF16) f(s, bf16(), (block - b.first[t]) * (BYTES / 2));
        else f(s, float(), (block - b.first[t]) * (BYTES / 4));
    }
}

// A lane's values of a block that begins at `at`: PIECES times 16 bytes, a workgroup's side by side.
template <class T>
struct Piece {
    static constexpr int V = 16 / sizeof(T), PIECES = BYTES / 16 / THREADS;
    static __device__ __forceinline__ int64_t at(int64_t block, int j) { return block + (j * THREADS + static_cast<int>(threadIdx.x)) * V; }
};

template <class T>
__device__ __forceinline__ Pack<T, 16 / sizeof(T)> take(const T *from, int64_t at, int64_t n, bool wide)
{
    constexpr int V = 16 / sizeof(T);
    if (wide && at + V <= n) return *reinterpret_cast<const Pack<T, V> *>(from + at);
    Pack<T, V> p;
#pragma unroll
    for (int i = 0; i < V; ++i) p.v[i] = at + i < n ? from[at + i] : T(0);
    return p;
}

__global__ __launch_bounds__(THREADS) void squares_kernel(const Batch b, double *parts)
{
    double sum = 0;
    over_blocks(b, [&](const Tensor &t, auto type, int64_t block) {
        using T = decltype(type);
        using P = Piece<T>;
        Pack<T, P::V> p[P::PIECES];
#pragma unroll
        for (int j = 0; j < P::PIECES; ++j) p[j] = take(static_cast<const T *>(t.grad), P::at(block, j), t.n, t.wide);
#pragma unroll
        for (int j = 0; j < P::PIECES; ++j)
#pragma unroll
            for (int i = 0; i < P::V; ++i) {
                const double x = widen(p[j].v[i]);
                sum = fma(x, x, sum);
            }
    });
    sum = workgroup_sum(sum);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__device__ __forceinline__ double sum_of(const double *parts, int64_t n)
{
    double s = 0;
    for (int64_t i = threadIdx.x; i < n; i += THREADS) s += parts[i];
    return workgroup_sum(s);
}

__global__ __launch_bounds__(THREADS) void join_kernel(const double *parts, int64_t n, double *sum)
{
    const double s = sum_of(parts, n);
    if (threadIdx.x == 0) *sum = s;
}

__global__ __launch_bounds__(THREADS) void clip_kernel(const Batch b, const double *parts, int64_t n_parts, double max_norm, float *norm_out)
{
    const double norm = sqrt(sum_of(parts, n_parts));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = static_cast<float>(norm);
    const float factor = max_norm >= norm || max_norm == INFINITY ? 1.0f : static_cast<float>(max_norm / norm);
    over_blocks(b, [&](const Tensor &t, auto type, int64_t block) {
        using T = decltype(type);
        using P = Piece<T>;
        if (t.grad == t.out && factor == 1.0f) return;
        Pack<T, P::V> p[P::PIECES];
#pragma unroll
        for (int j = 0; j < P::PIECES; ++j) p[j] = take(static_cast<const T *>(t.grad), P::at(block, j), t.n, t.wide);
#pragma unroll
        for (int j = 0; j < P::PIECES; ++j) {
            const int64_t at = P::at(block, j);
#pragma unroll
            for (int i = 0; i < P::V; ++i) p[j].v[i] = factor == 1.0f ? p[j].v[i] : narrow<T>(widen(p[j].v[i]) * factor);
            T *to = static_cast<T *>(t.out);
            if (t.wide && at + P::V <= t.n) {
                *reinterpret_cast<Pack<T, P::V> *>(to + at) = p[j];
            } else {
#pragma unroll
                for (int i = 0; i < P::V; ++i)
                    if (at + i < t.n) to[at + i] = p[j].v[i];
            }
        }
    });
}

int64_t blocks_of(const head_clip_tensor &t) { return ceil_div(t.n * value_bytes(t.dtype), BYTES); }

// launch(batch, workgroups) for all tensors that have values, TENSORS at a time.
template <class Launch>
hipError_t in_batches(const head_clip_tensor *tensors, int32_t n_tensors, Launch launch)
{
    Batch b{};
    for (int32_t i = 0; i <= n_tensors; ++i) {
        if (b.count == TENSORS || (i == n_tensors && b.count > 0)) {
            if (const hipError_t e = launch(b, std::min(b.first[b.count], MAX_GRID))) return e;
            b.count = 0;
        }
        if (i == n_tensors) break;
        const head_clip_tensor &s = tensors[i];
        if (s.n == 0) continue;
        b.tensor[b.count] = Tensor{s.grad, s.out, s.n, s.dtype, (address(s.grad) | address(s.out)) % 16 == 0};
        b.first[b.count + 1] = b.first[b.count] + blocks_of(s);
        ++b.count;
    }
    return hipSuccess;
}

// Numbers that the first launches leave, at most: their types are not known where the workspace is asked for.
int64_t parts_of(const head_clip_tensor *tensors, int32_t n_tensors)
{
    int64_t parts = 0;
    for (int32_t i = 0; i < n_tensors; ++i) parts += std::min(ceil_div(tensors[i].n * 4, BYTES), MAX_GRID);
    return std::min(parts, (n_tensors / TENSORS + 1) * MAX_GRID);
}

}  // namespace

int64_t clip_bytes(const head_clip_tensor *tensors, int32_t n_tensors) { return round_up((parts_of(tensors, n_tensors) + 1) * 8, 16); }

hipError_t launch_clip(const head_clip_tensor *tensors, int32_t n_tensors, double max_norm, float *norm, void *workspace, hipStream_t stream)
{
    double *sum = static_cast<double *>(workspace), *parts = sum + 1;
    int64_t n_parts = 0;
    if (const hipError_t e = in_batches(tensors, n_tensors, [&](const Batch &b, int64_t grid) {
            hipLaunchKernelGGL(squares_kernel, dim3(static_cast<uint32_t>(grid)), dim3(THREADS), 0, stream, b, parts + n_parts);
            n_parts += grid;
            return hipGetLastError();
        }))
        return e;
    if (n_parts > MAX_PARTS) {
        hipLaunchKernelGGL(join_kernel, dim3(1), dim3(THREADS), 0, stream, parts, n_parts, sum);
        parts = sum, n_parts = 1;
    }
    bool wanted = false;
    for (int32_t i = 0; i < n_tensors && !wanted; ++i) wanted = tensors[i].n > 0 && tensors[i].out;
    if (!wanted) {  // no tensors, or only their norm
        hipLaunchKernelGGL(clip_kernel, dim3(1), dim3(THREADS), 0, stream, Batch{}, parts, n_parts, max_norm, norm);
        return hipGetLastError();
    }
    float *once = norm;
    return in_batches(tensors, n_tensors, [&](const Batch &b, int64_t grid) {
        hipLaunchKernelGGL(clip_kernel, dim3(static_cast<uint32_t>(grid)), dim3(THREADS), 0, stream, b, parts, n_parts, max_norm, once);
        once = nullptr;
        return hipGetLastError();
    });
}

}  // namespace head_impl
