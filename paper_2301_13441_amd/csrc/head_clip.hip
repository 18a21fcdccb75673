// The 2-norm over many tensors and their clipping to a limit, on gfx950 (head.h).
//
//     norm = sqrt(sum of squares over all values of all tensors);  out = grad * min(1, max_norm / norm)
//
// Bound by memory: every value is read for the norm, and read and written once more where it is scaled.  Two launches for each TENSORS
// tensors, whose addresses go by value with the arguments; every workgroup leaves one number, and the second launch's workgroups add those
// numbers again, each for itself, in the same order.  Few values: one workgroup does both, in one launch.
//
// Squares of the 4 or 8 values that a lane reads at a time are added in float32, those sums in float64.  Sums that are not in the middle of
// float32's range are made again in float64.
// 131 MB of bfloat16: 22 us for the norm, 41 scaled (6.0 and 6.4 TB/s).  Results are
// stored past the caches, where they would be in the way of the next pass over the values (35 us for the norm).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "head_device.hpp"

namespace head_impl {
namespace {

constexpr int THREADS = 256;
constexpr int PIECES = 4;           // times 16 bytes of each lane in a block of a workgroup
constexpr int TENSORS = 64;         // tensors of a launch
constexpr int64_t MAX_GRID = 1024;  // workgroups that leave a number
constexpr int64_t MAX_CLIP_GRID = 2048;
constexpr int64_t MAX_PARTS = 4096; // numbers that every workgroup of the second launch adds; more are added by one workgroup before
constexpr int ALONE_THREADS = 1024;
constexpr int64_t ALONE = 160 << 10;  // bytes that one workgroup takes alone: of 30,000 values 7.4 us a call, against 9.4; of 60,000 10.5

// A block of values goes to a team of lanes: a workgroup, or (where one is alone) a wavefront, so that small tensors are read side by side.
constexpr int64_t block_bytes(int team) { return int64_t{team} * 16 * PIECES; }

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
    int32_t in_place;            // all of them
};

// The sum over a workgroup, in every lane.
template <int THREADS>
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

// f(tensor, a value, first value of the block) for every block of this team.
template <int TEAM, class F>
__device__ __forceinline__ void over_blocks(const Batch &b, F f)
{
    const int64_t blocks = b.first[b.count], teams = gridDim.x * (blockDim.x / TEAM);
    for (int64_t block = blockIdx.x * (blockDim.x / TEAM) + __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM); block < blocks; block += teams) {
        int t = 0, end = b.count;  // the last tensor that begins at the block or before
        while (end - t > 1) {
            const int mid = (t + end) / 2;
            if (b.first[mid] <= block) t = mid;
            else end = mid;
        }
        const Tensor &s = b.tensor[t];
        if (s.dtype == HEAD_BF16) f(s, bf16(), (block - b.first[t]) * (block_bytes(TEAM) / 2));
        else f(s, float(), (block - b.first[t]) * (block_bytes(TEAM) / 4));
    }
}

// Where a lane's piece j of a block begins.
template <class T, int TEAM>
__device__ __forceinline__ int64_t place(int64_t block, int j) { return block + (j * TEAM + static_cast<int>(threadIdx.x % TEAM)) * (16 / static_cast<int>(sizeof(T))); }

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

template <class T, int N>
__device__ __forceinline__ double squares(const Pack<T, N> &p)
{
    float s = 0;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = widen(p.v[i]);
        s = fmaf(x, x, s);
        any |= __float_as_uint(x) << 1;
    }
    if ((s >= 0x1p-90f && s < 0x1p120f) || any == 0) return s;
    double d = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const double x = widen(p.v[i]);
        d = fma(x, x, d);
    }
    return d;
}

template <int THREADS, int TEAM>
__device__ __forceinline__ double squares_of(const Batch &b)
{
    double sum = 0;
    over_blocks<TEAM>(b, [&](const Tensor &t, auto type, int64_t block) {
        using T = decltype(type);
        Pack<T, 16 / sizeof(T)> p[PIECES];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) p[j] = take(static_cast<const T *>(t.grad), place<T, TEAM>(block, j), t.n, t.wide);
#pragma unroll
        for (int j = 0; j < PIECES; ++j) sum += squares(p[j]);
    });
    return workgroup_sum<THREADS>(sum);
}

template <int TEAM>
__device__ __forceinline__ void scale_all(const Batch &b, double norm, double max_norm)
{
    const double share = max_norm >= norm || max_norm == INFINITY ? 1.0 : max_norm / norm;
    const bool same = static_cast<float>(share) == 1.0f;
    // A share that float32 holds with few bits or none, as of values near its end and a small limit, goes in two factors, the second a power of two.
    int down = 0;
    const float factor = static_cast<float>(share < 0x1p-100 ? frexp(share, &down) : share);
    if (same && b.in_place) return;
    over_blocks<TEAM>(b, [&](const Tensor &t, auto type, int64_t block) {
        using T = decltype(type);
        constexpr int V = 16 / sizeof(T);
        if (t.grad == t.out && same) return;
        Pack<T, V> p[PIECES];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) p[j] = take(static_cast<const T *>(t.grad), place<T, TEAM>(block, j), t.n, t.wide);
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int64_t at = place<T, TEAM>(block, j);
#pragma unroll
            for (int i = 0; i < V; ++i) p[j].v[i] = same ? p[j].v[i] : narrow<T>(ldexpf(widen(p[j].v[i]) * factor, down));
            T *to = static_cast<T *>(t.out);
            if (t.wide && at + V <= t.n) {
                store_past(to + at, p[j]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (at + i < t.n) to[at + i] = p[j].v[i];
            }
        }
    });
}

__global__ __launch_bounds__(THREADS) void squares_kernel(const Batch b, double *parts)
{
    const double sum = squares_of<THREADS, THREADS>(b);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__device__ __forceinline__ double sum_of(const double *parts, int64_t n)
{
    double s = 0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < n; i += THREADS) s += parts[i];
    return workgroup_sum<THREADS>(s);
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
    scale_all<THREADS>(b, norm, max_norm);
}

// Few values, by one workgroup; out may be null.
__global__ __launch_bounds__(ALONE_THREADS) void alone_kernel(const Batch b, int32_t scales, double max_norm, float *norm_out)
{
    const double norm = sqrt(squares_of<ALONE_THREADS, 64>(b));
    if (threadIdx.x == 0) *norm_out = static_cast<float>(norm);
    if (scales) scale_all<64>(b, norm, max_norm);
}

// launch(batch, workgroups) for all tensors that have values, TENSORS at a time, in blocks of that many bytes.
template <class Launch>
hipError_t in_batches(const head_clip_tensor *tensors, int32_t n_tensors, int64_t bytes, int64_t most, Launch launch)
{
    Batch b{};
    b.in_place = 1;
    for (int32_t i = 0; i <= n_tensors; ++i) {
        if (b.count == TENSORS || (i == n_tensors && b.count > 0)) {
            if (const hipError_t e = launch(b, std::min(b.first[b.count], most))) return e;
            b.count = 0;
            b.in_place = 1;
        }
        if (i == n_tensors) break;
        const head_clip_tensor &s = tensors[i];
        if (s.n == 0) continue;
        b.tensor[b.count] = Tensor{s.grad, s.out, s.n, s.dtype, (address(s.grad) | address(s.out)) % 16 == 0};
        b.first[b.count + 1] = b.first[b.count] + ceil_div(s.n * value_bytes(s.dtype), bytes);
        b.in_place &= s.grad == s.out;
        ++b.count;
    }
    return hipSuccess;
}

// Whether one workgroup takes all values.  Their types are not known where the workspace is asked for, so all count as float32.
bool is_alone(const head_clip_tensor *tensors, int32_t n_tensors)
{
    int64_t values = 0;
    int32_t some = 0;
    for (int32_t i = 0; i < n_tensors; ++i) values += tensors[i].n, some += tensors[i].n > 0;
    return some <= TENSORS && values <= ALONE / 4;
}

// Numbers that the first launches leave, at most.
int64_t parts_of(const head_clip_tensor *tensors, int32_t n_tensors)
{
    int64_t parts = 0;
    for (int32_t i = 0; i < n_tensors; ++i) parts += std::min(ceil_div(tensors[i].n * 4, block_bytes(THREADS)), MAX_GRID);
    return std::min(parts, (n_tensors / TENSORS + 1) * MAX_GRID);
}

}  // namespace

int64_t clip_bytes(const head_clip_tensor *tensors, int32_t n_tensors)
{
    return is_alone(tensors, n_tensors) ? 0 : round_up((parts_of(tensors, n_tensors) + 1) * 8, 16);
}

hipError_t launch_clip(const head_clip_tensor *tensors, int32_t n_tensors, double max_norm, float *norm, void *workspace, hipStream_t stream)
{
    bool wanted = false;
    for (int32_t i = 0; i < n_tensors && !wanted; ++i) wanted = tensors[i].n > 0 && tensors[i].out;
    if (is_alone(tensors, n_tensors)) {
        bool done = false;
        if (const hipError_t e = in_batches(tensors, n_tensors, block_bytes(64), 1, [&](const Batch &b, int64_t) {
                hipLaunchKernelGGL(alone_kernel, dim3(1), dim3(ALONE_THREADS), 0, stream, b, wanted, max_norm, norm);
                done = true;
                return hipGetLastError();
            }))
            return e;
        if (!done) hipLaunchKernelGGL(alone_kernel, dim3(1), dim3(ALONE_THREADS), 0, stream, Batch{}, 0, max_norm, norm);  // no values
        return hipGetLastError();
    }
    double *sum = static_cast<double *>(workspace), *parts = sum + 1;
    int64_t n_parts = 0;
    if (const hipError_t e = in_batches(tensors, n_tensors, block_bytes(THREADS), MAX_GRID, [&](const Batch &b, int64_t grid) {
            hipLaunchKernelGGL(squares_kernel, dim3(static_cast<uint32_t>(grid)), dim3(THREADS), 0, stream, b, parts + n_parts);
            n_parts += grid;
            return hipGetLastError();
        }))
        return e;
    if (n_parts > MAX_PARTS) {
        hipLaunchKernelGGL(join_kernel, dim3(1), dim3(THREADS), 0, stream, parts, n_parts, sum);
        parts = sum, n_parts = 1;
    }
    if (!wanted) {  // only the norm
        hipLaunchKernelGGL(clip_kernel, dim3(1), dim3(THREADS), 0, stream, Batch{}, parts, n_parts, max_norm, norm);
        return hipGetLastError();
    }
    float *once = norm;
    return in_batches(tensors, n_tensors, block_bytes(THREADS), MAX_CLIP_GRID, [&](const Batch &b, int64_t grid) {
        hipLaunchKernelGGL(clip_kernel, dim3(static_cast<uint32_t>(grid)), dim3(THREADS), 0, stream, b, parts, n_parts, max_norm, once);
        once = nullptr;
        return hipGetLastError();
    });
}

}  // namespace head_impl
