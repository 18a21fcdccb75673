// One AdamW step over many tensors, on gfx950 (the formulas and the 8-bit states: head.h).
//
// Bound by memory: 28 bytes a value with float32 gradients and states, 14 with bfloat16 gradients and states in 8 bits, 2 more for a copy.
// 16.4 million values, float32: 69 us, 6.6 TB/s; 65.6 million, 8 bits and a copy: 201 us, 5.2 TB/s.
// A launch takes up to TENSORS tensors, whose addresses go by value with its arguments: there is no table on the
// device to keep, and a captured launch carries its own.  A workgroup finds its tensor by the number of its block, the
// tensors' blocks being counted through.  A lane takes 8 adjacent values, so that 16 lanes hold the HEAD_BLOCK = 128 values
// of an 8-bit scale and their largest magnitude is four exchanges away.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "head_device.hpp"

namespace head_impl {
namespace {

constexpr int THREADS = 256;
constexpr int EACH = 8;                   // values of a lane
constexpr int VALUES_EACH = 8;            // of adamw_values_kernel
constexpr int TENSORS = 40;               // tensors of a launch
constexpr int64_t MAX_GRID = 8192;        // workgroups of a step, several for each CU: each makes its table once
constexpr int64_t MAX_VALUES_GRID = 65536;  // of adamw_values_kernel, which has none
static_assert(HEAD_BLOCK == 16 * EACH, "a scale's values are those of 16 lanes");

struct Tensor {
    float *param;
    const void *grad;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    bf16 *copy;
    int64_t n;
    uint32_t key;      // of the random numbers
    int32_t wide;      // all addresses are whole in pieces of EACH values, or 16 bytes
};
struct Batch {
    Tensor tensor[TENSORS];
    int64_t first[TENSORS + 1];  // first block of a tensor; the last entry: the number of blocks
    int32_t count;
};
struct Numbers {
    float beta1, rest1, beta2, rest2, decay, rate, root, eps;  // rest: 1 - beta; decay: times the rate; rate, root: with the corrections
};

// Multiplications and xor-shifts after which every bit depends on every other; the constants are those that C. Wellons published in 2018,
// found by a search for the least bias.
__host__ __device__ inline uint32_t hash(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}

template <class T, int N = EACH>
struct alignas(16) Values {
    T v[N];
};

// What the e4m3 codes of a lane stand for, times 2^(s - 134).
template <int N>
__device__ __forceinline__ void decode(const Values<uint8_t, N> &code, int s, float (&x)[N])
{
#pragma unroll
    for (int w = 0; w < N / 4; ++w) {
        const uint32_t four = reinterpret_cast<const uint32_t *>(code.v)[w];
        x[4 * w] = __builtin_amdgcn_cvt_f32_fp8(four, 0);
        x[4 * w + 1] = __builtin_amdgcn_cvt_f32_fp8(four, 1);
        x[4 * w + 2] = __builtin_amdgcn_cvt_f32_fp8(four, 2);
        x[4 * w + 3] = __builtin_amdgcn_cvt_f32_fp8(four, 3);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = ldexpf(x[i], s - 134);
}

// Scale byte of a block whose largest finite magnitude is `most`: its exponent + 127, at least 7, for 2^(134 - 7) is the largest power
// of two in float32; 0 for a block of zeros.
__device__ __forceinline__ int scale_of(float most)
{
    if (!(most > 0)) return 0;
    return max(7, static_cast<int>(__float_as_uint(most) >> 23));
}

// 2^(134 - s), by which a block of scale s is multiplied before it is coded.  By powf, which misses some powers by one rounding
// (2^16 among them): that is how torch.ldexp takes them here, and a step written in torch then gives the same codes of values other than
// zero as this kernel, where ldexpf would give about one of a million another one.  powf is long: a workgroup makes a table of them.
__device__ __forceinline__ float factor_of(int s) { return powf(2.0f, static_cast<float>(134 - s)); }

// The code of x in a block whose factor that is, rounded up where the rest plus `random` (16 bits, as a fraction) reaches one.
// Of a number of the format's normal range the code is its bits' upper ones, and the random number is added to the 20 bits below
// them; below 2^-6 steps are 2^-9 wide.
__device__ __forceinline__ uint32_t encode(float x, float factor, uint32_t random, bool keep)
{
    const float y = fabsf(x) * factor;  // below 256
    const uint32_t normal = ((__float_as_uint(y) + (random << 4)) >> 20) - ((127 - 7) << 3);
    const uint32_t below = static_cast<uint32_t>(fmaf(y, 0x1p25f, static_cast<float>(random))) >> 16;
    uint32_t code = y < 0x1p-6f ? below : normal;
    if (keep && x > 0) code = max(code, 1u);
    if (x < 0) code |= 128;
    return fabsf(x) < INFINITY ? code : 127;
}

// N adjacent values, `some` of which exist; `wide`: all do, and their address is whole in 16 bytes or their own length.
//
// Stores are non-temporal: a step goes once over more than any cache holds (65.6 million values with 8-bit states: 193 to 202 us, against 245;
// what these stand for: 70, against 97).  Loads are not: 212 us, and float32 states 87 against 71.
template <class T, int N>
__device__ __forceinline__ void take(Values<T, N> &to, const T *from, int some, bool wide)
{
    constexpr int P = sizeof(T) * N > 16 ? 16 / sizeof(T) : N;
    if (wide) {
#pragma unroll
        for (int i = 0; i < N; i += P) *reinterpret_cast<Pack<T, P> *>(to.v + i) = *reinterpret_cast<const Pack<T, P> *>(from + i);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) to.v[i] = i < some ? from[i] : T(0);
}
template <class T, int N>
__device__ __forceinline__ void put(T *to, const Values<T, N> &from, int some, bool wide)
{
    constexpr int P = sizeof(T) * N > 16 ? 16 / sizeof(T) : N;
    if (wide) {
#pragma unroll
        for (int i = 0; i < N; i += P) store_past(to + i, *reinterpret_cast<const Pack<T, P> *>(from.v + i));
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < some) to[i] = from.v[i];
}

// Largest finite magnitude of the 16 lanes of a block.
__device__ __forceinline__ float block_most(const float (&x)[EACH])
{
    float most = 0;  // a maximum leaves out NaN
#pragma unroll
    for (int i = 0; i < EACH; ++i) most = fmaxf(most, fabsf(x[i]));
    if (!(most < INFINITY)) {
        most = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) most = fmaxf(most, fabsf(x[i]) < INFINITY ? fabsf(x[i]) : 0.0f);
    }
#pragma unroll
    for (int d = 8; d > 0; d /= 2) most = fmaxf(most, __shfl_xor(most, d, 16));
    return most;
}

// The tensor of a block, and a lane's first value in it.
template <int N>
__device__ __forceinline__ int find(const Batch &b, int64_t block, int64_t &at)
{
    int t = 0, end = b.count;  // the last tensor that begins at the block or before
    while (end - t > 1) {
        const int mid = (t + end) / 2;
        if (b.first[mid] <= block) t = mid;
        else end = mid;
    }
    at = (block - b.first[t]) * (THREADS * N) + static_cast<int64_t>(threadIdx.x) * N;
    return t;
}

template <class G, bool EIGHT>
__global__ __launch_bounds__(THREADS) void adamw_kernel(const Batch b, const Numbers c)
{
    __shared__ float factor[256];
    if constexpr (EIGHT) {
        factor[threadIdx.x] = threadIdx.x >= 7 ? factor_of(threadIdx.x) : 0.0f;  // a block of zeros has scale 0
        __syncthreads();
    }
    const int64_t blocks = b.first[b.count];
    for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        int64_t at;
        const Tensor &t = b.tensor[find<EACH>(b, block, at)];
        const int some = static_cast<int>(std::max<int64_t>(0, std::min<int64_t>(EACH, t.n - at)));
        const bool wide = some == EACH && t.wide;
        if (!EIGHT && some == 0) continue;
        Values<float> p, m, v;
        Values<G> g;
        Values<uint8_t> mc, vc;
        take(p, t.param + at, some, wide);
        take(g, static_cast<const G *>(t.grad) + at, some, wide);
        if constexpr (EIGHT) {
            take(mc, static_cast<const uint8_t *>(t.m) + at, some, wide);
            take(vc, static_cast<const uint8_t *>(t.v) + at, some, wide);
            const int ms = some ? t.m_scale[at / HEAD_BLOCK] : 0, vs = some ? t.v_scale[at / HEAD_BLOCK] : 0;
            decode(mc, ms, m.v);
            decode(vc, vs, v.v);
#pragma unroll
            for (int i = 0; i < EACH; ++i) v.v[i] *= v.v[i];
        } else {
            take(m, static_cast<const float *>(t.m) + at, some, wide);
            take(v, static_cast<const float *>(t.v) + at, some, wide);
        }
        Values<bf16> copy;
        float root[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float x = widen(g.v[i]);
            // products and sums rounded one by one, as the formula has them: 8-bit states then round the same way wherever the
            // step is computed in float32
            m.v[i] = c.beta1 * m.v[i] + c.rest1 * x;
            v.v[i] = c.beta2 * v.v[i] + c.rest2 * x * x;
            root[i] = sqrtf(v.v[i]);
            // The quotient to two roundings, of a number that is small next to p.  Decay and step are one difference to p: 1 - rate decay would
            // itself be rounded, to 1 where rates are small.
            p.v[i] -= c.decay * p.v[i] + c.rate * m.v[i] * __builtin_amdgcn_rcpf(root[i] * c.root + c.eps);
            copy.v[i] = narrow<bf16>(p.v[i]);
        }
        put(t.param + at, p, some, wide);
        if (t.copy) put(t.copy + at, copy, some, wide);
        if constexpr (EIGHT) {
            const int ms = scale_of(block_most(m.v)), vs = scale_of(block_most(root));
            const float mf = factor[ms], vf = factor[vs];
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const uint64_t place = static_cast<uint64_t>(at) + i;
                const uint32_t random = hash(static_cast<uint32_t>(place) + t.key + static_cast<uint32_t>(place >> 32) * 0x9E3779B9u);
                mc.v[i] = static_cast<uint8_t>(encode(m.v[i], mf, random & 0xFFFF, false));
                vc.v[i] = static_cast<uint8_t>(encode(root[i], vf, random >> 16, true));
            }
            put(static_cast<uint8_t *>(t.m) + at, mc, some, wide);
            put(static_cast<uint8_t *>(t.v) + at, vc, some, wide);
            if (some && threadIdx.x % 16 == 0) {
                t.m_scale[at / HEAD_BLOCK] = static_cast<uint8_t>(ms);
                t.v_scale[at / HEAD_BLOCK] = static_cast<uint8_t>(vs);
            }
        } else {
            put(static_cast<float *>(t.m) + at, m, some, wide);
            put(static_cast<float *>(t.v) + at, v, some, wide);
        }
    }
}

// `param` and `copy` are where m and v go.
__global__ __launch_bounds__(THREADS) void adamw_values_kernel(const Batch b)
{
    constexpr int N = VALUES_EACH;
    const int64_t blocks = b.first[b.count];
    for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        int64_t at;
        const Tensor &t = b.tensor[find<N>(b, block, at)];
        const int some = static_cast<int>(std::max<int64_t>(0, std::min<int64_t>(N, t.n - at)));
        const bool wide = some == N && t.wide;
        if (some == 0) continue;
        Values<uint8_t, N> mc, vc;
        take(mc, static_cast<const uint8_t *>(t.m) + at, some, wide);
        take(vc, static_cast<const uint8_t *>(t.v) + at, some, wide);
        float x[N], root[N];
        decode(mc, t.m_scale[at / HEAD_BLOCK], x);
        decode(vc, t.v_scale[at / HEAD_BLOCK], root);
        Values<bf16, N> m, v;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            m.v[i] = narrow<bf16>(x[i]);
            v.v[i] = narrow<bf16>(root[i] * root[i]);
        }
        put(reinterpret_cast<bf16 *>(t.param) + at, m, some, wide);
        put(t.copy + at, v, some, wide);
    }
}

// Launches for all tensors that have values, TENSORS at a time; a workgroup's block has `values` of them, a launch at most `most` workgroups.
template <class Fill, class Launch>
hipError_t in_batches(int32_t n_tensors, int values, int64_t most, Fill fill, Launch launch)
{
    Batch b{};
    for (int32_t i = 0; i <= n_tensors; ++i) {
        if (b.count == TENSORS || (i == n_tensors && b.count > 0)) {
            const int64_t grid = std::min(b.first[b.count], most);
            launch(b, dim3(static_cast<uint32_t>(grid)));
            if (const hipError_t e = hipGetLastError()) return e;
            b.count = 0;
        }
        if (i == n_tensors) break;
        Tensor &t = b.tensor[b.count];
        fill(i, t);
        if (t.n == 0) continue;
        b.first[b.count + 1] = b.first[b.count] + ceil_div(t.n, values);
        ++b.count;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_adamw(const head_adamw_rule &rule, const head_adamw_tensor *tensors, int32_t n_tensors, hipStream_t stream)
{
    const double step = static_cast<double>(rule.step);
    const Numbers c{static_cast<float>(rule.beta1), static_cast<float>(1 - rule.beta1), static_cast<float>(rule.beta2),
                    static_cast<float>(1 - rule.beta2), static_cast<float>(rule.rate * rule.decay),
                    static_cast<float>(rule.rate / (1 - std::pow(rule.beta1, step))),
                    static_cast<float>(1 / std::sqrt(1 - std::pow(rule.beta2, step))), static_cast<float>(rule.eps)};
    const uint32_t key = hash(rule.seed + 0x9E3779B9u * static_cast<uint32_t>(rule.step));
    return in_batches(
        n_tensors, THREADS * EACH, MAX_GRID,
        [&](int32_t i, Tensor &t) {
            const head_adamw_tensor &s = tensors[i];
            t = Tensor{s.param, s.grad, s.m, s.v, s.m_scale, s.v_scale, static_cast<bf16 *>(s.copy), s.n,
                       hash(key + static_cast<uint32_t>(i)), 0};
            const uint64_t states = address(s.m) | address(s.v);
            t.wide = (address(s.param) | address(s.grad) | address(s.copy)) % 16 == 0 && states % (rule.bits == 8 ? EACH : 16) == 0;
        },
        [&](const Batch &b, dim3 grid) {
            const bool narrow_grad = rule.grad_dtype == HEAD_BF16;
            auto *kernel = rule.bits == 8 ? (narrow_grad ? adamw_kernel<bf16, true> : adamw_kernel<float, true>)
                                          : (narrow_grad ? adamw_kernel<bf16, false> : adamw_kernel<float, false>);
            hipLaunchKernelGGL(kernel, grid, dim3(THREADS), 0, stream, b, c);
        });
}

hipError_t launch_adamw_values(const head_adamw_tensor *tensors, void *const *out_m, void *const *out_v, int32_t n_tensors,
                               hipStream_t stream)
{
    return in_batches(
        n_tensors, THREADS * VALUES_EACH, MAX_VALUES_GRID,
        [&](int32_t i, Tensor &t) {
            const head_adamw_tensor &s = tensors[i];
            t = Tensor{static_cast<float *>(out_m[i]), nullptr, s.m, s.v, s.m_scale, s.v_scale, static_cast<bf16 *>(out_v[i]), s.n, 0, 0};
            t.wide = (address(s.m) | address(s.v)) % VALUES_EACH == 0 && (address(out_m[i]) | address(out_v[i])) % 16 == 0;
        },
        [&](const Batch &b, dim3 grid) { hipLaunchKernelGGL(adamw_values_kernel, grid, dim3(THREADS), 0, stream, b); });
}

}  // namespace head_impl
