// What the kernels of dense layers share (formulas: head.h): activations, their slopes, and what a layer's results go through.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "head_device.hpp"

namespace head_impl {

// f(the activation as a constant), so that loops are not full of choices.
template <class F>
__device__ __forceinline__ void with_activation(int32_t activation, F f)
{
    switch (activation) {
        case HEAD_RELU: return f(std::integral_constant<int, HEAD_RELU>());
        case HEAD_GELU: return f(std::integral_constant<int, HEAD_GELU>());
        case HEAD_SILU: return f(std::integral_constant<int, HEAD_SILU>());
        default: return f(std::integral_constant<int, HEAD_IDENTITY>());
    }
}

// exp(x) and 1 / y (y >= 1), to two or three roundings; the exponential besides to x roundings.  expf, erfcf and a division take a float32
// GELU's end from some 40 vector instructions to 150.
__device__ __forceinline__ float exp32(float x)
{
    constexpr float LOG2E = 1.44269502162933349609375f, REST = 1.925963033500011079e-08f;  // together log2(e)
    const float t = x * LOG2E, e = __builtin_amdgcn_exp2f(t), rest = fmaf(x, LOG2E, -t) + x * REST;
    return fabsf(rest) < 1 && e < INFINITY ? fmaf(e, rest * 0.693147180559945f, e) : e;  // infinite: no rest
}
__device__ __forceinline__ float reciprocal32(float y)
{
    const float r = __builtin_amdgcn_rcpf(y);
    return y < INFINITY ? fmaf(fmaf(-y, r, 1.0f), r, r) : r;
}

// Value and slope of an activation at x, for results of type T.  Those of bfloat16 results, whose own rounding is 2^-9 of them, are right to 2^-13: a shorter
// polynomial, and the exponential and the reciprocal as the instructions give them.
template <class T, int ACTIVATION>
struct Activation {
    float value, slope;

    __device__ __forceinline__ explicit Activation(float x)
    {
        if constexpr (ACTIVATION == HEAD_IDENTITY) {
            value = x;
            slope = 1;
        } else if constexpr (ACTIVATION == HEAD_RELU) {
            value = x <= 0 ? 0 : x;  // NaN stays
            slope = x > 0 ? 1 : 0;
        } else if constexpr (ACTIVATION == HEAD_SILU) {
            // value = x s, slope = s + x s (1 - s) with s = 1 / (1 + exp(-x))
            float s;
            if constexpr (sizeof(T) == 4) s = reciprocal32(1 + exp32(-x));
            else s = __builtin_amdgcn_rcpf(1 + __builtin_amdgcn_exp2f(x * -1.44269504088896341f));
            value = x * s;
            slope = s + value * (1 - s);
        } else {
            // value = x P, slope = P + x exp(-x^2 / 2) / sqrt(2 pi) with P(x) = erfc(-x / sqrt 2) / 2.  P(-a) = exp(-a^2 / 2) Q(1 / (1 + c a)) for a >= 0:
            // polynomials fitted (least squares of the relative difference, weighted until its extremes were even) to erfcx(a / sqrt 2) / 2 on
            // [0, 14], 2^-25.3 off at most for float32 results and 2^-14.9 for bfloat16 ones
            float t, e, q;
            if constexpr (sizeof(T) == 4) {
                constexpr float Q[] = {0.10375906527042389f, 0.1030166745185852f, 0.10303077846765518f, 0.05102564021945f, 0.160952627658844f,
                                       -0.15095585584640503f, 0.2514972984790802f, -0.15283173322677612f, 0.030505483970046043f};
                t = reciprocal32(fmaf(fabsf(x), 0.26f, 1.0f));
                e = exp32(-0.5f * x * x);
                q = Q[8];
#pragma unroll
                for (int k = 7; k >= 0; --k) q = fmaf(q, t, Q[k]);
            } else {
                t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.375f, 1.0f));
                e = __builtin_amdgcn_exp2f(x * x * -0.72134752044448170f);
                q = fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.09064799f, 0.20029321f), 0.08355508f), 0.15773682f), 0.14906072f);
            }
            q *= t * e;
            const float p = x > 0 ? 1 - q : q;
            value = x * p;
            slope = fmaf(x * e, 0.398942280401432678f, p);
        }
    }
};

// Where a layer's results go.  Null: not there, not wanted.
template <class T>
struct End {
    int32_t activation;
    const float *bias;
    const T *residual;
    int64_t residual_stride;
    float scale;
    T *y, *z;
    int64_t n_rows, outs;  // columns of y
    bool wide;             // rows of residual, y and z are whole in what a lane stores of them, and short
};

// A layer of few rows, forward (head_few.hip).  splits > 1: the sum's axis is cut, and the parts are added by a kernel of the caller's.
constexpr int64_t FEW_ROWS = 64;
constexpr int FEW_COLUMNS = 16;               // of y, of a workgroup of 512 lanes
constexpr int64_t FEW_WORKGROUPS = 1 << 22;   // of a launch: 2^31 lanes, a grid's axis has room for 2^32.  Layers of more columns go by tiles

// Whether it reads rows in whole pieces of 16 bytes; value by value otherwise.
inline bool few_wide(const head_layer &l)
{
    const uint64_t strides = static_cast<uint64_t>((l.x_stride | l.weight_stride | l.dim) * value_bytes(l.dtype));
    return (address(l.x) | address(l.weight) | strides) % 16 == 0;
}

template <class T, bool GATED>
hipError_t launch_few(const head_layer &l, const End<T> &end, int64_t splits, float *parts, hipStream_t stream);

}  // namespace head_impl
