// What the kernels of the trainable head share: the two types of values, rows read in pieces as wide as their alignment
// allows, and the launches that head_api.cpp makes after its checks.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>

#include "../../include/head.h"
#include "../../include/head_testing.h"

namespace head_impl {

using bf16 = __bf16;

// N adjacent values, read and written as one.
template <class T, int N>
struct alignas(sizeof(T) * N) Pack {
    T v[N];
};

template <class T>
__device__ __forceinline__ float widen(T x)
{
    return static_cast<float>(x);
}
template <class T>
__device__ __forceinline__ T narrow(float x)  // to nearest even
{
    return static_cast<T>(x);
}

// The machine word of that many bytes.
template <int BYTES> struct WordOf;
template <> struct WordOf<2> { using Type = uint16_t; };
template <> struct WordOf<4> { using Type = uint32_t; };
template <> struct WordOf<8> { using Type = uint32_t __attribute__((ext_vector_type(2))); };
template <> struct WordOf<16> { using Type = uint32_t __attribute__((ext_vector_type(4))); };

// A store of what nobody reads soon.
template <class T, int N>
__device__ __forceinline__ void store_past(T *to, const Pack<T, N> &p)
{
    using Word = typename WordOf<sizeof(T) * N>::Type;
    __builtin_nontemporal_store(*reinterpret_cast<const Word *>(&p), reinterpret_cast<Word *>(to));
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
inline int value_bytes(int32_t dtype) { return dtype == HEAD_BF16 ? 2 : 4; }

// Values in the widest piece, of at most 16 bytes, that addresses and lengths in bytes (all or'ed into `bits`) are whole in.
inline int piece(uint64_t bits, int value)
{
    int bytes = 16;
    while (bytes > value && bits % bytes) bytes /= 2;
    return bytes / value;
}
template <class P>
inline uint64_t address(const P *p)
{
    return reinterpret_cast<uintptr_t>(p);
}

// More than 64 KB of LDS has to be asked for, once for each kernel and device.
template <auto *KERNEL>
hipError_t allow_lds(size_t bytes)
{
    constexpr int DEVICES = 64;
    static std::atomic<bool> done[DEVICES];
    int device = -1;
    if (const hipError_t e = hipGetDevice(&device)) return e;
    if (device >= 0 && device < DEVICES && done[device].load(std::memory_order_relaxed)) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
    if (e == hipSuccess && device >= 0 && device < DEVICES) done[device].store(true, std::memory_order_relaxed);
    return e;
}

hipError_t launch_embed(const head_ids &ids, int32_t dtype, int64_t dim, const void *table, int64_t table_stride, float scale,
                        void *out, hipStream_t stream);
int64_t embed_grad_bytes(const head_ids &ids, int32_t dtype, int64_t dim);
hipError_t launch_embed_grad(const head_ids &ids, int32_t dtype, int64_t dim, const void *grad, int64_t grad_stride, float scale,
                             void *grad_table, void *workspace, hipStream_t stream);

hipError_t launch_layer_norm(int32_t dtype, int64_t n_rows, int64_t dim, const void *x, int64_t x_stride, const float *weight,
                             const float *bias, float eps, void *y, float *mean, float *rstd, hipStream_t stream);
int64_t layer_norm_grad_bytes(int32_t dtype, int64_t n_rows, int64_t dim);
hipError_t launch_layer_norm_grad(int32_t dtype, int64_t n_rows, int64_t dim, const void *grad, int64_t grad_stride, const void *x,
                                  int64_t x_stride, const float *weight, const float *mean, const float *rstd, void *grad_x,
                                  float *grad_weight, float *grad_bias, void *workspace, hipStream_t stream);

int64_t cross_entropy_bytes(const head_classes &c);
hipError_t launch_cross_entropy(const head_classes &c, float *loss, float *lse, void *workspace, hipStream_t stream);
int64_t cross_entropy_grad_bytes(const head_classes &c);
hipError_t launch_cross_entropy_grad(const head_classes &c, const float *lse, const float *grad_loss, void *grad_hidden,
                                     void *grad_weight, float *grad_bias, void *workspace, hipStream_t stream);

int64_t linear_bytes(const head_layer &l);
int64_t linear_grad_bytes(const head_layer &l);
int64_t gated_bytes(const head_layer &l);
int64_t gated_grad_bytes(const head_layer &l);
hipError_t launch_linear(const head_layer &l, const void *residual, int64_t residual_stride, float scale, void *y, void *z, void *workspace,
                         hipStream_t stream);
hipError_t launch_linear_grad(const head_layer &l, const void *z, int64_t z_stride, const void *grad, int64_t grad_stride, float scale,
                              void *grad_x, void *grad_weight, float *grad_bias, void *workspace, hipStream_t stream);
hipError_t launch_gated(const head_layer &l, void *y, void *z, void *workspace, hipStream_t stream);
hipError_t launch_gated_grad(const head_layer &l, const void *z, int64_t z_stride, const void *grad, int64_t grad_stride, void *grad_x,
                             void *grad_weight, float *grad_bias, void *workspace, hipStream_t stream);

head_layer_launch_t layer_launch(const head_layer &l, bool gated);

int64_t clip_bytes(const head_clip_tensor *tensors, int32_t n_tensors);
hipError_t launch_clip(const head_clip_tensor *tensors, int32_t n_tensors, double max_norm, float *norm, void *workspace, hipStream_t stream);

hipError_t launch_adamw(const head_adamw_rule &rule, const head_adamw_tensor *tensors, int32_t n_tensors, hipStream_t stream);
hipError_t launch_adamw_values(const head_adamw_tensor *tensors, void *const *out_m, void *const *out_v, int32_t n_tensors,
                               hipStream_t stream);

}  // namespace head_impl
