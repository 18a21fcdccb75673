// C ABI of the trainable head: the checks of every call, before any of its kernels.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/head.h"
#include "head_device.hpp"

using namespace head_impl;

namespace {

bool is_dtype(int32_t dtype) { return dtype == HEAD_F32 || dtype == HEAD_BF16; }

template <class P>
bool misaligned(const P *p, int bytes)
{
    return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) != 0;
}

// A pointer that is read or written through.
template <class P>
bool bad(const P *p, int bytes)
{
    return !p || misaligned(p, bytes);
}

int done(hipError_t e) { return e == hipSuccess ? HEAD_OK : HEAD_EHIP; }

int check_shape(int32_t dtype, int64_t n_rows, int64_t dim)
{
    if (!is_dtype(dtype) || n_rows < 0 || dim < 1) return HEAD_EINVAL;
    if (n_rows > HEAD_MAX_ROWS || dim > HEAD_MAX_DIM) return HEAD_ELIMIT;
    return HEAD_OK;
}

int check_ids(const head_ids *ids, int32_t dtype, int64_t dim)
{
    if (!ids || ids->n_ids < 0 || ids->n_vectors < 0) return HEAD_EINVAL;
    if (int rc = check_shape(dtype, ids->n_rows, dim)) return rc;
    if (ids->n_ids > HEAD_MAX_IDS || ids->n_vectors > HEAD_MAX_VECTORS) return HEAD_ELIMIT;
    return HEAD_OK;
}

// A row of n values that start every `stride`.
bool bad_stride(int64_t stride, int64_t n) { return stride < n || stride > (int64_t{1} << 40); }

int check_id_pointers(const head_ids &ids)
{
    if (ids.n_rows == 0 || ids.n_ids == 0) return HEAD_OK;
    if (bad(ids.ids, 4) || bad_stride(ids.ids_stride, ids.n_ids) || misaligned(ids.offset, 8)) return HEAD_EINVAL;
    return HEAD_OK;
}

int check_classes(const head_classes *c)
{
    if (!c || c->n_classes < 1) return HEAD_EINVAL;
    if (int rc = check_shape(c->dtype, c->n_rows, c->dim)) return rc;
    if (c->n_classes > HEAD_MAX_VECTORS || (c->n_rows > 0 && c->n_classes > HEAD_MAX_LOGITS / c->n_rows)) return HEAD_ELIMIT;
    return HEAD_OK;
}

int check_class_pointers(const head_classes &c)
{
    const int e = value_bytes(c.dtype);
    if (bad(c.weight, e) || bad_stride(c.weight_stride, c.dim) || misaligned(c.bias, 4)) return HEAD_EINVAL;
    if (c.n_rows > 0 && (bad(c.hidden, e) || bad_stride(c.hidden_stride, c.dim) || bad(c.target, 4))) return HEAD_EINVAL;
    return HEAD_OK;
}

// A layer whose z has `halves` times n_outputs columns.
int check_layer(const head_layer *l, int halves)
{
    if (!l || l->n_outputs < 1 || l->activation < HEAD_IDENTITY || l->activation > HEAD_SILU) return HEAD_EINVAL;
    if (int rc = check_shape(l->dtype, l->n_rows, l->dim)) return rc;
    if (l->n_outputs > HEAD_MAX_VECTORS / halves || (l->n_rows > 0 && l->n_outputs > HEAD_MAX_LOGITS / halves / l->n_rows)) return HEAD_ELIMIT;
    return HEAD_OK;
}

int check_layer_pointers(const head_layer &l)
{
    const int e = value_bytes(l.dtype);
    if (bad(l.weight, e) || bad_stride(l.weight_stride, l.dim) || misaligned(l.bias, 4)) return HEAD_EINVAL;
    if (l.n_rows > 0 && (bad(l.x, e) || bad_stride(l.x_stride, l.dim))) return HEAD_EINVAL;
    return HEAD_OK;
}

int check_layer_grad(const head_layer &l, int halves, bool has_z, int64_t bytes, const void *z, int64_t z_stride, const void *grad, int64_t grad_stride,
                     const void *grad_x, const void *grad_weight, const float *grad_bias, const void *workspace)
{
    if (int rc = check_layer_pointers(l)) return rc;
    const int e = value_bytes(l.dtype);
    if (bad(grad_weight, e) || misaligned(grad_bias, 4) || (bytes > 0 && bad(workspace, 16))) return HEAD_EINVAL;
    if (l.n_rows == 0) return HEAD_OK;
    if (bad(grad, e) || bad_stride(grad_stride, l.n_outputs) || bad(grad_x, e)) return HEAD_EINVAL;
    if (has_z && (bad(z, e) || bad_stride(z_stride, halves * l.n_outputs))) return HEAD_EINVAL;
    return HEAD_OK;
}

int check_clip(const head_clip_tensor *tensors, int32_t n_tensors)
{
    if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return HEAD_EINVAL;
    if (n_tensors > HEAD_MAX_TENSORS) return HEAD_ELIMIT;
    for (int32_t i = 0; i < n_tensors; ++i) {
        if (tensors[i].n < 0) return HEAD_EINVAL;
        if (tensors[i].n > (int64_t{1} << 40)) return HEAD_ELIMIT;
    }
    return HEAD_OK;
}

int check_tensors(const head_adamw_tensor *tensors, int32_t n_tensors)
{
    if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return HEAD_EINVAL;
    if (n_tensors > HEAD_MAX_TENSORS) return HEAD_ELIMIT;
    for (int32_t i = 0; i < n_tensors; ++i) {
        if (tensors[i].n < 0) return HEAD_EINVAL;
        if (tensors[i].n > (int64_t{1} << 40)) return HEAD_ELIMIT;
    }
    return HEAD_OK;
}

}  // namespace

extern "C" {

int head_embed(const head_ids *ids, int32_t dtype, int64_t dim, const void *table, int64_t table_stride, float scale, void *out,
               void *stream)
{
    if (int rc = check_ids(ids, dtype, dim)) return rc;
    if (ids->n_rows == 0) return HEAD_OK;
    if (int rc = check_id_pointers(*ids)) return rc;
    const int e = value_bytes(dtype);
    if (bad(out, e)) return HEAD_EINVAL;
    if (ids->n_vectors > 0 && (bad(table, e) || bad_stride(table_stride, dim))) return HEAD_EINVAL;
    return done(launch_embed(*ids, dtype, dim, table, table_stride, scale, out, static_cast<hipStream_t>(stream)));
}

int64_t head_embed_grad_bytes(const head_ids *ids, int32_t dtype, int64_t dim)
{
    if (int rc = check_ids(ids, dtype, dim)) return rc;
    if (ids->n_ids > 0 && ids->n_rows > HEAD_MAX_TOKENS / ids->n_ids) return HEAD_ELIMIT;
    return embed_grad_bytes(*ids, dtype, dim);
}

int head_embed_grad(const head_ids *ids, int32_t dtype, int64_t dim, const void *grad, int64_t grad_stride, float scale,
                    void *grad_table, void *workspace, void *stream)
{
    const int64_t bytes = head_embed_grad_bytes(ids, dtype, dim);
    if (bytes < 0) return static_cast<int>(bytes);
    if (ids->n_vectors == 0) return HEAD_OK;
    if (int rc = check_id_pointers(*ids)) return rc;
    const int e = value_bytes(dtype);
    if (bad(grad_table, e) || (bytes > 0 && bad(workspace, 16))) return HEAD_EINVAL;
    if (ids->n_rows > 0 && (bad(grad, e) || bad_stride(grad_stride, dim))) return HEAD_EINVAL;
    return done(launch_embed_grad(*ids, dtype, dim, grad, grad_stride, scale, grad_table, workspace, static_cast<hipStream_t>(stream)));
}

int head_layer_norm(int32_t dtype, int64_t n_rows, int64_t dim, const void *x, int64_t x_stride, const float *weight,
                    const float *bias, float eps, void *y, float *mean, float *rstd, void *stream)
{
    if (int rc = check_shape(dtype, n_rows, dim)) return rc;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return HEAD_EINVAL;
    if (n_rows == 0) return HEAD_OK;
    const int e = value_bytes(dtype);
    if (bad(x, e) || bad_stride(x_stride, dim) || bad(weight, 4) || misaligned(bias, 4)) return HEAD_EINVAL;
    if (bad(y, e) || bad(mean, 4) || bad(rstd, 4)) return HEAD_EINVAL;
    return done(launch_layer_norm(dtype, n_rows, dim, x, x_stride, weight, bias, eps, y, mean, rstd, static_cast<hipStream_t>(stream)));
}

int64_t head_layer_norm_grad_bytes(int32_t dtype, int64_t n_rows, int64_t dim)
{
    if (int rc = check_shape(dtype, n_rows, dim)) return rc;
    return layer_norm_grad_bytes(dtype, n_rows, dim);
}

int head_layer_norm_grad(int32_t dtype, int64_t n_rows, int64_t dim, const void *grad, int64_t grad_stride, const void *x,
                         int64_t x_stride, const float *weight, const float *mean, const float *rstd, void *grad_x,
                         float *grad_weight, float *grad_bias, void *workspace, void *stream)
{
    const int64_t bytes = head_layer_norm_grad_bytes(dtype, n_rows, dim);
    if (bytes < 0) return static_cast<int>(bytes);
    if (bad(grad_weight, 4) || bad(grad_bias, 4) || (bytes > 0 && bad(workspace, 16))) return HEAD_EINVAL;
    const int e = value_bytes(dtype);
    if (n_rows > 0) {
        if (bad(grad, e) || bad_stride(grad_stride, dim) || bad(x, e) || bad_stride(x_stride, dim)) return HEAD_EINVAL;
        if (bad(weight, 4) || bad(mean, 4) || bad(rstd, 4) || bad(grad_x, e)) return HEAD_EINVAL;
    }
    return done(launch_layer_norm_grad(dtype, n_rows, dim, grad, grad_stride, x, x_stride, weight, mean, rstd, grad_x, grad_weight,
                                       grad_bias, workspace, static_cast<hipStream_t>(stream)));
}

int64_t head_cross_entropy_bytes(const head_classes *c)
{
    if (int rc = check_classes(c)) return rc;
    return cross_entropy_bytes(*c);
}

int head_cross_entropy(const head_classes *c, float *loss, float *lse, void *workspace, void *stream)
{
    const int64_t bytes = head_cross_entropy_bytes(c);
    if (bytes < 0) return static_cast<int>(bytes);
    if (int rc = check_class_pointers(*c)) return rc;
    if (c->n_rows == 0) return HEAD_OK;
    if (bad(loss, 4) || bad(lse, 4) || (bytes > 0 && bad(workspace, 16))) return HEAD_EINVAL;
    return done(launch_cross_entropy(*c, loss, lse, workspace, static_cast<hipStream_t>(stream)));
}

int64_t head_cross_entropy_grad_bytes(const head_classes *c)
{
    if (int rc = check_classes(c)) return rc;
    return cross_entropy_grad_bytes(*c);
}

int head_cross_entropy_grad(const head_classes *c, const float *lse, const float *grad_loss, void *grad_hidden,
                            void *grad_weight, float *grad_bias, void *workspace, void *stream)
{
    const int64_t bytes = head_cross_entropy_grad_bytes(c);
    if (bytes < 0) return static_cast<int>(bytes);
    if (int rc = check_class_pointers(*c)) return rc;
    const int e = value_bytes(c->dtype);
    if (bad(grad_weight, e) || misaligned(grad_bias, 4) || (bytes > 0 && bad(workspace, 16))) return HEAD_EINVAL;
    if (c->n_rows > 0 && (bad(lse, 4) || bad(grad_loss, 4) || bad(grad_hidden, e))) return HEAD_EINVAL;
    return done(launch_cross_entropy_grad(*c, lse, grad_loss, grad_hidden, grad_weight, grad_bias, workspace,
                                          static_cast<hipStream_t>(stream)));
}

int64_t head_linear_bytes(const head_layer *l)
{
    if (int rc = check_layer(l, 1)) return rc;
    return linear_bytes(*l);
}

int head_linear(const head_layer *l, const void *residual, int64_t residual_stride, float scale, void *y, void *z, void *workspace,
                void *stream)
{
    const int64_t bytes = head_linear_bytes(l);
    if (bytes < 0) return static_cast<int>(bytes);
    if (int rc = check_layer_pointers(*l)) return rc;
    if (l->n_rows == 0) return HEAD_OK;
    const int e = value_bytes(l->dtype);
    if (bad(y, e) || misaligned(z, e) || (bytes > 0 && bad(workspace, 16))) return HEAD_EINVAL;
    if (residual && (misaligned(residual, e) || bad_stride(residual_stride, l->n_outputs))) return HEAD_EINVAL;
    return done(launch_linear(*l, residual, residual_stride, scale, y, z, workspace, static_cast<hipStream_t>(stream)));
}

int64_t head_linear_grad_bytes(const head_layer *l)
{
    if (int rc = check_layer(l, 1)) return rc;
    if (l->n_outputs > HEAD_MAX_OUTPUTS) return HEAD_ELIMIT;
    return linear_grad_bytes(*l);
}

int head_linear_grad(const head_layer *l, const void *z, int64_t z_stride, const void *grad, int64_t grad_stride, float scale,
                     void *grad_x, void *grad_weight, float *grad_bias, void *workspace, void *stream)
{
    const int64_t bytes = head_linear_grad_bytes(l);
    if (bytes < 0) return static_cast<int>(bytes);
    if (int rc = check_layer_grad(*l, 1, l->activation != HEAD_IDENTITY, bytes, z, z_stride, grad, grad_stride, grad_x, grad_weight, grad_bias,
                                  workspace))
        return rc;
    return done(launch_linear_grad(*l, z, z_stride, grad, grad_stride, scale, grad_x, grad_weight, grad_bias, workspace,
                                   static_cast<hipStream_t>(stream)));
}

int64_t head_gated_bytes(const head_layer *l)
{
    if (int rc = check_layer(l, 2)) return rc;
    return gated_bytes(*l);
}

int head_gated(const head_layer *l, void *y, void *z, void *workspace, void *stream)
{
    const int64_t bytes = head_gated_bytes(l);
    if (bytes < 0) return static_cast<int>(bytes);
    if (int rc = check_layer_pointers(*l)) return rc;
    if (l->n_rows == 0) return HEAD_OK;
    const int e = value_bytes(l->dtype);
    if (bad(y, e) || misaligned(z, e) || (bytes > 0 && bad(workspace, 16))) return HEAD_EINVAL;
    return done(launch_gated(*l, y, z, workspace, static_cast<hipStream_t>(stream)));
}

int64_t head_gated_grad_bytes(const head_layer *l)
{
    if (int rc = check_layer(l, 2)) return rc;
    if (l->n_outputs > HEAD_MAX_OUTPUTS) return HEAD_ELIMIT;
    return gated_grad_bytes(*l);
}

int head_gated_grad(const head_layer *l, const void *z, int64_t z_stride, const void *grad, int64_t grad_stride, void *grad_x,
                    void *grad_weight, float *grad_bias, void *workspace, void *stream)
{
    const int64_t bytes = head_gated_grad_bytes(l);
    if (bytes < 0) return static_cast<int>(bytes);
    if (int rc = check_layer_grad(*l, 2, true, bytes, z, z_stride, grad, grad_stride, grad_x, grad_weight, grad_bias, workspace)) return rc;
    return done(launch_gated_grad(*l, z, z_stride, grad, grad_stride, grad_x, grad_weight, grad_bias, workspace, static_cast<hipStream_t>(stream)));
}

int head_layer_launch(const head_layer *l, int32_t gated, head_layer_launch_t *out)
{
    if (int rc = check_layer(l, gated ? 2 : 1)) return rc;
    if (!out || l->n_rows < 1) return HEAD_EINVAL;
    *out = layer_launch(*l, gated != 0);
    return HEAD_OK;
}

int head_adamw(const head_adamw_rule *rule, const head_adamw_tensor *tensors, int32_t n_tensors, void *stream)
{
    if (!rule || !is_dtype(rule->grad_dtype) || (rule->bits != 32 && rule->bits != 8) || rule->step < 1) return HEAD_EINVAL;
    if (!std::isfinite(rule->rate) || !std::isfinite(rule->decay) || !(rule->eps >= 0) || !std::isfinite(rule->eps)) return HEAD_EINVAL;
    if (!(rule->beta1 >= 0 && rule->beta1 < 1 && rule->beta2 >= 0 && rule->beta2 < 1)) return HEAD_EINVAL;
    if (int rc = check_tensors(tensors, n_tensors)) return rc;
    const int state = rule->bits == 32 ? 4 : 1;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const head_adamw_tensor &t = tensors[i];
        if (t.n == 0) continue;
        if (bad(t.param, 4) || bad(t.grad, value_bytes(rule->grad_dtype)) || bad(t.m, state) || bad(t.v, state)) return HEAD_EINVAL;
        if (misaligned(t.copy, 2) || (rule->bits == 8 && (!t.m_scale || !t.v_scale))) return HEAD_EINVAL;
    }
    return done(launch_adamw(*rule, tensors, n_tensors, static_cast<hipStream_t>(stream)));
}

int head_adamw_values(const head_adamw_tensor *tensors, void *const *out_m, void *const *out_v, int32_t n_tensors, void *stream)
{
    if (int rc = check_tensors(tensors, n_tensors)) return rc;
    if (n_tensors > 0 && (!out_m || !out_v)) return HEAD_EINVAL;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const head_adamw_tensor &t = tensors[i];
        if (t.n == 0) continue;
        if (!t.m || !t.v || !t.m_scale || !t.v_scale || bad(out_m[i], 2) || bad(out_v[i], 2)) return HEAD_EINVAL;
    }
    return done(launch_adamw_values(tensors, out_m, out_v, n_tensors, static_cast<hipStream_t>(stream)));
}

int64_t head_clip_bytes(const head_clip_tensor *tensors, int32_t n_tensors)
{
    if (int rc = check_clip(tensors, n_tensors)) return rc;
    return clip_bytes(tensors, n_tensors);
}

int head_clip(const head_clip_tensor *tensors, int32_t n_tensors, double max_norm, float *norm, void *workspace, void *stream)
{
    const int64_t bytes = head_clip_bytes(tensors, n_tensors);
    if (bytes < 0) return static_cast<int>(bytes);
    if (!(max_norm > 0) || bad(norm, 4) || (bytes > 0 && bad(workspace, 16))) return HEAD_EINVAL;
    int32_t outs = 0, some = 0;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const head_clip_tensor &t = tensors[i];
        if (!is_dtype(t.dtype)) return HEAD_EINVAL;
        if (t.n == 0) continue;
        const int e = value_bytes(t.dtype);
        if (bad(t.grad, e) || misaligned(t.out, e)) return HEAD_EINVAL;
        ++some;
        outs += t.out != nullptr;
    }
    if (outs != 0 && outs != some) return HEAD_EINVAL;
    return done(launch_clip(tensors, n_tensors, max_norm, norm, workspace, static_cast<hipStream_t>(stream)));
}

const char *head_strerror(int code)
{
    switch (code) {
        case HEAD_OK: return "ok";
        case HEAD_EINVAL: return "invalid argument";
        case HEAD_EHIP: return "HIP runtime error";
        case HEAD_ELIMIT: return "a size exceeds a documented limit";
        default: return "unknown error";
    }
}

}  // extern "C"
