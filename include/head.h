/*
 * head.h -- C ABI of the trainable head over leaf ids of the MI355X (gfx950) library.
 *
 * A forest turns a row into one leaf per tree (forest_predict_leaves).  A head has a vector of `dim` values for every
 * node, sums the vectors of a row's leaves, normalises the sum and scores classes with a linear softmax model: what
 * refits the leaves of a forest on other data, or uses its trees as feature encoders.  Here are the operators that train
 * it, each with its gradient, and the update of its weights; a trained head of up to LINEAR_MAX_OUTPUTS classes is served
 * by head_embed, head_layer_norm and linear_predict.
 *
 * Same conventions as forest.h and linear.h: extern "C", plain pointers and sizes, 0 or a negative HEAD_E* code, no
 * exceptions, no aborts.  All pointers to values are DEVICE memory of the current device unless marked otherwise;
 * all calls are asynchronous on `stream` (hipStream_t, NULL = default stream), allocate nothing, keep nothing and touch no
 * shared state, so that calls on different streams with different workspaces may overlap.  The caller keeps inputs,
 * outputs and workspace alive until the stream has run the work.  Results do not depend on timing: the same call gives
 * the same bits.  Kernels only, so that every call can be captured into a graph.
 *
 * Values are float32 or bfloat16 (dtype).  Sums, statistics and states are float32; a bfloat16 output is rounded once,
 * to nearest even, and inside head_cross_entropy_grad the gradient of a logit is rounded before it is multiplied: to
 * bfloat16 where there are many logits (at least 256 rows and 256 classes, that fill or begin 256 tiles of 256 x 256: some 2^24), to two of
 * them (16 bits) elsewhere.  Pointers are aligned to their elements.  A row stride counts elements and is at least the row's length;
 * the elements of a row are adjacent.  Outputs are contiguous, and overlap neither inputs nor each other.
 */
#ifndef HEAD_H_
#define HEAD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { HEAD_F32 = 0, HEAD_BF16 = 1 };

enum {
    HEAD_OK = 0,
    HEAD_EINVAL = -1, /* null or misaligned pointer, bad size, stride or enum value */
    HEAD_EHIP = -6,   /* a HIP runtime call failed (no device, launch error, ...) */
    HEAD_ELIMIT = -7  /* a size exceeds a documented limit */
};

/* Documented limits (HEAD_ELIMIT): */
#define HEAD_MAX_DIM 16384           /* dim */
#define HEAD_MAX_ROWS 1000000000     /* n_rows */
#define HEAD_MAX_VECTORS 1000000000  /* n_vectors, n_classes */
#define HEAD_MAX_IDS 2147483647      /* n_ids */
#define HEAD_MAX_TOKENS 2147483647   /* n_rows * n_ids, of head_embed_grad */
#define HEAD_MAX_LOGITS (INT64_C(1) << 44) /* n_rows * n_classes */
#define HEAD_MAX_TENSORS 1000000     /* tensors of one head_adamw call */
#define HEAD_BLOCK 128               /* values that share a scale byte in the 8-bit states */

/*
 * The ids of a batch: row r has n_ids ids, ids[r * ids_stride + t].  Id t of a row stands for vector ids[..] + offset[t]
 * (offset NULL: zeros).  With the ids of forest_predict_leaves, offset is the forest's tree_offset, and there is a
 * vector for every node; n_ids == 1 is a plain lookup.  A negative id, or one whose vector is outside [0, n_vectors), stands
 * for nothing: it adds nothing to the sum and gets no gradient, and a row with no other ids has the sum 0.
 */
typedef struct head_ids {
    int64_t n_rows;
    int64_t n_ids;
    int64_t n_vectors;
    const int32_t *ids;
    int64_t ids_stride;
    const int64_t *offset; /* [n_ids] or NULL */
} head_ids;

/* out[r][.] = scale * sum_t table[vector of id t of row r][.]; table [n_vectors][dim], out [n_rows][dim], both of dtype. */
int head_embed(const head_ids *ids, int32_t dtype, int64_t dim, const void *table, int64_t table_stride, float scale, void *out,
               void *stream);

/* Bytes of workspace (16-byte aligned) head_embed_grad needs; negative HEAD_E* on error.  Pointers in `ids` are not read. */
int64_t head_embed_grad_bytes(const head_ids *ids, int32_t dtype, int64_t dim);

/*
 * grad_table[v][.] = scale * sum of grad[r][.] over all ids of all rows that stand for vector v; zero for a vector that none
 * stands for.  grad [n_rows][dim], grad_table [n_vectors][dim], both of dtype.  The ids are sorted by their vectors, and
 * each vector's rows are added in a fixed order.
 */
int head_embed_grad(const head_ids *ids, int32_t dtype, int64_t dim, const void *grad, int64_t grad_stride, float scale,
                    void *grad_table, void *workspace, void *stream);

/*
 * Layer norm: mean[r] and rstd[r] = 1 / sqrt(variance + eps) over the dim >= 1 values of row r (variance without
 * correction), y = (x - mean) * rstd * weight + bias.  x, y of dtype; weight, bias [dim], mean, rstd [n_rows] float32; bias
 * may be NULL (zeros).  eps >= 0.
 */
int head_layer_norm(int32_t dtype, int64_t n_rows, int64_t dim, const void *x, int64_t x_stride, const float *weight,
                    const float *bias, float eps, void *y, float *mean, float *rstd, void *stream);

/* Bytes of workspace (16-byte aligned) head_layer_norm_grad needs; negative HEAD_E* on error. */
int64_t head_layer_norm_grad_bytes(int32_t dtype, int64_t n_rows, int64_t dim);

/*
 * Its gradients from grad [n_rows][dim] (of y): grad_x of dtype, grad_weight and grad_bias [dim] float32.  mean and rstd are
 * what head_layer_norm gave.
 */
int head_layer_norm_grad(int32_t dtype, int64_t n_rows, int64_t dim, const void *grad, int64_t grad_stride, const void *x,
                         int64_t x_stride, const float *weight, const float *mean, const float *rstd, void *grad_x,
                         float *grad_weight, float *grad_bias, void *workspace, void *stream);

/*
 * A linear softmax model and its batch: logit[r][k] = sum_d hidden[r][d] * weight[k][d] + bias[k].  hidden [n_rows][dim]
 * and weight [n_classes][dim] of dtype, bias [n_classes] float32 or NULL (zeros).  target[r] outside [0, n_classes) (-1, say):
 * the row has no target, its loss is 0 and it has no gradient: grad_hidden is 0 there, and what the row of hidden, lse and
 * grad_loss holds, finite or not, counts for no gradient.
 */
typedef struct head_classes {
    int32_t dtype;
    int64_t n_rows;
    int64_t dim;
    int64_t n_classes;
    const void *hidden;
    int64_t hidden_stride;
    const void *weight;
    int64_t weight_stride;
    const float *bias;
    const int32_t *target; /* [n_rows] */
} head_classes;

/* Bytes of workspace (16-byte aligned) of the two calls below; negative HEAD_E* on error.  Of the pointers and strides in
 * `c` only the alignment counts.  The gradients' grows with the rows: it has room for 1,024 classes of all of them, or for fewer where
 * there are fewer. */
int64_t head_cross_entropy_bytes(const head_classes *c);
int64_t head_cross_entropy_grad_bytes(const head_classes *c);

/*
 * lse[r] = log sum_k exp(logit[r][k]), loss[r] = lse[r] - logit[r][target[r]], both [n_rows] float32.  The logits are taken
 * in pieces and never kept.
 */
int head_cross_entropy(const head_classes *c, float *loss, float *lse, void *workspace, void *stream);

/*
 * The gradients of sum_r grad_loss[r] * loss[r] (grad_loss [n_rows] float32): grad_hidden [n_rows][dim] and grad_weight
 * [n_classes][dim] of dtype, grad_bias [n_classes] float32 or NULL (not wanted).  lse is what head_cross_entropy gave for
 * the same batch; the logits are computed again, in pieces of the classes.
 */
int head_cross_entropy_grad(const head_classes *c, const float *lse, const float *grad_loss, void *grad_hidden,
                            void *grad_weight, float *grad_bias, void *workspace, void *stream);

/*
 * One AdamW step over all tensors.  For every value, with step >= 1 counting from the first one:
 *     m = beta1 * m + (1 - beta1) * g;  v = beta2 * v + (1 - beta2) * g * g
 *     param -= rate * decay * param + rate / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * bits == 32: m, v are float32 [n].  bits == 8: m, v are e4m3 codes [n], of m and of the root of v, and m_scale, v_scale
 * have a byte s for each HEAD_BLOCK values: a code's value counts times 2^(s - 134), where s - 127 is the exponent of the
 * block's largest magnitude, or -120 where that is less (s == 0: a block of zeros; states start as zero bytes).  Codes, of
 * values times 2^(134 - s) to a float32 rounding, are rounded up where the fraction that they cannot hold plus a random number reaches one, so that they are right on average, and small changes
 * of v are not lost; a root of v above 0 never gets the code of 0, because m divided by it would have no bound.  The random
 * number is a hash of seed, step, the tensor's place in the list and the value's in the tensor.  A state that is not
 * finite is kept as the code of NaN, and does not count for the block's scale.
 * copy (or NULL): a bfloat16 copy of the new param.  grad is of grad_dtype.  The list and what it says is HOST memory, borrowed
 * for the call; the numbers of a captured call (step, rate) are those of its capture.
 */
typedef struct head_adamw_tensor {
    float *param;
    const void *grad;
    void *m, *v;
    uint8_t *m_scale, *v_scale; /* [ceil(n / HEAD_BLOCK)], bits == 8 only */
    void *copy;
    int64_t n;
} head_adamw_tensor;

typedef struct head_adamw_rule {
    int32_t grad_dtype;
    int32_t bits; /* 32 or 8 */
    int64_t step;
    double rate, beta1, beta2, eps, decay; /* finite; 0 <= beta < 1; eps >= 0 */
    uint32_t seed;
} head_adamw_rule;

int head_adamw(const head_adamw_rule *rule, const head_adamw_tensor *tensors, int32_t n_tensors, void *stream);

/*
 * What 8-bit states stand for: m and v of every tensor as bfloat16 (exact where bfloat16 has the exponent).  Of a tensor
 * only m, v, m_scale, v_scale and n are used; out_m[i] and out_v[i] ([n] bfloat16) are HOST arrays of device pointers.
 */
int head_adamw_values(const head_adamw_tensor *tensors, void *const *out_m, void *const *out_v, int32_t n_tensors, void *stream);

const char *head_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* HEAD_H_ */
