/*
 * head_testing.h -- host-only view of what a call on a layer of the trainable head launches, for the library's tests.
 * Not part of the head's ABI (include/head.h); no GPU needed.
 */
#ifndef HEAD_TESTING_H_
#define HEAD_TESTING_H_

#include <stdint.h>

#include "head.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct head_layer_launch_t {
    int32_t few;                          /* forward: parts of the sum's axis in the kernel for few rows; 0: by tiles */
    int32_t copies_x, copies_weight;      /* by tiles and backward, 1: copied first to rows that products can read */
    int32_t tile, splits;                 /* forward by tiles: rows of a tile, parts of the sum's axis; 0: not by tiles */
    int32_t to_x_tile, to_x_splits;       /* the gradient of x; 0: the layer has too many outputs for gradients */
    int32_t to_weight_tile, to_weight_splits;
} head_layer_launch_t;

/*
 * What head_linear and head_linear_grad, or (gated) head_gated and head_gated_grad, launch for a layer of at least one row.  Of its pointers and strides
 * that counts which counts for the workspace.  Returns HEAD_OK, HEAD_EINVAL or HEAD_ELIMIT.
 */
int head_layer_launch(const head_layer *l, int32_t gated, head_layer_launch_t *out);

#ifdef __cplusplus
}
#endif
#endif /* HEAD_TESTING_H_ */
