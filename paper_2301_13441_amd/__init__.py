"""MI355X-native tree-ensemble inference (dense operator representation, hand-written HIP).

Thin binding over the C ABI declared in include/forest.h, include/linear.h and include/head.h: ctypes, and a CPython extension on
torch's C++ interface for the calls whose time is the host's (csrc/short_call.cpp), without which they go the ctypes way.
PyTorch is used only for device memory and streams, and by LeafHead for its first values, the number of a batch's targets and the mean
loss.  There is no CPU fallback: without the built HIP library, or without a GPU at load time, the calls raise.
"""
from .binding import (Forest, ForestError, forest_load, forest_pack, lib_path, load_library,
                      AGG_SUM, AGG_MEAN, TRANSFORM_NONE, TRANSFORM_SIGMOID, TRANSFORM_SOFTMAX,
                      OUT_SCORES, OUT_LABELS, OUT_BOTH)

from .linear_binding import Linear, LinearError, linear_load
from .head_binding import (HeadError, head_adamw, head_adamw_state, head_adamw_values, head_cross_entropy,
                           head_cross_entropy_grad, head_embed, head_embed_grad, head_layer_norm, head_layer_norm_grad)
from .leaf_head import LeafHead

__all__ = ["Linear", "LinearError", "linear_load", "Forest", "ForestError", "forest_load", "forest_pack", "lib_path", "load_library",
           "AGG_SUM", "AGG_MEAN", "TRANSFORM_NONE", "TRANSFORM_SIGMOID", "TRANSFORM_SOFTMAX",
           "OUT_SCORES", "OUT_LABELS", "OUT_BOTH",
           "HeadError", "head_adamw", "head_adamw_state", "head_adamw_values", "head_cross_entropy", "head_cross_entropy_grad",
           "head_embed", "head_embed_grad", "head_layer_norm", "head_layer_norm_grad", "LeafHead"]
