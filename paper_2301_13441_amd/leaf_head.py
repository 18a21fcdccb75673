"""A linear softmax model over the leaves of a forest: the operators of include/head.h, put together.

The forest turns a row into a leaf of each tree, the head sums the leaves' vectors, normalises the sum and scores
classes.  That refits a forest's answers to other labels, or uses its trees as encoders of the rows; only the head is trained.

    head = LeafHead(forest.tree_offset, n_classes=10, dim=64)
    for X, targets in batches:                    # X: float32 [n, F], targets: int32 [n], both on the device
        loss = head.train_step(model.predict_leaves(X), targets, rate=1e-3)
    probabilities, labels = head.predict(model.predict_leaves(X))

Up to 32 classes a trained head is served by the framework's linear kernels (`predict`); more classes are scored by
`losses` against given targets only.
"""
from __future__ import annotations

from types import SimpleNamespace

from .binding import OUT_BOTH, TRANSFORM_NONE, TRANSFORM_SOFTMAX
from .head_binding import (head_adamw, head_adamw_state, head_cross_entropy, head_cross_entropy_grad, head_embed,
                           head_embed_grad, head_layer_norm, head_layer_norm_grad)
from .linear_binding import linear_load


class LeafHead:
    """Vectors, layer norm and classes over the leaf ids of a forest, with their optimizer's states.

    tree_offset: [n_trees + 1], the first node of each tree, as in the forest that was loaded.  dtype: of activations, of the
    vectors and class weights that the products read and of their gradients, float32 or bfloat16; parameters are float32 in
    either case.  bits: of the optimizer's states, 32 or 8.
    """

    def __init__(self, tree_offset, n_classes: int, dim: int = 64, dtype=None, bits: int = 32, seed: int = 0, device=None):
        import torch
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self.dtype = torch.float32 if dtype is None else dtype
        if self.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"dtype must be float32 or bfloat16, not {self.dtype}")
        offset = torch.as_tensor(tree_offset, dtype=torch.int64)
        self.offsets, self.n_vectors, self.n_classes, self.seed, self.step = offset[:-1].to(device), int(offset[-1]), n_classes, seed, 0
        self.scale = len(self.offsets) ** -0.5
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.vectors = torch.randn(self.n_vectors, dim, generator=g, device=device) * 0.1
        self.norm_weight, self.norm_bias = torch.ones(dim, device=device), torch.zeros(dim, device=device)
        self.weight = torch.randn(n_classes, dim, generator=g, device=device) * dim ** -0.5
        self.bias = torch.zeros(n_classes, device=device)
        self.states = [head_adamw_state(p, bits) for p in self.params()]
        self._copies = None
        if self.dtype == torch.bfloat16:  # what the products read; the small parameters are read as they are
            self._copies = [self.vectors.bfloat16(), None, None, self.weight.bfloat16(), None]

    def params(self):
        return [self.vectors, self.norm_weight, self.norm_bias, self.weight, self.bias]

    def _read(self):
        """The vectors and the class weights as the operators read them."""
        return (self.vectors, self.weight) if self._copies is None else (self._copies[0], self._copies[3])

    def _hidden(self, leaves):
        x = head_embed(self._read()[0], leaves, self.offsets, self.scale)
        return x, *head_layer_norm(x, self.norm_weight, self.norm_bias)

    def losses(self, leaves, targets):
        """The cross entropy of each row, float32 [n_rows]; 0 where the target is no class."""
        return head_cross_entropy(self._hidden(leaves)[1], self._read()[1], targets, self.bias)[0]

    def train_step(self, leaves, targets, rate: float, decay: float = 0.01):
        """One step on the mean loss of the rows that have a target.  leaves: int32 [n_rows, n_trees], -1 where a tree
        is to be left out; targets: int32 [n_rows].  Returns the loss before the step, a tensor of one value."""
        vectors, weight = self._read()
        x, hidden, mean, rstd = self._hidden(leaves)
        loss, lse = head_cross_entropy(hidden, weight, targets, self.bias)
        share = 1.0 / ((targets >= 0) & (targets < self.n_classes)).sum().clamp(min=1).float()
        g_hidden, g_weight, g_bias = head_cross_entropy_grad(share.expand(len(targets)).contiguous(), hidden, weight, targets, lse, self.bias)
        g_x, g_norm_weight, g_norm_bias = head_layer_norm_grad(g_hidden, x, self.norm_weight, mean, rstd)
        g_vectors = head_embed_grad(g_x, leaves, self.n_vectors, self.offsets, self.scale)
        grads = [g_vectors, g_norm_weight, g_norm_bias, g_weight, g_bias]
        self.step += 1
        wide = [k for k, g in enumerate(grads) if g.dtype == grads[1].dtype]  # float32 gradients, and the others
        for call, some in enumerate((wide, [k for k in range(len(grads)) if k not in wide])):
            head_adamw([self.params()[k] for k in some], [grads[k] for k in some], [self.states[k] for k in some], self.step, rate,
                       decay=decay, copies=None if self._copies is None else [self._copies[k] for k in some], seed=2 * self.seed + call)
        return loss.sum() * share

    def linear(self, probabilities: bool = True):
        """The class weights as a linear model of the framework (up to its number of outputs), on the normalised sums."""
        return linear_load(SimpleNamespace(n_features=self.weight.shape[1], n_outputs=self.n_classes,
                                           weight=self.weight.T.cpu().numpy(), bias=self.bias.cpu().numpy(),
                                           transform=TRANSFORM_SOFTMAX if probabilities and self.n_classes > 1 else TRANSFORM_NONE,
                                           output=OUT_BOTH))

    def predict(self, leaves, linear=None):
        """(probabilities, labels) of the rows.  linear: what linear() gave, kept over calls; by default it is made anew."""
        import torch
        if self.n_classes == 1:  # a linear model of one output has a threshold and no softmax
            n = leaves.shape[0]
            return torch.ones(n, 1, device=self.bias.device), torch.zeros(n, dtype=torch.int32, device=self.bias.device)
        made = linear is None
        linear = self.linear() if made else linear
        try:
            return linear.predict(self._hidden(leaves)[1].float())
        finally:
            if made:
                torch.cuda.current_stream().synchronize()  # the weights go with the handle
                linear.close()
