"""The trainable head (include/head.h) where its kernels change their ways: sizes at which another kernel, tile or number of
pieces takes over, rows that do not count, states at the ends of their range, and what is refused.

Tolerances are bounds on rounding as in test_head.py, element by element: n float32 terms differ from their exact sum by at most
n * 2^-24 * (sum of their magnitudes), a bfloat16 result by up to 2^-8 of itself more.  References are computed in float64.
"""
import numpy as np
import pytest

import paper_2301_13441_amd as pk

U = 2.0 ** -24
TINY = 1e-37


def _within(got, want, bound, what=""):
    import torch
    off, bound = (got.double() - want).abs(), bound + TINY
    assert got.shape == want.shape, what
    assert (off <= bound).all(), (what, (off / bound).max().item(), torch.nonzero(~(off <= bound))[0].tolist())


def _classes(seed, n, dim, classes, dtype):
    """hidden, weight, bias and targets, a tenth of which are no class."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(n, dim, generator=g, device="cuda").to(dtype)
    w = (torch.randn(classes, dim, generator=g, device="cuda") * dim ** -0.5).to(dtype)
    b = torch.randn(classes, generator=g, device="cuda") * 0.5
    t = torch.randint(0, classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    t[torch.rand(n, generator=g, device="cuda") < 0.1] = -1
    t[n // 2], t[-1] = classes, -7
    return h, w, b, t


# Tiles of 64, 128 and 256; rows and classes that end inside one; operands that are whole in 16 bytes and that are not.
TILES = [("float32", 200, 16, 50), ("float32", 1021, 33, 10), ("float32", 3001, 24, 3003), ("bfloat16", 130, 16, 70), ("bfloat16", 77, 21, 3000),
         ("bfloat16", 2101, 40, 2111), ("bfloat16", 4099, 72, 4200)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,dim,classes", TILES)
def test_cross_entropy_rows_without_a_target_may_hold_anything(dtype, n, dim, classes):
    """Values, grad_loss and lse of rows without a target are read by no gradient: infinities and NaN there change no bit of it."""
    import torch
    h, w, b, t = _classes(n, n, dim, classes, getattr(torch, dtype))
    none = (t < 0) | (t >= classes)
    loss, lse = pk.head_cross_entropy(h, w, t, b)
    gl = torch.rand(n, device="cuda") / n
    h[none], gl[none], lse[none] = 0, 0, 0
    want = pk.head_cross_entropy_grad(gl, h, w, t, lse, b)
    assert all(torch.isfinite(x).all() for x in want) and (want[0][none] == 0).all()
    at = torch.nonzero(none)[:, 0]
    for k, value in enumerate((float("nan"), float("inf"), -float("inf"))):
        h[at[k::3]] = value
        gl[at[k::3]], lse[at[(k + 1) % 3::3]] = value, value
    got = pk.head_cross_entropy_grad(gl, h, w, t, lse, b)
    for x, y, what in zip(got, want, ("grad_hidden", "grad_weight", "grad_bias")):
        assert torch.equal(x, y), what
    loss2, _ = pk.head_cross_entropy(h, w, t, b)
    assert torch.equal(loss, loss2)
    w[classes // 3] = float("nan")                       # rows with a target: NaN; the others have no gradient still
    gh = pk.head_cross_entropy_grad(gl, h, w, t, lse, b)[0]
    assert (gh[none] == 0).all() and torch.isnan(gh[~none]).all()


@pytest.mark.gpu
def test_cross_entropy_of_rows_none_of_which_has_a_target():
    import torch
    for dtype, n, dim, classes in (("float32", 70, 16, 9), ("bfloat16", 4099, 72, 4200)):
        h, w, b, t = _classes(1, n, dim, classes, getattr(torch, dtype))
        t.fill_(-1)
        loss, lse = pk.head_cross_entropy(h, w, t, b)
        assert (loss == 0).all() and torch.isfinite(lse).all()
        for x in pk.head_cross_entropy_grad(torch.ones(n, device="cuda"), h.fill_(float("inf")), w, t, lse, b):
            assert (x == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n,dim,classes", [(4099, 72, 4200), (66_001, 16, 300)])
def test_cross_entropy_rows_without_a_target_have_no_say_in_the_precision(n, dim, classes):
    """bfloat16 in tiles of 256 divides grad_loss by its largest magnitude: that of the rows that count."""
    import torch
    h, w, b, t = _classes(n, n, dim, classes, torch.bfloat16)
    none = (t < 0) | (t >= classes)
    loss, lse = pk.head_cross_entropy(h, w, t, b)
    gl = torch.rand(n, device="cuda") / n
    gl[none] = 0
    want = pk.head_cross_entropy_grad(gl, h, w, t, lse, b)
    gl[none] = 3e38
    for x, y, what in zip(pk.head_cross_entropy_grad(gl, h, w, t, lse, b), want, ("grad_hidden", "grad_weight", "grad_bias")):
        assert torch.equal(x, y), what


@pytest.mark.gpu
@pytest.mark.parametrize("n,dim,classes", [(1, 64, 70_000), (5, 64, 100_000), (255, 24, 66_000), (66_001, 24, 10), (66_001, 24, 255), (500, 40, 3000)])
def test_cross_entropy_of_few_rows_or_classes_keeps_gradients_of_logits_in_16_bits(n, dim, classes):
    """Two bfloat16 planes hold the gradient of a logit to 2^-16 of itself, wherever there are fewer than 256 rows or classes, or few of both."""
    import torch
    h, w, b, t = _classes(n + classes, n, dim, classes, torch.bfloat16)
    t[0] = classes - 1
    has = (t >= 0) & (t < classes)
    h64, w64 = h.double(), w.double()
    logits, size = h64 @ w64.T + b.double(), h64.abs() @ w64.abs().T + b.double().abs()
    lse64 = torch.logsumexp(logits, 1)
    gl = torch.rand(n, device="cuda") / n
    lse = lse64.float()
    got_h, got_w, got_b = pk.head_cross_entropy_grad(gl, h, w, t, lse, b)
    p = torch.exp(logits - lse64[:, None])
    rel = 4 * (dim + 2) * U * size + 2 * U * (lse64.abs()[:, None] + logits.abs()) + 8 * U
    g = (gl.double() * has)[:, None]
    off = g * (2 * p * rel + 4 * U)
    row = torch.nonzero(has)[:, 0]
    p[row, t[row].long()] -= 1
    p *= g
    off += 2.0 ** -16 * p.abs()
    want = p @ w64
    _within(got_h, want, off @ w64.abs() * 1.01 + 4 * (classes + 8) * U * (p.abs() @ w64.abs()) + 2.0 ** -8 * 1.01 * want.abs(), "grad_hidden")
    want = p.T @ h64
    _within(got_w, want, off.T @ h64.abs() * 1.01 + 4 * (n + 8) * U * (p.abs().T @ h64.abs()) + 2.0 ** -8 * 1.01 * want.abs(), "grad_weight")
    _within(got_b, p.sum(0), off.sum(0) + (n + 8) * U * p.abs().sum(0), "grad_bias")
