"""The head's layers (head_linear, head_gated, their gradients), head_clip, and a head with residual blocks: checks of arguments that need no GPU,
and the operators on the GPU against their definitions in float64, computed here with numpy.

Tolerances are bounds on rounding, element by element.  A float32 sum of n terms in any order is off by at most n * 2^-24 * (sum of their
magnitudes), and by two more where a bias is added or parts are joined; a rounding to bfloat16 by 2^-8 of the value.  Activations of
float32 values: exp and erfc to a few units, of arguments that are themselves rounded, which the function turns into x^2 units
(x exp(-x^2 / 2)); 2^-24 * (16 + 2 x^2) of the value covers them, and 2^-19 their slopes (at most 1.13, of terms below 1.5 whose errors
are 16 units at most).  Of bfloat16 values both are right to 2^-13, as head.h says; slopes are at most 1.13, so z's error counts 1.13 times in y.
"""
import math

import numpy as np
import pytest

import paper_2301_13441_amd as pk
from paper_2301_13441_amd import head_binding as hb

U = 2.0 ** -24
TINY = 1e-37
DTYPES = ["float32", "bfloat16"]
ACTS = [None, "relu", "gelu", "silu"]


def _ulp(dtype):
    return 2.0 ** -8 if dtype == "bfloat16" else U


def _torch(a, dtype=None):
    import torch
    t = torch.from_numpy(np.array(a)).cuda()
    return t if dtype is None else t.to(getattr(torch, dtype))


def _np(t):
    return t.detach().double().cpu().numpy()


def _close(got, want, bound, what=""):
    got, bound = _np(got), np.broadcast_to(np.asarray(bound) + TINY, np.shape(want))
    assert got.shape == np.shape(want), what
    off = np.abs(got - want)
    worst = np.unravel_index(np.argmax(off / bound), off.shape) if off.size else None
    assert off.size == 0 or (off <= bound).all(), (what, worst, got[worst], np.asarray(want)[worst], bound[worst])


def _rows(rng, n, dim, dtype, spread=0, shift=0, scale=1.0):
    """(device tensor, float64 array) of [n, dim] values, its rows `spread` elements further apart than they are long and
    beginning `shift` elements into their memory."""
    whole = _torch(rng.standard_normal((n, dim + spread + shift)).astype(np.float32) * np.float32(scale), dtype)
    t = whole[:, shift:shift + dim] if spread or shift else whole
    return t, _np(t)


def _act(name, x):
    from scipy.special import erfc
    if name == "silu":
        return x / (1 + np.exp(-x))
    if name == "gelu":
        return x * erfc(-x / math.sqrt(2)) / 2
    return np.maximum(x, 0) if name == "relu" else x


def _slope(name, x):
    from scipy.special import erfc
    if name == "silu":
        s = 1 / (1 + np.exp(-x))
        return s + x * s * (1 - s)
    if name == "gelu":
        return erfc(-x / math.sqrt(2)) / 2 + x * np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    return (x > 0).astype(float) if name == "relu" else np.ones_like(x)


def _act_off(name, x, dtype):
    """How far the activation of x may be off, next to that of x exactly."""
    if name in (None, "relu"):
        return 0
    return np.abs(_act(name, x)) * (2.0 ** -13 if dtype == "bfloat16" else U * (16 + 2 * x * x))


def _slope_off(name, dtype):
    return 0 if name in (None, "relu") else 2.0 ** -13 if dtype == "bfloat16" else 2.0 ** -19


def _z(x, w, b):
    """z and how far a float32 sum may be from it."""
    z, magnitude = x @ w.T, np.abs(x) @ np.abs(w).T
    if b is not None:
        z, magnitude = z + b, magnitude + np.abs(b)
    return z, (x.shape[1] + 64) * U * magnitude


def _check_z(z, off, got, dtype, what):
    _close(got, z, off * (1 + _ulp(dtype)) + _ulp(dtype) * np.abs(z), what)


# ---------------------------------------------------------------- no GPU needed

def _layer(dtype=0, act=0, n=4, dim=8, outs=5, x=64, xs=8, w=64, ws=8, b=64):
    return hb._Layer(dtype, act, n, dim, outs, x, xs, w, ws, b)


def test_layers_refuse_bad_arguments_before_any_device_call():
    lib = hb._lib()

    def linear(d, residual=64, rs=5, y=64, z=64, work=64):
        return lib.head_linear(d, residual, rs, 1.0, y, z, work, None)

    def linear_grad(d, z=64, zs=5, g=64, gs=5, gx=64, gw=64, gb=64, work=64):
        return lib.head_linear_grad(d, z, zs, g, gs, 1.0, gx, gw, gb, work, None)

    def gated(d, y=64, z=64, work=64):
        return lib.head_gated(d, y, z, work, None)

    def gated_grad(d, z=64, zs=10, g=64, gs=5, gx=64, gw=64, gb=64, work=64):
        return lib.head_gated_grad(d, z, zs, g, gs, gx, gw, gb, work, None)

    for f in (linear, linear_grad, gated, gated_grad):
        assert f(None) == -1
        for bad in (dict(dtype=2), dict(dtype=-1), dict(act=-1), dict(act=4), dict(n=-1), dict(dim=0), dict(outs=0), dict(x=None), dict(x=66),
                    dict(xs=7), dict(w=None), dict(w=66), dict(ws=7), dict(b=66)):
            assert f(_layer(**bad)) == -1, bad
        for far in (dict(dim=16385), dict(n=10 ** 9 + 1), dict(outs=10 ** 9 + 1), dict(n=10 ** 9, outs=17_593)):
            assert f(_layer(**far)) == -7, far
    for f in (gated, gated_grad):
        assert f(_layer(outs=500_000_001)) == -7
    for f in (linear_grad, gated_grad):
        assert f(_layer(outs=262_145)) == -7
    for f in (linear, gated):
        assert f(_layer(), y=None) == f(_layer(), y=66) == f(_layer(), z=66) == -1
        odd = _layer(dtype=1, n=100, dim=7, xs=7, ws=7)  # rows at odd addresses, which are copied
        assert f(odd, work=None) == f(odd, work=72) == -1
        assert f(_layer(n=0, x=None), y=None, work=None) == 0
    assert linear(_layer(), residual=66) == linear(_layer(), rs=4) == -1
    for f, zs in ((linear_grad, 5), (gated_grad, 10)):
        a = _layer(act=3)
        assert f(a, z=None) == f(a, z=66) == f(a, zs=zs - 1) == f(a, g=None) == f(a, g=66) == f(a, gs=4) == -1
        assert f(a, gx=None) == f(a, gx=66) == f(a, gw=None) == f(a, gw=66) == f(a, gb=66) == f(a, work=None) == f(a, work=72) == -1
        assert f(_layer(n=0, x=None), gw=None) == -1
    assert gated_grad(_layer(), z=None) == -1  # the values are needed whatever the activation is
    for name in ("linear", "gated"):
        assert getattr(lib, f"head_{name}_grad_bytes")(_layer()) > 0
        assert getattr(lib, f"head_{name}_bytes")(_layer(n=0)) == getattr(lib, f"head_{name}_grad_bytes")(_layer(n=0)) == 0
        assert getattr(lib, f"head_{name}_bytes")(_layer(dtype=1, n=100, dim=7, xs=7, ws=7)) > 0


def test_clip_refuses_bad_arguments_before_any_device_call():
    lib = hb._lib()

    def call(grad=64, out=64, n=10, dtype=0, count=1, limit=1.0, norm=64, work=64, more=()):
        rows = [hb._ClipTensor(grad, out, n, dtype), *more]
        return lib.head_clip((hb._ClipTensor * len(rows))(*rows), count + len(more), limit, norm, work, None)

    for bad in (dict(grad=None), dict(grad=66), dict(out=66), dict(n=-1), dict(dtype=2), dict(count=-1), dict(limit=0.0), dict(limit=-1.0),
                dict(limit=math.nan), dict(norm=None), dict(norm=66), dict(n=10 ** 6, work=None), dict(n=10 ** 6, work=72)):
        assert call(**bad) == -1, bad
    assert call(more=[hb._ClipTensor(64, None, 10, 0)]) == -1  # some with a result and some without
    assert call(n=2 ** 40 + 1) == call(count=1_000_001) == -7
    assert lib.head_clip(None, 1, 1.0, 64, 64, None) == lib.head_clip_bytes(None, 1) == -1
    assert lib.head_clip_bytes(None, 0) >= 0  # there is a norm of nothing


def test_python_refuses_what_no_layer_is():
    import torch
    x, w = torch.zeros(3, 8), torch.zeros(4, 8)
    for call in (lambda: pk.head_linear(x, w), lambda: pk.head_gated(x, w), lambda: pk.head_linear_grad(x, x, w), lambda: pk.head_gated_grad(x, x, w, x),
                 lambda: pk.head_clip([x], 1.0), lambda: pk.head_clip([x], 1.0, in_place=True)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    for call in (lambda: pk.head_linear(x, w, activation="tanh"), lambda: pk.head_gated(x, w, activation=[]),
                 lambda: pk.head_linear_grad(x, x, w, activation="none"), lambda: pk.head_gated_grad(x, x, w, x, activation=1)):
        with pytest.raises(ValueError, match="activation must be one of"):
            call()
    with pytest.raises(ValueError, match="no tensors"):
        pk.head_clip([], 1.0)
    for limit in (0.0, -1.0, math.nan):
        with pytest.raises(ValueError, match="above 0"):
            pk.head_clip([x], limit)


# ---------------------------------------------------------------- layers

# rows, dim, outs: one value; few rows, either side of 16, 32 and 64; sums cut into parts; rows and columns at the ends of tiles of 64, 128
# and 256; widths that are whole in 16 bytes and not
SHAPES = [(1, 1, 1), (1, 64, 256), (5, 90, 31), (16, 8, 17), (17, 129, 16), (33, 1024, 40), (64, 257, 100), (65, 2048, 8), (100, 31, 65),
          (129, 16, 300), (700, 1000, 72), (515, 90, 331), (2049, 64, 1025), (1024, 320, 2304)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,dim,outs", SHAPES)
def test_linear(n, dim, outs, dtype):
    import torch
    rng = np.random.default_rng(n + dim + outs)
    for k, act in enumerate(ACTS):
        # rows apart from each other and not aligned; bias, residual and z there and not
        (x, x64) = _rows(rng, n, dim, dtype, *((3, 1) if k == 1 else (8, 8) if k == 3 else ()))
        (w, w64) = _rows(rng, outs, dim, dtype, *((5, 0) if k == 2 else ()), scale=dim ** -0.5)
        b = rng.standard_normal(outs).astype(np.float32) if k % 2 else None
        (r, r64), scale = (_rows(rng, n, outs, dtype, *((1, 1) if k == 3 else ())), 0.75) if k > 1 else ((None, 0), 1.0)
        got = pk.head_linear(x, w, None if b is None else _torch(b), act, r, scale, keep=k != 1)
        z64, z_off = _z(x64, w64, None if b is None else b.astype(np.float64))
        if k != 1:
            got, z = got
            assert z.dtype == x.dtype
            _check_z(z64, z_off, z, dtype, ("z", act))
        want = scale * _act(act, z64) + r64
        off = scale * (1.13 * z_off + _act_off(act, z64, dtype)) + 4 * U * (np.abs(scale * _act(act, z64)) + np.abs(r64))
        assert got.dtype == x.dtype
        _close(got, want, off * (1 + _ulp(dtype)) + _ulp(dtype) * np.abs(want), ("y", act))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,dim,outs", SHAPES)
def test_gated(n, dim, outs, dtype):
    rng = np.random.default_rng(n + dim + outs)
    for k, act in enumerate(ACTS):
        (x, x64), (w, w64) = _rows(rng, n, dim, dtype, *((3, 1) if k == 1 else ())), _rows(rng, 2 * outs, dim, dtype, *((8, 8) if k == 2 else ()), scale=dim ** -0.5)
        b = rng.standard_normal(2 * outs).astype(np.float32) if k % 2 else None
        got = pk.head_gated(x, w, None if b is None else _torch(b), act, keep=k != 1)
        z64, z_off = _z(x64, w64, None if b is None else b.astype(np.float64))
        if k != 1:
            got, z = got
            _check_z(z64, z_off, z, dtype, ("z", act))
        (gate, value), (gate_off, value_off) = np.split(z64, 2, 1), np.split(z_off, 2, 1)
        a, a_off = _act(act, gate), 1.13 * gate_off + _act_off(act, gate, dtype)
        want = a * value
        off = a_off * np.abs(value) + (np.abs(a) + a_off) * value_off + 4 * U * np.abs(want)
        assert got.dtype == x.dtype
        _close(got, want, off * (1 + _ulp(dtype)) + _ulp(dtype) * np.abs(want), ("y", act))


def _check_grads(got, x, w, dz, dz_off, scale, dtype, what):
    """Gradients of x, weight and bias from dz, of which the products see dz_off less or more, and the rounding of their type."""
    grad_x, grad_w, grad_b = got
    b_off = scale * (dz_off.sum(0) + (len(dz) + 64) * U * np.abs(dz).sum(0))
    if grad_b is not None:
        _close(grad_b, scale * dz.sum(0), b_off + 2 * U * np.abs(scale * dz.sum(0)), (what, "bias"))
    dz_off = dz_off + _ulp(dtype) * (np.abs(dz) + dz_off)
    size = np.abs(dz) + dz_off
    for g, want, off, magnitude, n in ((grad_x, dz @ w, dz_off @ np.abs(w), size @ np.abs(w), dz.shape[1]),
                                       (grad_w, dz.T @ x, dz_off.T @ np.abs(x), size.T @ np.abs(x), len(dz))):
        off = abs(scale) * (off + (n + 64) * U * magnitude)
        want = scale * want
        _close(g, want, off * (1 + _ulp(dtype)) + (_ulp(dtype) + 2 * U) * np.abs(want), (what, "x" if g is grad_x else "weight"))


GRAD_SHAPES = [(1, 1, 1), (1, 64, 256), (3, 90, 31), (17, 129, 16), (64, 40, 1030), (65, 2048, 8), (129, 16, 300), (515, 90, 331), (5001, 24, 10),
               (2049, 64, 514), (1024, 300, 264)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,dim,outs", GRAD_SHAPES)
def test_linear_gradient(n, dim, outs, dtype):
    rng = np.random.default_rng(n + dim + outs)
    for k, act in enumerate(ACTS):
        (x, x64), (w, w64) = _rows(rng, n, dim, dtype, *((3, 1) if k == 1 else ())), _rows(rng, outs, dim, dtype, *((5, 0) if k == 2 else ()), scale=dim ** -0.5)
        (g, g64), (z, z64) = _rows(rng, n, outs, dtype, *((3, 0) if k in (0, 3) else ()), scale=0.1), _rows(rng, n, outs, dtype, *((8, 8) if k == 2 else ()), scale=2)
        scale = 0.75 if k % 2 else 1.0
        got = pk.head_linear_grad(g, x, w, None if act is None else z, act, scale, bias=k != 2)
        assert (got[2] is None) == (k == 2) and got[0].dtype == got[1].dtype == x.dtype
        dz = g64 * _slope(act, z64)
        off = np.abs(g64) * (_slope_off(act, dtype) + 2 * U * np.abs(_slope(act, z64)))
        _check_grads(got, x64, w64, dz, off, scale, dtype, act)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,dim,outs", GRAD_SHAPES)
def test_gated_gradient(n, dim, outs, dtype):
    rng = np.random.default_rng(n + dim + outs)
    for k, act in enumerate(ACTS):
        (x, x64), (w, w64) = _rows(rng, n, dim, dtype, *((3, 1) if k == 1 else ())), _rows(rng, 2 * outs, dim, dtype, *((5, 0) if k == 2 else ()), scale=dim ** -0.5)
        (g, g64), (z, z64) = _rows(rng, n, outs, dtype, *((3, 0) if k == 3 else ()), scale=0.1), _rows(rng, n, 2 * outs, dtype, *((8, 8) if k == 2 else ()), scale=2)
        got = pk.head_gated_grad(g, x, w, z, act, bias=k != 2)
        gate, value = np.split(z64, 2, 1)
        dz = np.concatenate([g64 * value * _slope(act, gate), g64 * _act(act, gate)], 1)
        off = np.concatenate([np.abs(g64 * value) * (_slope_off(act, dtype) + 4 * U * np.abs(_slope(act, gate))),
                              np.abs(g64) * (_act_off(act, gate, dtype) + 2 * U * np.abs(_act(act, gate)))], 1)
        _check_grads(got, x64, w64, dz, off, 1.0, dtype, act)


@pytest.mark.gpu
@pytest.mark.parametrize("n,dim,outs", [(4100, 64, 4200), (300, 40, 60_001), (70, 24, 262_144), (8300, 2100, 300), (2048, 2100, 2056)])
def test_layers_in_large_tiles(n, dim, outs):
    """bfloat16, sampled rows and columns of products that fill the device."""
    import torch
    rng = np.random.default_rng(n)
    dtype = "bfloat16"
    x, w = _rows(rng, n, dim, dtype)[0], _rows(rng, 2 * (outs // 2), dim, dtype, scale=dim ** -0.5)[0]
    outs = w.shape[0]
    b = _torch(rng.standard_normal(outs).astype(np.float32))
    r, g = _rows(rng, n, outs, dtype)[0], _rows(rng, n, outs, dtype, scale=0.1)[0]
    rows, columns = np.unique(np.r_[0, n - 1, rng.integers(0, n, 40)]), np.unique(np.r_[0, outs // 2 - 1, rng.integers(0, outs // 2, 40)])
    x64, w64, b64 = _np(x), _np(w), _np(b)
    y, z = pk.head_linear(x, w, b, "gelu", r, 0.5, keep=True)
    z64, z_off = _z(x64[rows], w64, b64)
    _check_z(z64, z_off, z[rows], dtype, "z")
    want = 0.5 * _act("gelu", z64) + _np(r[rows])
    off = 0.5 * (1.13 * z_off + _act_off("gelu", z64, dtype)) + 4 * U * (np.abs(want) + 2 * np.abs(_np(r[rows])))
    _close(y[rows], want, off * (1 + _ulp(dtype)) + _ulp(dtype) * np.abs(want), "y")
    h, z2 = pk.head_gated(x, w, b, "silu", keep=True)
    _check_z(z64, z_off, z2[rows], dtype, "gated z")
    (gate, value), (gate_off, value_off) = np.split(z64, 2, 1), np.split(z_off, 2, 1)
    a, a_off = _act("silu", gate), 1.13 * gate_off + _act_off("silu", gate, dtype)
    off = a_off * np.abs(value) + (np.abs(a) + a_off) * value_off + 4 * U * np.abs(a * value)
    _close(h[rows], a * value, off * (1 + _ulp(dtype)) + _ulp(dtype) * np.abs(a * value), "h")
    # the gradients: rows of grad_x and of grad_weight
    for gated in (False, True):
        gr = g[:, :outs // 2].contiguous() if gated else g
        got = pk.head_gated_grad(gr, x, w, z2, "silu") if gated else pk.head_linear_grad(gr, x, w, z, "gelu", 0.5)
        g64, zz, scale = _np(gr), _np(z2 if gated else z), 1.0 if gated else 0.5
        if gated:
            gate, value = np.split(zz, 2, 1)
            dz = np.concatenate([g64 * value * _slope("silu", gate), g64 * _act("silu", gate)], 1)
            off = np.concatenate([np.abs(g64 * value) * (2.0 ** -13 + 8 * U), np.abs(g64) * (_act_off("silu", gate, dtype) + 2 * U * np.abs(_act("silu", gate)))], 1)
        else:
            dz = g64 * _slope("gelu", zz)
            off = np.abs(g64) * (2.0 ** -13 + 4 * U)
        off_b = scale * (off.sum(0) + (n + 64) * U * np.abs(dz).sum(0))
        _close(got[2], scale * dz.sum(0), off_b + 2 * U * np.abs(dz.sum(0)), "bias")
        off = off + _ulp(dtype) * (np.abs(dz) + off)
        pick = np.r_[columns, columns + outs // 2]
        for t, a, b_, o, m in ((got[0][rows], dz[rows], w64, off[rows], outs), (got[1][pick], dz[:, pick].T, x64, off[:, pick].T, n)):
            want = scale * (a @ b_)
            bound = scale * (o @ np.abs(b_) + (m + 64) * U * ((np.abs(a) + o) @ np.abs(b_)))
            _close(t, want, bound * (1 + _ulp(dtype)) + (_ulp(dtype) + 2 * U) * np.abs(want), ("gated" if gated else "linear", m))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_layers_of_no_rows(dtype):
    import torch
    x, w, b = (torch.ones(s, device="cuda", dtype=getattr(torch, dtype)) for s in ((0, 8), (6, 8), (6,)))
    b = b.float()
    y, z = pk.head_linear(x, w, b, "silu", keep=True)
    assert y.shape == z.shape == (0, 6)
    y, z = pk.head_gated(x, w, b, keep=True)
    assert y.shape == (0, 3) and z.shape == (0, 6)
    for grads in (pk.head_linear_grad(x.new_empty(0, 6), x, w, x.new_empty(0, 6), "silu"), pk.head_gated_grad(x.new_empty(0, 3), x, w, x.new_empty(0, 6))):
        assert grads[0].shape == (0, 8) and not grads[1].any() and not grads[2].any() and grads[1].shape == (6, 8) and grads[2].shape == (6,)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,dim,outs", [(9, 70, 33), (200, 70, 33), (700, 1000, 72)])
def test_layers_keep_infinities_and_nan_to_their_rows(n, dim, outs, dtype):
    import torch
    rng = np.random.default_rng(0)
    x, w = _rows(rng, n, dim, dtype)[0], _rows(rng, 2 * outs, dim, dtype, scale=dim ** -0.5)[0]
    clean = [pk.head_linear(x, w, None, "gelu"), pk.head_gated(x, w)]
    bad = x.clone()
    bad[1, 3], bad[n - 1, dim - 1], bad[4, 0] = math.nan, math.inf, -math.inf
    got = [pk.head_linear(bad, w, None, "gelu"), pk.head_gated(bad, w)]
    others = [r for r in range(n) if r not in (1, 4, n - 1)]
    for a, b in zip(got, clean):
        assert torch.equal(a[others], b[others])
        assert a[1].isnan().all() and not a[n - 1].isfinite().all()
    # an infinite value in a column of z where relu stops it
    z = _rows(rng, n, outs, dtype)[0]
    g, wl = _rows(rng, n, outs, dtype)[0], w[:outs]
    z[:, 2] = -math.inf
    gx, gw, gb = pk.head_linear_grad(g, x, wl, z, "relu")
    assert not gw[2].any() and gb[2] == 0 and gx.isfinite().all()
    g[:, 2] = math.inf
    assert all(torch.equal(a, b) for a, b in zip(pk.head_linear_grad(g, x, wl, z, "relu"), (gx, gw, gb)))


@pytest.mark.gpu
@pytest.mark.parametrize("n,dim,outs", [(20, 96, 70), (130, 96, 70), (700, 200, 700)])
def test_float32_products_over_the_range(n, dim, outs):
    """Values far from 1, subnormal ones and the largest: float32 sums are as near as near 1."""
    import torch
    rng = np.random.default_rng(dim)
    x0, w0 = rng.standard_normal((n, dim)).astype(np.float32), rng.standard_normal((2 * outs, dim)).astype(np.float32)
    for up, down in ((-100, 100), (-100, 0), (60, 60), (120, -120), (-60, -40)):
        x, w = x0 * np.float32(2.0 ** up), w0 * np.float32(2.0 ** down)
        z, off = _z(x.astype(np.float64), w.astype(np.float64), None)
        # below 2^-109 what is below 2^-133 of a value may be lost, times the other's magnitude
        off = off + 2.0 ** -133 * (np.abs(w).astype(np.float64).sum(1)[None, :] + np.abs(x).astype(np.float64).sum(1)[:, None])
        _close(pk.head_linear(_torch(x), _torch(w)), z, off + 2.0 ** -149, (up, down))
    # the largest values have no bfloat16 near them
    x, w = x0.copy(), w0 * np.float32(1e-30)
    x[n - 1, 5], x[3, dim - 1] = 3.4e38, -3.402e38
    z, off = _z(x.astype(np.float64), w.astype(np.float64), None)
    got, kept = pk.head_gated(_torch(x), _torch(w), None, None, keep=True)
    _check_z(z, off, kept, "float32", "largest")
    g = rng.standard_normal((n, 2 * outs)).astype(np.float32)
    gx, gw, gb = pk.head_linear_grad(_torch(g), _torch(x), _torch(w))
    # 3.4e38 times a gradient past 1 is past the largest float32, 3.4028e38: its sum is infinite, in any order, as the other terms
    # are below 1e31 of it.  Where it is within 1e-4 of the largest, either is right.
    want, largest = g.astype(np.float64).T @ x.astype(np.float64), float(np.finfo(np.float32).max)
    past, near = np.abs(want) * (1 - 1e-4) > largest, np.abs(want) * (1 + 1e-4) > largest
    assert past.any() and (_np(gw)[past] == np.sign(want[past]) * math.inf).all()
    gw = torch.where(torch.from_numpy(near).cuda(), torch.from_numpy(want).cuda(), gw.double())
    _check_grads((gx, gw, gb), x.astype(np.float64), w.astype(np.float64), g.astype(np.float64), np.zeros_like(g, dtype=np.float64), 1.0, "float32", "largest")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,dim,outs", [(9, 70, 33), (70, 66, 40), (700, 200, 72)])
def test_layers_read_nothing_between_rows(n, dim, outs, dtype):
    """Rows that lie apart, with NaN between them and behind the last, give what rows that lie together give."""
    import torch
    rng = np.random.default_rng(n)
    kept = [_rows(rng, r, c, dtype)[0] for r, c in ((n, dim), (2 * outs, dim), (n, 2 * outs), (n, outs))]
    x, w, g, half = kept
    nan = lambda t, to: torch.cat([t, t.new_full((len(t), to - t.shape[1]), math.nan)], 1)[:, :t.shape[1]]  # noqa: E731
    for to in (1, 2, 64):
        ax, aw, ag, ahalf = (nan(t, t.shape[1] + to) for t in kept)
        y, z = pk.head_gated(x, w, keep=True)
        for a, b in ((pk.head_linear(ax, aw), pk.head_linear(x, w)), (pk.head_gated(ax, aw), y), (pk.head_linear_grad(ag, ax, aw), pk.head_linear_grad(g, x, w)),
                     (pk.head_gated_grad(ahalf, ax, aw, nan(z, 2 * outs + to)), pk.head_gated_grad(half, x, w, z))):
            for p, q in zip(*((t,) if torch.is_tensor(t) else t for t in (a, b))):
                off = (p.double() - q.double()).abs().max()  # another alignment may sum in another order
                assert off <= (1e-4 if dtype == "float32" else 2e-2) * q.double().abs().max()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,dim,outs", [(9, 70, 33), (200, 70, 33), (700, 1000, 72), (300, 64, 700)])
def test_infinite_values_have_their_sign(n, dim, outs, dtype):
    rng = np.random.default_rng(8)
    x, w = _rows(rng, n, dim, dtype)[0], _rows(rng, 2 * outs, dim, dtype)[0]
    x[2, 3], x[n - 1, dim - 1] = math.inf, -math.inf
    w[1, 0] = -math.inf
    with np.errstate(invalid="ignore"):
        want = _np(x) @ _np(w).T
    for got in (pk.head_linear(x, w), pk.head_gated(x, w, None, None, keep=True)[1]):
        got = _np(got)
        assert (np.isnan(got) == np.isnan(want)).all() and (got[np.isinf(want)] == want[np.isinf(want)]).all() and (np.isinf(got) == np.isinf(want)).all()
    gx, gw, _ = pk.head_linear_grad(x[:, :1].expand(n, 2 * outs).contiguous() * 0 + 1, x, w)
    assert (np.isinf(_np(gx)) == np.isinf(_np(w).sum(0))[None, :]).all()
    column = _np(gw)[0]
    assert column[3] == math.inf and column[dim - 1] == -math.inf and np.isfinite(np.delete(column, [3, dim - 1])).all()


@pytest.mark.gpu
def test_relu_and_its_slope_at_the_border():
    import torch
    x = torch.tensor([[0.0], [-0.0], [1e-30], [-1e-30], [math.nan]], device="cuda")
    one = torch.ones(1, 1, device="cuda")
    y = pk.head_linear(x, one, None, "relu")
    assert y[:4, 0].tolist() == [0, 0, x[2, 0].item(), 0] and y[4].isnan().all()
    gx = pk.head_linear_grad(torch.ones_like(x), x, one, x, "relu")[0]
    assert gx[:4, 0].tolist() == [0, 0, 1, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_activations_over_their_range(dtype):
    """Every binade of z, both signs, through a layer whose product is z itself."""
    import torch
    x64 = np.concatenate([s * np.concatenate([2.0 ** np.linspace(-30, 6.6, 4000), np.linspace(0, 14, 4000)]) for s in (1, -1)])
    x = _torch(x64.astype(np.float32), dtype)[:, None].contiguous()
    x64 = _np(x)
    one = torch.ones(1, 1, device="cuda", dtype=x.dtype)
    for act in ACTS:
        want = _act(act, x64)
        # results below 2^-126 may be zero, and a factor of 2^-126 below 1 with them
        _close(pk.head_linear(x, one, None, act), want, _act_off(act, x64, dtype) + _ulp(dtype) * np.abs(want) + 2.0 ** -118, act)
        got = pk.head_linear_grad(torch.ones_like(x), x, one, x, act)[0]
        want = _slope(act, x64)
        _close(got, want, _slope_off(act, dtype) * (1 + _ulp(dtype)) + 2 * _ulp(dtype) * np.abs(want), (act, "slope"))


@pytest.mark.gpu
def test_layers_past_32_bits():
    """More than 2^31 values in x, z and y, and in the gradient of z."""
    import torch
    n, dim, outs = 70_000_003, 8, 32
    x = torch.zeros(n, dim, device="cuda", dtype=torch.bfloat16)
    g = torch.zeros(n, outs, device="cuda", dtype=torch.bfloat16)
    rng = np.random.default_rng(5)
    at = [0, 1, n // 2, n - 2, n - 1]
    x[at], g[at] = _rows(rng, 5, dim, "bfloat16")[0], _rows(rng, 5, outs, "bfloat16")[0]
    w = _rows(rng, outs, dim, "bfloat16")[0]
    y, z = pk.head_linear(x, w, None, "silu", keep=True)
    small, small_z = pk.head_linear(x[at], w, None, "silu", keep=True)
    assert torch.equal(z[at], small_z) and torch.equal(y[at], small)
    assert not y[2:1000].any() and not y[n // 2 + 1:n - 2].any()
    gx, gw, gb = pk.head_linear_grad(g, x, w, z, "silu")
    sx, sw, sb = pk.head_linear_grad(g[at], x[at], w, z[at], "silu")
    assert torch.equal(gx[at], sx) and not gx[n // 2 + 1:n - 2].any()
    # the same five terms in another order
    assert ((gw.double() - sw.double()).abs() <= (2.0 ** -8 + 16 * U) * sw.double().abs() + 16 * U * 5 * 10).all()
    assert ((gb - sb).abs() <= 16 * U * 5 * 5).all()


@pytest.mark.gpu
def test_layer_gradients_agree_with_differences():
    """Central differences of sum(weights * y) in float64 through the formulas, whose forward the kernels were compared with."""
    rng = np.random.default_rng(3)
    n, dim, outs = 7, 12, 9
    x, w, b, c = rng.standard_normal((n, dim)), rng.standard_normal((2 * outs, dim)) * 0.4, rng.standard_normal(2 * outs) * 0.1, rng.standard_normal((n, outs))

    def f(x, w, b, act, gated):
        z = x @ w.T + b
        return (c * (_act(act, z[:, :outs]) * z[:, outs:] if gated else 0.5 * _act(act, z))).sum()

    for gated in (True, False):
        ww, bb = (w, b) if gated else (w[:outs], b[:outs])
        for act in ("gelu", "silu", None):
            tx, tw, tb, tc = (_torch(a.astype(np.float32)) for a in (x, ww, bb, c))
            _, z = pk.head_gated(tx, tw, tb, act, keep=True) if gated else pk.head_linear(tx, tw, tb, act, keep=True)
            got = pk.head_gated_grad(tc, tx, tw, z, act) if gated else pk.head_linear_grad(tc, tx, tw, z, act, 0.5)
            for which, t in enumerate((x, ww, bb)):
                for _ in range(12):
                    i = tuple(rng.integers(0, s) for s in t.shape)
                    ends = []
                    for h in (1e-5, -1e-5):
                        moved = [x.copy(), ww.copy(), bb.copy()]
                        moved[which][i] += h
                        ends.append(f(*moved, act, gated))
                    # differences: h^2 times third derivatives (10 of 1e2 terms) and 1e-16 * 1e2 / h; float32: 1e2 terms of size 10
                    assert abs((ends[0] - ends[1]) / 2e-5 - _np(got[which])[i]) < 1e-7 + 1e3 * U * 10, (gated, act, which, i)


# ---------------------------------------------------------------- clipping

def _clip64(arrays, limit):
    norm = math.sqrt(sum((a * a).sum() for a in arrays))
    return norm, [a * min(1.0, limit / norm) if norm else a for a in arrays]


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("shapes", [[(1,)], [(3,), (0,), (5, 7)], [(4096,), (4097,), (8191, 3)], [(k % 50 + 1,) for k in range(150)], [(40_960,)], [(40_000,), (961,)],
                                    [(300_001, 33), (10,)]])
def test_clip(shapes, in_place):
    import torch
    rng = np.random.default_rng(len(shapes))
    for k, share in enumerate((0.5, 2.0, 1e-3)):
        grads = [_torch((rng.standard_normal(s) * 1e-3).astype(np.float32), DTYPES[(i + k) % 2]) for i, s in enumerate(shapes)]
        if k == 2:  # not aligned
            grads = [torch.cat([g.new_zeros(1), g.reshape(-1)])[1:].reshape(g.shape) for g in grads]
        arrays = [_np(g) for g in grads]
        limit = share * _clip64(arrays, 1.0)[0]
        want_norm, want = _clip64(arrays, limit)
        before = [g.clone() for g in grads]
        norm, got = pk.head_clip(grads, limit, in_place=in_place)
        assert norm.shape == () and norm.dtype == torch.float32 and len(got) == len(grads)
        # 8 squares in float32 are off by 8 U of their sum at most (a product and seven sums), the root of the whole by half of that, and it is rounded
        assert abs(norm.item() - want_norm) <= 5 * U * want_norm
        for g, o, b, w in zip(grads, got, before, want):
            assert o.dtype == g.dtype and o.shape == g.shape
            assert (o is g) == in_place and (in_place or torch.equal(g, b))
            assert share < 1 or torch.equal(o, b)
            _close(o, w, (_ulp("bfloat16" if g.dtype == torch.bfloat16 else "float32") + 4 * U) * np.abs(w), g.shape)


@pytest.mark.gpu
def test_clip_of_large_and_small_magnitudes_infinities_and_nan():
    import torch
    g = torch.full((1000,), 1e30, device="cuda")
    norm, (got,) = pk.head_clip([g], 1.0)
    assert abs(norm.item() / (1e30 * math.sqrt(1000)) - 1) < 1e-6 and abs(got[0].item() * math.sqrt(1000) - 1) < 1e-6
    norm, (got,) = pk.head_clip([g * 1e-60], 1.0)
    assert norm.item() == 0 and torch.equal(got, g * 1e-60)
    small = torch.full((10_000,), 1e-30, device="cuda")
    norm, (got,) = pk.head_clip([small], 1e-29)
    assert abs(norm.item() / 1e-28 - 1) < 1e-6 and abs(got[5].item() / 1e-31 - 1) < 1e-6
    norm, (got,) = pk.head_clip([torch.full((10,), 3e38, device="cuda")], 1.0)  # a norm that float32 does not hold
    assert norm.item() == math.inf and abs(got[0].item() * math.sqrt(10) - 1) < 1e-6
    norm, (got,) = pk.head_clip([torch.tensor([1.0, math.inf], device="cuda")], 1.0)
    assert norm.item() == math.inf and got[0].item() == 0 and got[1].isnan()
    a, b = torch.tensor([1.0, math.nan], device="cuda"), torch.ones(70_000, device="cuda", dtype=torch.bfloat16)
    norm, got = pk.head_clip([a, b], 1.0)
    assert norm.isnan() and all(t.isnan().all() for t in got)
    norm, got = pk.head_clip([a, b], math.inf)
    assert norm.isnan() and torch.equal(got[1], b) and got[0][0] == 1
    norm, got = pk.head_clip([torch.zeros(5, device="cuda")], 1e-3)
    assert norm.item() == 0 and not got[0].any()
    norm, got = pk.head_clip([torch.zeros(0, device="cuda")], 1.0)
    assert norm.item() == 0 and got[0].shape == (0,)


@pytest.mark.gpu
def test_clip_of_more_values_than_32_bits_count_and_of_very_many_tensors():
    import torch
    g = torch.full((2 ** 31 + 70_001,), 0.5, device="cuda", dtype=torch.bfloat16)
    norm, _ = pk.head_clip([g], 1.0, in_place=True)
    want = 0.5 * math.sqrt(2 ** 31 + 70_001)
    assert abs(norm.item() / want - 1) < 1e-6
    value = torch.tensor(0.5 / want).bfloat16().item()
    assert g[0].item() == g[-1].item() == g[2 ** 31].item() == value and bool((g[2 ** 31 - 5:] == value).all())
    del g
    many = list(torch.ones(9000, 3, device="cuda").unbind(0)) + [torch.ones(2_000_003, device="cuda", dtype=torch.bfloat16)]
    norm, got = pk.head_clip(many, 3.0)
    want = math.sqrt(27_000 + 2_000_003)
    assert abs(norm.item() / want - 1) < 1e-6
    assert all(abs(float(t[k].item()) - 3 / want) <= 2.0 ** -8 * 3 / want for t in (got[0], got[4500], got[8999], got[9000]) for k in (0, -1))


# ---------------------------------------------------------------- calls

@pytest.mark.gpu
def test_layer_calls_on_another_stream_and_from_a_graph():
    """The same bits on a stream of one's own, and on every replay of a captured block, with eager work between."""
    import torch
    rng = np.random.default_rng(2)
    for n, dim, hidden, dtype in ((7, 48, 100, "float32"), (300, 48, 100, "bfloat16"), (3000, 72, 130, "float32")):
        x, g = _rows(rng, n, dim, dtype)[0], _rows(rng, n, dim, dtype)[0]
        w1, w2 = _rows(rng, 2 * hidden, dim, dtype, scale=dim ** -0.5)[0], _rows(rng, dim, hidden, dtype, scale=hidden ** -0.5)[0]
        b1, b2 = (_torch(rng.standard_normal(k).astype(np.float32)) for k in (2 * hidden, dim))

        def block(stream=None):
            k = dict(stream=stream)
            h, z = pk.head_gated(x, w1, b1, "gelu", keep=True, **k)
            y, z2 = pk.head_linear(h, w2, b2, "silu", x, 0.5, keep=True, **k)
            gh, gw2, gb2 = pk.head_linear_grad(g, h, w2, z2, "silu", 0.5, **k)
            gx, gw1, gb1 = pk.head_gated_grad(gh, x, w1, z, "gelu", **k)
            norm, clipped = pk.head_clip([gw1, gb1, gw2, gb2], 0.5, **k)
            return [y, gx, norm, *clipped]

        want = [a.clone() for a in block()]
        torch.cuda.synchronize()
        other = torch.cuda.Stream()
        got = block(other)
        other.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = block()
        for k in range(4):
            x.mul_(0.75)
            want = [a.clone() for a in block()]
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(captured, want)), k
        with pytest.raises(ValueError, match="stream"):
            pk.head_linear(x, w1, stream=_OtherDevice())


class _OtherDevice:
    device = "another"


@pytest.mark.gpu
def test_layer_calls_of_two_threads_and_two_graphs_at_once():
    """Two threads on streams of their own, and two graphs replayed in turn, give the bits of calls one after the other."""
    import threading

    import torch
    rng = np.random.default_rng(3)
    sides = []
    for n, dim, hidden, dtype in ((2100, 600, 520, "bfloat16"), (900, 331, 200, "float32")):
        x, g = _rows(rng, n, dim, dtype)[0], _rows(rng, n, hidden, dtype)[0]
        w = _rows(rng, 2 * hidden, dim, dtype, scale=dim ** -0.5)[0]

        def run(x=x, g=g, w=w, stream=None):
            h, z = pk.head_gated(x, w, keep=True, stream=stream)
            gx, gw, gb = pk.head_gated_grad(g, x, w, z, stream=stream)
            norm, clipped = pk.head_clip([gw, gb], 0.5, stream=stream)
            return [h, pk.head_linear(h, w[:, :h.shape[1]], stream=stream) if h.shape[1] <= w.shape[1] else h, gx, norm, *clipped]
        sides.append((run, run()))
    torch.cuda.synchronize()
    failed = []

    def many(run, want):
        try:
            stream = torch.cuda.Stream()
            for k in range(30):
                if k % 2:
                    got = run(stream=stream)
                else:
                    with torch.cuda.stream(stream):
                        got = run()
                stream.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, want)), k
        except BaseException as e:  # noqa: BLE001  (told by the main thread)
            failed.append(e)

    threads = [threading.Thread(target=many, args=side) for side in sides]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    graphs = []
    for run, _ in sides:
        graphs.append((torch.cuda.CUDAGraph(), []))
        with torch.cuda.graph(graphs[-1][0]):
            graphs[-1][1].extend(run())
    for k in range(3):
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (_, got), (run, want) in zip(graphs, sides):
            assert all(torch.equal(a, b) for a, b in zip(got, want)), k
            run()
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_python_refuses_layers_that_do_not_fit():
    import torch
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(6, 8, device="cuda")
    g, z = torch.zeros(4, 6, device="cuda"), torch.zeros(4, 6, device="cuda")
    linear, gated, linear_grad, gated_grad = pk.head_linear, pk.head_gated, pk.head_linear_grad, pk.head_gated_grad
    for call, what in ((lambda: linear(x, w[:, :7]), "weight"), (lambda: linear(x, w.bfloat16()), "weight"), (lambda: linear(x.half(), w.half()), "float32 or"),
                       (lambda: linear(x[0], w), "shape"), (lambda: linear(x, w, torch.zeros(5, device="cuda")), "bias"),
                       (lambda: linear(x, w, torch.zeros(6, device="cuda").bfloat16()), "bias"), (lambda: linear(x, w, residual=g[:, :5]), "residual"),
                       (lambda: linear(x, w, residual=g[:1].expand(4, 6)), "overlap"), (lambda: linear(x.t(), w), "contiguous"),
                       (lambda: gated(x, w[:5]), "gates"),
                       (lambda: linear_grad(g[:, :5], x, w), "grad"), (lambda: linear_grad(g, x, w, None, "silu"), "z is what"),
                       (lambda: linear_grad(g, x, w, z[:3], "silu"), "z"), (lambda: gated_grad(g, x, w, z), "grad"),
                       (lambda: gated_grad(g[:, :3], x, w, z[:, :3]), "z"), (lambda: gated_grad(g[:, :3], x, w, None), "z is what"),
                       (lambda: pk.head_clip([g, w.half()], 1.0), "float32 or"), (lambda: pk.head_clip([g, w[:, :3]], 1.0), "contiguous"),
                       (lambda: pk.head_clip([g, g], 1.0, in_place=True), "overlap"),
                       (lambda: pk.head_clip([g.view(-1)[:10], g], 1.0, in_place=True), "overlap"),
                       (lambda: pk.head_clip([g, torch.zeros(3)], 1.0), "CUDA"), (lambda: pk.head_clip([g], 0.0), "above 0")):
        with pytest.raises(ValueError, match=what):
            call()
    with pytest.raises(pk.HeadError, match="invalid argument"):
        linear(x, w[:0])
    with pytest.raises(pk.HeadError, match="limit"):
        linear(torch.zeros(1, 16385, device="cuda"), torch.zeros(1, 16385, device="cuda"))
    grads = pk.head_clip([g, g], 1.0)[1]  # results of their own
    assert grads[0].data_ptr() != grads[1].data_ptr()
    for t in (x, w):
        t.requires_grad_()
        with pytest.raises(ValueError, match="requires a gradient"):
            linear(x, w)
        with pytest.raises(ValueError, match="requires a gradient"):
            pk.head_clip([t], 1.0)
        with torch.no_grad():
            linear(x, w)
        t.requires_grad_(False)


@pytest.mark.gpu
def test_clip_in_place_tells_autograd_that_it_wrote():
    import torch
    a = torch.ones(5, device="cuda", requires_grad=True)
    g = torch.full((5,), 3.0, device="cuda")
    y = (a * g).sum()
    pk.head_clip([g], 1.0, in_place=True)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    g = torch.full((5,), 3.0, device="cuda")
    y = (a * g).sum()
    pk.head_clip([g], 1.0)
    y.backward()
    assert a.grad.tolist() == [3.0] * 5


# ---------------------------------------------------------------- a head with blocks

class _Forest:
    def __init__(self, trees, depth):
        self.nodes = (2 << depth) - 1
        self.tree_offset = np.arange(trees + 1) * self.nodes


def _leaves(rng, n, trees, depth):
    return _torch(rng.integers(2 ** depth - 1, 2 ** (depth + 1) - 1, (n, trees)).astype(np.int32))


@pytest.mark.gpu
def test_gradients_of_a_head_with_blocks_agree_with_differences():
    """The gradients that a step takes, recovered from a step without momentum's division: they are read where the optimizer gets them."""
    import torch
    from paper_2301_13441_amd import leaf_head
    rng = np.random.default_rng(1)
    trees, depth, n, classes = 6, 3, 40, 5
    forest = _Forest(trees, depth)
    head = pk.LeafHead(forest.tree_offset, classes, dim=16, blocks=2, hidden=24, activation="gelu")
    leaves, targets = _leaves(rng, n, trees, depth), _torch(rng.integers(0, classes, n).astype(np.int32))
    seen, step = [], leaf_head.head_adamw
    leaf_head.head_adamw = lambda params, grads, *a, **k: seen.append((params, grads))
    try:
        head.train_step(leaves, targets, rate=0.0)
        head.train_step(leaves, targets, rate=0.0, max_norm=0.01)
    finally:
        leaf_head.head_adamw = step
    params, grads = seen[0]
    assert len(params) == len(grads) == 5 + 12
    norm = math.sqrt(sum((_np(g) ** 2).sum() for g in grads))
    assert abs(head.grad_norm.item() - norm) <= 1e-6 * norm and norm > 0.01
    for g, c in zip(grads, seen[1][1]):
        _close(c, _np(g) * (0.01 / norm), 1e-6 * np.abs(_np(g)))

    def loss():
        return _np(head.losses(leaves, targets)).mean()

    for k, (p, g) in enumerate(zip(params, grads)):
        direction = torch.sign(g) * (torch.rand_like(g) < 0.7)
        h = 1e-2 / max(1.0, float(direction.abs().sum()) ** 0.5)
        p.add_(direction, alpha=h)
        up = loss()
        p.add_(direction, alpha=-2 * h)
        down = loss()
        p.add_(direction, alpha=h)
        want = (_np(g) * _np(direction)).sum()
        # losses near 2 to some 1e-6 over 2 h, and h^2 of third derivatives next to a slope of the direction's own size
        assert abs((up - down) / (2 * h) - want) <= 4e-6 / (2 * h) + 0.02 * want, (k, (up - down) / (2 * h), want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,bits", [("float32", 32), ("bfloat16", 8)])
def test_a_head_with_blocks_runs(dtype, bits):
    import torch
    rng = np.random.default_rng(4)
    trees, depth, n, classes = 20, 4, 300, 40
    forest = _Forest(trees, depth)
    head = pk.LeafHead(forest.tree_offset, classes, dim=48, dtype=getattr(torch, dtype), bits=bits, blocks=3, hidden=70)
    leaves, targets = _leaves(rng, n, trees, depth), _torch(rng.integers(-1, classes, n).astype(np.int32))
    before = [p.clone() for p in head.params()]
    for _ in range(3):
        loss = head.train_step(leaves, targets, rate=1e-3, max_norm=1.0)
        assert loss.isfinite().all() and head.grad_norm.isfinite()
    assert all(not torch.equal(a, b) for a, b in zip(before, head.params()))
    logits = head.logits(leaves)
    assert logits.shape == (n, classes) and logits.dtype == head.dtype
    # the losses are those of the logits: of float32 to rounding, of bfloat16 to that of the logits
    l64, t = _np(logits), _np(targets).astype(int)
    want = np.where(t >= 0, np.log(np.exp(l64).sum(1)) - l64[np.arange(n), np.maximum(t, 0)], 0)
    _close(head.losses(leaves, targets), want, (2 * _ulp(dtype) + 200 * U) * (np.abs(l64).max(1) + 4))


@pytest.mark.gpu
def test_a_head_with_blocks_is_served():
    rng = np.random.default_rng(7)
    forest = _Forest(10, 3)
    head = pk.LeafHead(forest.tree_offset, 7, dim=32, blocks=1)
    for n in (1, 5, 200):
        leaves = _leaves(rng, n, 10, 3)
        probabilities, labels = head.predict(leaves)
        l64 = _np(head.logits(leaves))
        want = np.exp(l64) / np.exp(l64).sum(1, keepdims=True)
        _close(probabilities, want, 1e-5)
        assert (_np(labels) == l64.argmax(1)).all()
