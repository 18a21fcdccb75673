"""The trainable head (include/head.h): ABI checks that need no GPU, and the operators on the GPU against their definitions in
float64, computed here with numpy.

Tolerances are bounds on rounding, element by element, of float32 sums in any order: n terms differ from their exact sum by
at most n * 2^-24 * (sum of their magnitudes), and a bfloat16 result by half a unit in its last place, up to 2^-8 of itself, more.
"""
import ctypes
import os
import re

import numpy as np
import pytest

import paper_2301_13441_amd as pk
from paper_2301_13441_amd import head_binding as hb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24
TINY = 1e-37
DTYPES = ["float32", "bfloat16"]


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


def _rows(rng, n, dim, dtype, spread=0, shift=0):
    """(device tensor, float64 array) of [n, dim] values, its rows `spread` elements further apart than they are long and
    beginning `shift` elements into their memory."""
    whole = _torch(rng.standard_normal((n, dim + spread + shift)).astype(np.float32), dtype)
    t = whole[:, shift:shift + dim] if spread or shift else whole
    return t, _np(t)


# ---------------------------------------------------------------- no GPU needed

def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "head.h")).read()
    code = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(head_[a-z_]+)\s*\(", code))
    assert declared == set(hb.HEAD_EXPORTS)
    lib = hb._lib()
    assert all(hasattr(lib, name) for name in declared)
    assert f"#define HEAD_BLOCK {hb.BLOCK} " in re.sub(r" +", " ", header)


def _ids(n_rows=4, n_ids=3, n_vectors=10, ids=64, stride=3, offset=None):
    return hb._Ids(n_rows, n_ids, n_vectors, ids, stride, offset)


def test_embed_refuses_bad_arguments_before_any_device_call():
    lib = hb._lib()

    def call(i, dtype=0, dim=8, table=64, stride=8, out=64):
        return lib.head_embed(i, dtype, dim, table, stride, 1.0, out, None)

    def grad(i, dtype=0, dim=8, table=64, stride=8, out=64, work=64):
        return lib.head_embed_grad(i, dtype, dim, table, stride, 1.0, out, work, None)

    for f in (call, grad):
        assert f(None) == -1
        assert f(_ids(n_rows=-1)) == f(_ids(n_ids=-1)) == f(_ids(n_vectors=-1)) == -1
        assert f(_ids(), dtype=2) == f(_ids(), dtype=-1) == f(_ids(), dim=0) == -1
        assert f(_ids(), dim=16385, stride=16385) == f(_ids(n_rows=10 ** 9 + 1)) == f(_ids(n_vectors=10 ** 9 + 1)) == -7
        assert f(_ids(ids=None)) == f(_ids(ids=66)) == f(_ids(stride=2)) == f(_ids(offset=68)) == -1
        assert f(_ids(), table=None) == f(_ids(), table=66) == f(_ids(), stride=7) == -1
        assert f(_ids(), out=None) == f(_ids(), out=65) == -1
    assert grad(_ids(), work=None) == grad(_ids(), work=72) == -1
    assert grad(_ids(n_rows=10 ** 6, n_ids=2148, stride=2148)) == -7      # n_rows * n_ids
    assert call(_ids(n_rows=0), table=None, out=None) == 0
    assert lib.head_embed_grad_bytes(_ids(), 0, 8) > 0
    assert lib.head_embed_grad_bytes(_ids(n_rows=0), 0, 8) == 0


def test_layer_norm_refuses_bad_arguments_before_any_device_call():
    lib = hb._lib()

    def call(dtype=0, n=4, dim=8, x=64, xs=8, w=64, b=64, eps=1e-5, y=64, mean=64, rstd=64):
        return lib.head_layer_norm(dtype, n, dim, x, xs, w, b, eps, y, mean, rstd, None)

    def grad(dtype=0, n=4, dim=8, g=64, gs=8, x=64, xs=8, w=64, mean=64, rstd=64, gx=64, gw=64, gb=64, work=64):
        return lib.head_layer_norm_grad(dtype, n, dim, g, gs, x, xs, w, mean, rstd, gx, gw, gb, work, None)

    for f in (call, grad):
        assert f(dtype=2) == f(n=-1) == f(dim=0) == f(x=None) == f(x=66) == f(xs=7) == f(w=None) == f(w=66) == -1
        assert f(mean=None) == f(rstd=66) == -1
        assert f(dim=16385) == f(n=10 ** 9 + 1) == -7
    assert call(eps=-1.0) == call(eps=float("nan")) == call(eps=float("inf")) == call(y=None) == call(b=66) == -1
    assert grad(g=None) == grad(gs=7) == grad(gx=66) == grad(gw=None) == grad(gb=None) == grad(work=None) == grad(work=8) == -1
    assert call(n=0, x=None, y=None) == 0
    assert lib.head_layer_norm_grad_bytes(0, 100, 8) > 0


def test_cross_entropy_refuses_bad_arguments_before_any_device_call():
    lib = hb._lib()

    def desc(dtype=0, n=4, dim=8, classes=5, h=64, hs=8, w=64, ws=8, b=64, t=64):
        return hb._Classes(dtype, n, dim, classes, h, hs, w, ws, b, t)

    def call(d, loss=64, lse=64, work=64):
        return lib.head_cross_entropy(d, loss, lse, work, None)

    def grad(d, lse=64, g=64, gh=64, gw=64, gb=64, work=64):
        return lib.head_cross_entropy_grad(d, lse, g, gh, gw, gb, work, None)

    for f in (call, grad):
        assert f(None) == -1
        for bad in (dict(dtype=2), dict(n=-1), dict(dim=0), dict(classes=0), dict(h=None), dict(h=66), dict(hs=7), dict(w=None),
                    dict(ws=7), dict(b=66), dict(t=None), dict(t=66)):
            assert f(desc(**bad)) == -1, bad
        for far in (dict(dim=16385), dict(n=10 ** 9 + 1), dict(classes=10 ** 9 + 1), dict(n=10 ** 9, classes=17_593)):
            assert f(desc(**far)) == -7, far
        assert f(desc(), work=None) == f(desc(), work=72) == f(desc(), lse=None) == -1
    assert call(desc(), loss=None) == call(desc(), loss=66) == -1
    assert grad(desc(), g=None) == grad(desc(), gh=None) == grad(desc(), gw=None) == grad(desc(), gb=66) == -1
    assert call(desc(n=0, h=None, t=None), loss=None, lse=None, work=None) == 0
    assert lib.head_cross_entropy_bytes(desc()) > 0 and lib.head_cross_entropy_grad_bytes(desc()) > 0
    assert lib.head_cross_entropy_bytes(desc(n=0)) == lib.head_cross_entropy_grad_bytes(desc(n=0)) == 0


def test_adamw_refuses_bad_arguments_before_any_device_call():
    lib = hb._lib()

    def call(n=1, **kw):
        rule = dict(grad_dtype=0, bits=32, step=1, rate=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, decay=0.0, seed=0)
        tensor = dict(param=64, grad=64, m=64, v=64, m_scale=64, v_scale=64, copy=None, n=8)
        rule.update((k, v) for k, v in kw.items() if k in rule)
        tensor.update((k, v) for k, v in kw.items() if k in tensor)
        rows = (hb._AdamwTensor * 1)(hb._AdamwTensor(**tensor))
        return lib.head_adamw(hb._AdamwRule(**rule), rows if n else None, n, None)

    inf, nan = float("inf"), float("nan")
    for bad in (dict(grad_dtype=2), dict(bits=16), dict(step=0), dict(rate=inf), dict(rate=nan), dict(decay=nan), dict(beta1=1.0),
                dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan), dict(eps=-1.0), dict(eps=nan), dict(param=None), dict(param=66),
                dict(grad=None), dict(m=None), dict(v=66), dict(copy=65), dict(bits=8, m_scale=None), dict(bits=8, v_scale=None)):
        assert call(**bad) == -1, bad
    assert lib.head_adamw(hb._AdamwRule(0, 32, 1, 0, 0, 0, 0, 0, 0), None, 1, None) == -1
    assert lib.head_adamw(None, None, 0, None) == -1
    assert lib.head_adamw(hb._AdamwRule(0, 32, 1, 0, 0, 0, 0, 0, 0), None, -1, None) == -1
    assert lib.head_adamw(hb._AdamwRule(0, 32, 1, 0, 0, 0, 0, 0, 0), None, 1000001, None) == -1
    assert call(n=0) == 0                                                   # no tensors
    rows = (hb._AdamwTensor * 1)(hb._AdamwTensor(n=8))
    assert lib.head_adamw_values(rows, None, None, 1, None) == -1
    at = (ctypes.c_void_p * 1)(64)
    assert lib.head_adamw_values(rows, at, at, 1, None) == -1               # no codes
    assert lib.head_strerror(-1).decode() == "invalid argument"


def test_python_refuses_what_is_not_a_device_tensor():
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="CUDA"):
        pk.head_layer_norm(x, torch.ones(8))
    with pytest.raises(ValueError, match="CUDA"):
        pk.head_embed(x, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        pk.head_cross_entropy(x, x, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        pk.head_adamw([x], [x], [pk.head_adamw_state(x)], 1, 1e-3)
    with pytest.raises(ValueError, match="length"):
        pk.head_adamw([x], [], [], 1, 1e-3)
    with pytest.raises(ValueError, match="bits"):
        pk.head_adamw_state(x, 16)


# ---------------------------------------------------------------- embedding

def _leaf_ids(rng, n, t, vectors, none=0.15):
    """Ids into t blocks of vectors, some negative, some past the end; rows 0 and n // 2 have no vector at all."""
    each = max(1, vectors // max(1, t))
    ids = rng.integers(0, each, (n, t)).astype(np.int32)
    ids[rng.random((n, t)) < 0.3] //= 7                  # some vectors are frequent
    ids[rng.random((n, t)) < none] = -1
    ids[rng.random((n, t)) < none / 3] = 2 ** 31 - 1
    if n > 2:
        ids[[0, n // 2]] = -5
    return ids, (np.arange(t, dtype=np.int64) * each)


def _vectors_of(ids, offsets, n_vectors):
    at = ids.astype(np.int64) + offsets
    return at, (ids >= 0) & (at >= 0) & (at < n_vectors)


EMBED = [  # rows, ids, vectors, dim
    (1, 1, 1, 1), (1, 500, 5000, 64), (1, 3, 9, 257), (2, 40, 400, 31), (3, 0, 5, 8), (5, 1, 7, 2), (64, 130, 1300, 8), (257, 7, 70, 50),
    (1000, 16, 64, 96), (1500, 100, 3000, 200), (4099, 3, 50, 128), (700, 1, 30, 1000), (33, 9, 17, 520), (20000, 2, 70000, 4)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,t,vectors,dim", EMBED)
def test_embed_and_its_gradient(n, t, vectors, dim, dtype):
    rng = np.random.default_rng(n * 31 + t * 7 + dim)
    ids, offsets = _leaf_ids(rng, n, t, vectors)
    for spread, shift in ((0, 0), (3, 1)):
        table, table64 = _rows(rng, vectors, dim, dtype, spread, shift)
        grad, grad64 = _rows(rng, n, dim, dtype, spread, shift)
        wide = np.full((n, t + spread), -1, np.int32)
        wide[:, :t] = ids
        ids_d, off_d = _torch(wide)[:, :t], _torch(offsets)
        at, here = _vectors_of(ids, offsets, vectors)
        want, size = np.zeros((n, dim)), np.zeros((n, dim))
        want_g, size_g, count = np.zeros((vectors, dim)), np.zeros((vectors, dim)), np.zeros(vectors)
        for k in range(t):
            r = np.nonzero(here[:, k])[0]
            want[r] += table64[at[r, k]]
            size[r] += np.abs(table64[at[r, k]])
            np.add.at(want_g, at[r, k], grad64[r])
            np.add.at(size_g, at[r, k], np.abs(grad64[r]))
            np.add.at(count, at[r, k], 1)
        scale = 0.37
        got = pk.head_embed(table, ids_d, off_d, scale)
        _close(got, scale * want, scale * ((t + 2) * U * size + _ulp(dtype) * np.abs(want)), "forward")
        got_g = pk.head_embed_grad(grad, ids_d, vectors, off_d, scale)
        _close(got_g, scale * want_g, scale * ((count[:, None] + 2) * U * size_g + _ulp(dtype) * np.abs(want_g)), "gradient")
        assert (_np(got_g)[count == 0] == 0).all()
        import torch
        assert torch.equal(got_g, pk.head_embed_grad(grad, ids_d, vectors, off_d, scale))      # the same bits


@pytest.mark.gpu
@pytest.mark.parametrize("n,vectors", [(1, 5), (63, 5), (64, 1), (65, 300), (4096, 70_000), (4097, 3), (300_000, 1), (300_001, 2 ** 24 + 5)])
def test_embed_gradient_of_plain_lookups(n, vectors):
    """One id a row: every length around the chunks and tiles of the sort, all rows on one vector, ids of one to four bytes."""
    rng = np.random.default_rng(n + vectors)
    ids = rng.integers(0, vectors, n).astype(np.int32)
    if n > 100:
        ids[rng.random(n) < 0.5] = vectors - 1
    grad = rng.integers(-8, 9, (n, 4)).astype(np.float32)                      # sums of small whole numbers are exact
    want = np.zeros((vectors, 4))
    np.add.at(want, ids, grad)
    got = pk.head_embed_grad(_torch(grad), _torch(ids), vectors)
    assert np.array_equal(_np(got), want)


@pytest.mark.gpu
def test_embed_offsets_past_32_bits():
    import torch
    vectors, dim = 18_000_000, 128                                             # 2.3e9 values
    table = torch.zeros(vectors, dim, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([[vectors - 1, 5], [17_000_000, -1], [3, 16_777_216]], dtype=torch.int32, device="cuda")
    table[vectors - 1], table[5], table[17_000_000], table[3], table[16_777_216] = 1, 2, 4, 8, 16
    assert _np(pk.head_embed(table, ids))[:, 0].tolist() == [3, 4, 24]
    # the same vectors through offsets beyond 32 bits of values
    off = torch.tensor([0, 16_000_000], dtype=torch.int64, device="cuda")
    shifted = torch.tensor([[5, 777_216], [3, 1_999_999]], dtype=torch.int32, device="cuda")
    assert _np(pk.head_embed(table, shifted, off))[:, 127].tolist() == [18, 9]
    del table
    grad = torch.tensor([[1.0], [2.0], [4.0]], device="cuda").expand(3, dim).contiguous().bfloat16()
    out = pk.head_embed_grad(grad, ids, vectors)
    for v, want in ((vectors - 1, 1), (5, 1), (17_000_000, 2), (3, 4), (16_777_216, 4), (0, 0), (vectors - 2, 0)):
        assert (out[v] == want).all(), v
    assert out.float().sum().item() == 12 * dim


@pytest.mark.gpu
def test_embed_keeps_infinities_and_nan_to_their_rows():
    table = np.ones((6, 8), np.float32)
    table[1], table[2] = np.inf, np.nan
    ids = np.array([[0, 3], [1, 0], [2, 0], [-1, 4], [-1, -1]], np.int32)
    got = _np(pk.head_embed(_torch(table), _torch(ids)))
    assert (got[[0, 3, 4], 0] == [2, 1, 0]).all() and np.isinf(got[1]).all() and np.isnan(got[2]).all()
    grad = np.ones((5, 8), np.float32)
    grad[4], grad[1] = np.nan, np.inf                                          # row 4 has no id: its gradient goes nowhere
    got = _np(pk.head_embed_grad(_torch(grad), _torch(ids), 6))
    assert got[:, 0].tolist() == [np.inf, np.inf, 1, 1, 1, 0]


# ---------------------------------------------------------------- layer norm

NORM = [(1, 1), (1, 64), (3, 2), (7, 90), (1000, 8), (129, 33), (2049, 50), (65, 256), (40, 513), (31, 1000), (17, 2047), (9, 2048), (5, 4100),
        (3, 9001), (2, 16384), (5000, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,dim", NORM)
def test_layer_norm_and_its_gradient(n, dim, dtype):
    rng = np.random.default_rng(n * 17 + dim)
    w, b = (rng.standard_normal(dim).astype(np.float32) for _ in range(2))
    eps = 1e-5
    for spread, shift in ((0, 0), (5, 3)):
        x, x64 = _rows(rng, n, dim, dtype, spread, shift)
        x += 2
        x64 = _np(x)
        g, g64 = _rows(rng, n, dim, dtype, spread, shift)
        mean = x64.mean(1)
        var = ((x64 - mean[:, None]) ** 2).mean(1)
        rstd = 1 / np.sqrt(var + eps)
        unit = (x64 - mean[:, None]) * rstd[:, None]
        most = np.abs(x64).max(1)
        gamma = (dim + 16) * U
        got_y, got_m, got_r = pk.head_layer_norm(x, _torch(w), _torch(b), eps)
        _close(got_m, mean, gamma * most, "mean")
        # the variance is a sum of dim squares whose terms are off by the mean's error, and rstd takes half its relative error
        _close(got_r, rstd, rstd * gamma * (2 + 4 * most * rstd), "rstd")
        y = unit * w + b
        bound = gamma * (4 * most * rstd + 4)[:, None] * (1 + np.abs(unit)) * np.abs(w) + 4 * U * (np.abs(unit * w) + np.abs(b))
        _close(got_y, y, bound + _ulp(dtype) * np.abs(y), "y")
        got_y, _, _ = pk.head_layer_norm(x, _torch(w), None, eps)
        _close(got_y, unit * w, bound + _ulp(dtype) * np.abs(unit * w), "y without bias")

        m32, r32 = mean.astype(np.float32), rstd.astype(np.float32)            # as they are given to the gradient
        m64, r64 = m32.astype(np.float64)[:, None], r32.astype(np.float64)[:, None]
        u = (x64 - m64) * r64
        size = (np.abs(x64) + np.abs(m64)) * r64                               # of unit's terms
        gw = g64 * w
        dx = r64 * (gw - gw.mean(1, keepdims=True) - u * (gw * u).mean(1, keepdims=True))
        got_x, got_w, got_b = pk.head_layer_norm_grad(g, x, _torch(w), _torch(m32), _torch(r32))
        bound = gamma * r64 * (np.abs(gw) + np.abs(gw).mean(1, keepdims=True) + 2 * size * (np.abs(gw) * size).mean(1, keepdims=True))
        _close(got_x, dx, bound + _ulp(dtype) * np.abs(dx), "dx")
        _close(got_w, (g64 * u).sum(0), (n + 16) * U * (np.abs(g64) * size).sum(0), "dw")
        _close(got_b, g64.sum(0), (n + 16) * U * np.abs(g64).sum(0), "db")


@pytest.mark.gpu
def test_layer_norm_of_no_rows_and_constant_rows():
    import torch
    w = torch.ones(8, device="cuda")
    y, mean, rstd = pk.head_layer_norm(torch.empty(0, 8, device="cuda"), w)
    assert y.shape == (0, 8) and mean.shape == rstd.shape == (0,)
    none = torch.empty(0, 8, device="cuda")
    gx, gw, gb = pk.head_layer_norm_grad(none, none, w, mean, rstd)
    assert gx.shape == (0, 8) and (gw == 0).all() and (gb == 0).all()
    y, mean, rstd = pk.head_layer_norm(torch.full((3, 8), 5.0, device="cuda"), w, None, 1e-4)
    assert (y == 0).all() and (mean == 5).all()
    np.testing.assert_allclose(_np(rstd), 100, rtol=4 * U)
    x = torch.randn(4, 8, device="cuda")
    x[1, 3], x[2, 0] = float("inf"), float("nan")
    y = pk.head_layer_norm(x, w)[0]
    assert torch.isfinite(y[[0, 3]]).all() and torch.isnan(y[[1, 2]]).any(1).all()


@pytest.mark.gpu
def test_layer_norm_rows_past_32_bits():
    import torch
    n, dim = 2_200_000, 1024                                                   # 2.25e9 values
    x = torch.zeros(n, dim, dtype=torch.bfloat16, device="cuda")
    x[-1, ::2] = 1
    y, mean, rstd = pk.head_layer_norm(x, torch.ones(dim, device="cuda"), None, 0.0 + 1e-6)
    assert mean[-1] == 0.5 and (y[-1, ::2] == 1).all() and (y[-1, 1::2] == -1).all() and (y[-2] == 0).all()
    del y
    g = torch.zeros_like(x)
    g[-1] = 2
    gx, gw, gb = pk.head_layer_norm_grad(g, x, torch.ones(dim, device="cuda"), mean, rstd)
    assert (gb == 2).all() and torch.allclose(gw.abs(), torch.full_like(gw, 2.0), rtol=1e-5) and (gx[-1].abs() < 1e-2).all()


# ---------------------------------------------------------------- cross entropy

LOSS = [  # rows, dim, classes
    (1, 1, 1), (1, 64, 10), (1, 512, 5003), (2, 8, 129), (33, 50, 2), (127, 90, 128), (128, 64, 127), (129, 16, 257), (300, 31, 1000),
    (1021, 64, 10), (64, 200, 4099), (515, 128, 2048), (1500, 72, 333)]


def _cross_entropy(h, w, b, t):
    """(logits, lse, loss, sizes of the logits' terms) in float64."""
    logits, size = h @ w.T + b, np.abs(h) @ np.abs(w).T + np.abs(b)
    most = logits.max(1)
    lse = most + np.log(np.exp(logits - most[:, None]).sum(1))
    has = (t >= 0) & (t < len(w))
    loss = np.where(has, lse - logits[np.arange(len(h)), np.where(has, t, 0)], 0)
    return logits, lse, loss, size, has


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,dim,classes", LOSS)
def test_cross_entropy_and_its_gradient(n, dim, classes, dtype):
    _check_cross_entropy(n, dim, classes, dtype, ((0, 0, True), (3, 1, False), (8, 8, True)))


@pytest.mark.gpu
@pytest.mark.parametrize("n,dim,classes", [(4099, 72, 4200), (300, 24, 40_000), (9000, 300, 2050)])
def test_cross_entropy_in_large_tiles(n, dim, classes):
    """Enough tiles of 256 x 256 that bfloat16 products run in them, with rows, classes and dim that end inside one."""
    _check_cross_entropy(n, dim, classes, "bfloat16", ((0, 0, True),))


def _check_cross_entropy(n, dim, classes, dtype, variants):
    rng = np.random.default_rng(n * 13 + dim * 5 + classes)
    for spread, shift, biased in variants:
        h, h64 = _rows(rng, n, dim, dtype, spread, shift)
        w, w64 = _rows(rng, classes, dim, dtype, spread, shift)
        h *= 0.7
        w *= dim ** -0.5
        h64, w64 = _np(h), _np(w)
        b = (rng.standard_normal(classes) * 0.5).astype(np.float32) if biased else np.zeros(classes, np.float32)
        t = rng.integers(0, classes, n).astype(np.int32)
        if n > 3:
            t[1], t[n // 2], t[-1] = -1, classes, -7
        logits, lse, loss, size, has = _cross_entropy(h64, w64, b, t)
        # A logit is off by the rounding of its sum (in matrix instructions: 4 U a term), lse by the largest of that, and its own.
        off = 4 * (dim + 2) * U * size
        off_lse = off.max(1) + (classes + 16) * U + 4 * U * (np.abs(lse) + np.abs(logits).max(1))
        bias = _torch(b) if biased else None
        got, got_lse = pk.head_cross_entropy(h, w, _torch(t), bias)
        _close(got_lse, lse, off_lse, "lse")
        _close(got, loss, np.where(has, off_lse + off.max(1), 0), "loss")

        g = (rng.standard_normal(n) / n).astype(np.float32)
        lse32 = lse.astype(np.float32)
        p = np.exp(logits - lse[:, None])
        delta = p.copy()
        r = np.nonzero(has)[0]
        delta[r, t[r]] -= 1
        delta *= (g * has)[:, None]
        # p is off by its logit's error and lse's, relatively, and by the rounding of the argument; then by its own rounding
        rel = off + 2 * U * (np.abs(lse)[:, None] + np.abs(logits)) + 8 * U
        off_delta = np.abs(g * has)[:, None] * (2 * p * rel + 4 * U) * has[:, None]
        got_h, got_w, got_b = pk.head_cross_entropy_grad(_torch(g), h, w, _torch(t), _torch(lse32), bias)
        rounded = off_delta + _ulp(dtype) * np.abs(delta) if dtype == "bfloat16" else off_delta
        dh, dw = delta @ w64, delta.T @ h64
        _close(got_h, dh, rounded @ np.abs(w64) * 1.01 + 4 * (classes + 8) * U * (np.abs(delta) @ np.abs(w64)) + _ulp(dtype) * np.abs(dh) * 1.01, "grad_hidden")
        _close(got_w, dw, rounded.T @ np.abs(h64) * 1.01 + 4 * (n + 8) * U * (np.abs(delta).T @ np.abs(h64)) + _ulp(dtype) * np.abs(dw) * 1.01, "grad_weight")
        if biased:
            _close(got_b, delta.sum(0), off_delta.sum(0) + (n + 8) * U * np.abs(delta).sum(0), "grad_bias")
        else:
            assert got_b is None
        assert (_np(got_h)[~has] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n,dim,classes", [(70_001, 16, 10), (300_003, 8, 3)])
def test_cross_entropy_of_many_rows_and_few_classes(n, dim, classes):
    """Rows' tiles by the hundreds of few classes, a grad_loss of rows of very different weight, some of them none."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(n)
    h = torch.randn(n, dim, generator=g, device="cuda").bfloat16()
    w = torch.randn(classes, dim, generator=g, device="cuda").bfloat16()
    b = torch.randn(classes, generator=g, device="cuda")
    t = torch.randint(0, classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    gl = torch.rand(n, generator=g, device="cuda") ** 8 / n
    gl[::7] = 0
    loss, lse = pk.head_cross_entropy(h, w, t, b)
    gh, gw, gb = pk.head_cross_entropy_grad(gl, h, w, t, lse, b)
    h64, w64 = h.double(), w.double()
    logits = h64 @ w64.T + b.double()
    want_lse = torch.logsumexp(logits, 1)
    p = torch.softmax(logits, 1)
    p[torch.arange(n, device="cuda"), t.long()] -= 1
    p *= gl.double()[:, None]
    # logits to 4 (dim + 2) U of their terms, which are below 60 here; p to that and its own rounding, relative to grad_loss
    off = 4 * (dim + 2) * U * 60 + 64 * U
    _close(lse, _np(want_lse), off)
    size = gl.double()[:, None].expand(n, classes) * (2 * off) + p.abs() * 2.0 ** -8
    want = p @ w64
    _close(gh, _np(want), _np(size @ w64.abs()) * 1.01 + 2.0 ** -8 * 1.01 * np.abs(_np(want)))
    want = p.T @ h64
    _close(gw, _np(want), _np(size.T @ h64.abs()) * 1.01 + n * U / 16 * _np(p.abs().T @ h64.abs()) + 2.0 ** -8 * 1.01 * np.abs(_np(want)))
    _close(gb, _np(p.sum(0)), _np((gl.double()[:, None] * 2 * off).sum(0)) + n * U / 16 * _np(p.abs().sum(0)))
    none = pk.head_cross_entropy_grad(torch.zeros_like(gl), h, w, t, lse, b)
    assert all((x == 0).all() for x in none)


@pytest.mark.gpu
def test_embed_offsets_that_lead_out_of_the_table():
    """Offsets below zero, and so large that no sum of theirs is a vector."""
    import torch
    table = torch.arange(5, dtype=torch.float32, device="cuda")[:, None].expand(5, 8).contiguous()
    ids = torch.tensor([[4, 3, 2 ** 31 - 1], [1, 0, 1], [-1, 2 ** 31 - 1, 0]], dtype=torch.int32, device="cuda")
    off = torch.tensor([-1, 2 ** 63 - 1, 3 - 2 ** 31], dtype=torch.int64, device="cuda")
    assert _np(pk.head_embed(table, ids, off))[:, 0].tolist() == [3 + 2, 0, 0]      # 4 - 1; 2^31 - 1 + 3 - 2^31; 1 - 1
    got = pk.head_embed_grad(torch.tensor([[1.0], [2.0], [4.0]], device="cuda").expand(3, 8).contiguous(), ids, 5, off)
    assert _np(got)[:, 0].tolist() == [2, 0, 1, 1, 0]


@pytest.mark.gpu
def test_cross_entropy_of_no_rows():
    import torch
    h, w, b = torch.empty(0, 8, device="cuda"), torch.randn(5, 8, device="cuda"), torch.zeros(5, device="cuda")
    t = torch.empty(0, dtype=torch.int32, device="cuda")
    loss, lse = pk.head_cross_entropy(h, w, t, b)
    assert loss.shape == lse.shape == (0,)
    gh, gw, gb = pk.head_cross_entropy_grad(loss, h, w, t, lse, b)
    assert gh.shape == (0, 8) and (gw == 0).all() and (gb == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_cross_entropy_masks_classes_by_a_bias_of_minus_infinity(dtype):
    """Classes whose bias is -inf, or the type's lowest value, have no share; whole tiles of them, and rows whose
    target is the only class left."""
    import torch
    rng = np.random.default_rng(5)
    n, dim, classes = 130, 40, 700
    h, h64 = _rows(rng, n, dim, dtype)
    w, w64 = _rows(rng, classes, dim, dtype)
    for low in (-np.inf, np.finfo(np.float32).min):
        b = np.full(classes, low, np.float32)
        b[[300, 301, 650]] = 0
        t = np.full(n, 300, np.int32)
        keep = [300, 301, 650]
        logits, lse, loss, size, _ = _cross_entropy(h64, w64[keep], np.zeros(3), np.zeros(n, np.int64))
        got, got_lse = pk.head_cross_entropy(h, w, _torch(t), _torch(b))
        off = 4 * (dim + 2) * U * size.max(1) + 8 * U * (1 + np.abs(logits).max(1))
        _close(got_lse, lse, off)
        _close(got, loss, 2 * off)
        g = np.full(n, 1 / n, np.float32)
        gh, gw, gb = pk.head_cross_entropy_grad(_torch(g), h, w, _torch(t), got_lse, _torch(b))
        for grad in (gh, gw, gb):
            assert torch.isfinite(grad).all()
        masked = np.setdiff1d(np.arange(classes), keep)
        assert (_np(gw)[masked] == 0).all() and (_np(gb)[masked] == 0).all()


@pytest.mark.gpu
def test_cross_entropy_keeps_nan_to_its_row_and_ignores_rows_without_target():
    import torch
    h, w = torch.randn(200, 16, device="cuda"), torch.randn(50, 16, device="cuda")
    t = torch.zeros(200, dtype=torch.int32, device="cuda")
    t[7] = -1
    h[7], h[9] = float("nan"), float("nan")
    loss, lse = pk.head_cross_entropy(h, w, t)
    assert loss[7] == 0 and torch.isnan(loss[9]) and torch.isfinite(loss[[*range(7), 8, *range(10, 200)]]).all()
    big = torch.full((3, 4), 1e4, device="cuda")                               # logits of 4e8: no overflow
    loss, lse = pk.head_cross_entropy(big, big[:2].contiguous() * 10, torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert torch.isfinite(loss).all()


@pytest.mark.gpu
def test_cross_entropy_in_several_pieces_of_the_classes():
    """So many rows that p of all classes is larger than a piece: the pieces' gradients add up."""
    import torch
    n, dim, classes = 270_000, 8, 2_100
    g = torch.Generator(device="cuda").manual_seed(3)
    h = torch.randn(n, dim, generator=g, device="cuda")
    w = torch.randn(classes, dim, generator=g, device="cuda") * 0.3
    b = torch.randn(classes, generator=g, device="cuda") * 0.1
    t = torch.randint(0, classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    loss, lse = pk.head_cross_entropy(h, w, t, b)
    gl = torch.full((n,), 1.0 / n, device="cuda")
    got = pk.head_cross_entropy_grad(gl, h, w, t, lse, b)
    want_w, want_b, want_h, size_w, size_b = 0, 0, [], 0, 0
    for lo in range(0, n, 30_000):
        h64, t64 = h[lo:lo + 30_000].double(), t[lo:lo + 30_000].long()
        logits = h64 @ w.double().T + b.double()
        p = torch.softmax(logits, 1)
        p[torch.arange(len(t64), device="cuda"), t64] -= 1
        p /= n
        want_h.append(p @ w.double())
        want_w, want_b = want_w + p.T @ h64, want_b + p.sum(0)
        size_w, size_b = size_w + p.abs().T @ h64.abs(), size_b + p.abs().sum(0)
    # p to 64 U of itself (logits of a few units), and a sum's rounding at its length over the 256 lanes and tiles it is cut into
    u = 64 * U + n * U / 16
    _close(got[1], _np(want_w), u * _np(size_w))
    _close(got[2], _np(want_b), u * _np(size_b))
    _close(got[0], _np(torch.cat(want_h)), (64 + classes) * 4 * U * _np(torch.cat(want_h).abs() + w.double().abs().max() / n))


# ---------------------------------------------------------------- gradients against differences

@pytest.mark.gpu
def test_gradients_agree_with_differences_of_the_whole_head():
    """d loss along a direction in every parameter, by central differences of the head in float64, against the
    operators' gradients through embed, layer norm and cross entropy."""
    rng = np.random.default_rng(11)
    n, t, vectors, dim, classes, eps, h = 37, 5, 60, 24, 9, 1e-5, 1e-5
    ids, offsets = _leaf_ids(rng, n, t, vectors)
    targets = rng.integers(-1, classes, n).astype(np.int32)
    has = targets >= 0
    theta = [rng.standard_normal(s).astype(np.float32) for s in ((vectors, dim), (dim,), (dim,), (classes, dim), (classes,))]
    at, here = _vectors_of(ids, offsets, vectors)

    def loss(theta):
        e, nw, nb, w, b = theta
        x = (e[np.where(here, at, 0)] * here[..., None]).sum(1) * 0.5
        mean = x.mean(1, keepdims=True)
        y = (x - mean) / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps) * nw + nb
        return _cross_entropy(y, w, b, targets)[2].sum() / has.sum()

    d = [_torch(p) for p in theta]
    ids_d, off_d, t_d = _torch(ids), _torch(offsets), _torch(targets)
    x = pk.head_embed(d[0], ids_d, off_d, 0.5)
    y, mean, rstd = pk.head_layer_norm(x, d[1], d[2], eps)
    _, lse = pk.head_cross_entropy(y, d[3], t_d, d[4])
    share = np.full(n, 1 / has.sum(), np.float32)
    gy, gw, gb = pk.head_cross_entropy_grad(_torch(share), y, d[3], t_d, lse, d[4])
    gx, gnw, gnb = pk.head_layer_norm_grad(gy, x, d[1], mean, rstd)
    ge = pk.head_embed_grad(gx, ids_d, vectors, off_d, 0.5)
    for k, grad in enumerate((ge, gnw, gnb, gw, gb)):
        direction = rng.standard_normal(theta[k].shape)
        ahead, back = ([p + s * h * direction if i == k else p.astype(np.float64) for i, p in enumerate(theta)] for s in (1, -1))
        slope = (loss(ahead) - loss(back)) / (2 * h)
        # differences: h^2 times third derivatives (rows without ids have rstd = 316, whose cube counts), and 2^-52 / h; sums
        # of some thousand float32 products of magnitude 1 on the other side
        assert abs((_np(grad) * direction).sum() - slope) < 2e-4 * max(1, np.abs(_np(grad) * direction).sum()), k


# ---------------------------------------------------------------- AdamW

RULE = dict(rate=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, decay=0.02)


def _adamw64(p, g, m, v, step, rate, beta1, beta2, eps, decay):
    m, v = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    update = rate / (1 - beta1 ** step) * m / (np.sqrt(v) / np.sqrt(1 - beta2 ** step) + eps)
    return p * (1 - rate * decay) - update, m, v, update


def _decoded(code, scale):
    """Values of e4m3 codes and scale bytes, from the format's definition."""
    code, scale = _np(code).astype(np.int64), np.repeat(_np(scale).astype(np.int64), 128)[:len(code)]
    e, d = code >> 3 & 15, code & 7
    y = np.where(e > 0, (8 + d) * 2.0 ** (e - 10.0), d * 2.0 ** -9) * 2.0 ** (scale - 134.0)
    y = np.where(code & 127 == 127, np.nan, y)
    return np.where(code > 127, -y, y)


SIZES = [1, 7, 8, 127, 128, 129, 2047, 2048, 2049, 100_003]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_steps(bits, dtype):
    """Ninety tensors (several launches) of odd sizes, some beginning off a 16-byte boundary, over three steps."""
    import torch
    rng = np.random.default_rng(bits)
    params, grads, copies, p64 = [], [], [], []
    for k in range(90):
        n, shift = SIZES[k % len(SIZES)], k % 3
        whole = _torch(rng.standard_normal(n + 4).astype(np.float32))
        params.append(whole[shift:shift + n])
        copies.append(torch.empty(n + 8, dtype=torch.bfloat16, device="cuda")[shift:shift + n] if k % 2 else None)
        p64.append(_np(params[-1]))
    states = [pk.head_adamw_state(p, bits) for p in params]
    for step in (1, 2, 3):
        grads = [_torch((rng.standard_normal(p.numel()) * 10.0 ** rng.integers(-6, 2)).astype(np.float32), dtype) for p in params]
        before = [(_np(s[0]), _np(s[1])) if bits == 32 else (_decoded(s[0], s[1]), _decoded(s[2], s[3]) ** 2) for s in states]
        pk.head_adamw(params, grads, states, step, copies=copies, seed=9, **RULE)
        values = pk.head_adamw_values(states, params) if bits == 8 else states
        for k, (p, g, s) in enumerate(zip(params, grads, states)):
            want, m, v, update = _adamw64(p64[k], _np(g), *before[k], step, **RULE)
            # the update is a quotient of float32 values of few roundings each; the sums of m may cancel, which counts in their size
            size = np.abs(update) + RULE["rate"] / (1 - RULE["beta1"] ** step) * (np.abs(RULE["beta1"] * before[k][0]) + np.abs(0.1 * _np(g))) / (
                np.sqrt(v) / np.sqrt(1 - RULE["beta2"] ** step) + RULE["eps"])
            _close(p, want, 4 * U * np.abs(p64[k]) + 16 * U * size, ("param", k, step))
            if bits == 32:
                _close(s[0], m, 4 * U * (np.abs(before[k][0]) + np.abs(_np(g))), ("m", k))
                _close(s[1], v, 4 * U * v, ("v", k))
            else:
                for got, want_s, (code, scale), off in ((values[k][0], m, s[:2], np.abs(before[k][0]) + np.abs(_np(g))),
                                                        (values[k][1], np.sqrt(v), s[2:], np.sqrt(v))):
                    root = got is values[k][1]
                    have = _decoded(code, scale)
                    assert np.array_equal(_np(got), have ** 2 if root else have), ("values", k)
                    most = np.array([np.abs(want_s[i:i + 128]).max() for i in range(0, len(want_s), 128)])
                    # one step of the code at most: 2^-3 of the power of two below, 2^-9 of the scale's range, which is 2^7
                    room = 2.0 ** -3 * np.maximum(np.abs(want_s), np.repeat(most * 2.0 ** -13, 128)[:len(want_s)]) * 1.01 + 4 * U * off
                    assert (np.abs(have - want_s) <= room).all(), ("state", k, step)
                    if root:
                        assert (have[want_s > 1e-30] > 0).all()
            if copies[k] is not None:
                assert torch.equal(copies[k], p.bfloat16()), ("copy", k)
            p64[k] = _np(p)


@pytest.mark.gpu
def test_adamw_rounds_8_bit_states_right_on_average():
    """A constant m and v between two codes: the mean of what is kept is the value itself, within 6 standard errors; and other
    seeds, steps and tensors round otherwise."""
    import torch
    n = 1 << 20
    p = torch.zeros(n, device="cuda")
    g = torch.full((n,), 0.7371, device="cuda")
    g[::128] = 1.0                                        # the scale's value
    kept = []
    for seed, step in ((1, 1), (2, 1), (1, 2)):
        states = [pk.head_adamw_state(p, 8), pk.head_adamw_state(p, 8)]
        pk.head_adamw([p, p.clone()], [g, g], states, step, 0.0, 0.0, 0.0, seed=seed)    # m = g, root of v = |g|
        for s in states:
            m, root = _decoded(s[0], s[1]), _decoded(s[2], s[3])
            for x in (m, root):
                x = np.delete(x.reshape(-1, 128), 0, 1)
                assert set(np.unique(x)) == {0.6875, 0.75}
                assert abs(x.mean() - np.float32(0.7371)) < 6 * 0.0625 / 2 / np.sqrt(x.size)
            assert (m != root).any()
            kept.append(m)
    for a in range(len(kept)):
        for b in range(a):
            assert 0.2 < (kept[a] != kept[b]).mean() < 0.5     # independent: 2 * 0.206 * 0.794 = 0.327


@pytest.mark.gpu
def test_adamw_8_bit_states_of_zeros_infinities_and_nan():
    import torch
    n = 300
    p, g = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda")
    g[130], g[131], g[260] = float("inf"), float("nan"), 1e-3
    state = pk.head_adamw_state(p, 8)
    pk.head_adamw([p], [g], [state], 1, 1e-2, decay=0.0)
    assert (p[:130] == 1).all() and (p[132:260] == 1).all() and torch.isnan(p[130:132]).all()
    (m, v), = pk.head_adamw_values([state], [p])
    assert torch.isnan(m[130:132]).all() and torch.isnan(v[130:132]).all() and (m[:130] == 0).all() and (m[132:256] == 0).all()
    assert abs(p[260].item() - 0.99) < 1e-5 and m[260] > 0 and v[260] > 0
    assert state.m_scale.tolist()[:2] == [0, 0] and (state.m[:128] == 0).all()
    # a root far below its block's largest keeps a code above zero, so that m is never divided by zero
    g = torch.full((128,), 1e-12, device="cuda")
    g[0] = 1
    q, state = torch.zeros(128, device="cuda"), pk.head_adamw_state(torch.zeros(128, device="cuda"), 8)
    for step in range(1, 20):
        pk.head_adamw([q], [g], [state], step, 1e-3, decay=0.0, seed=step)
    assert (state.v > 0).all() and (q.abs() <= 0.04).all()   # 19 steps of 1e-3, give or take the codes' eighths


@pytest.mark.gpu
def test_adamw_of_more_values_than_32_bits_count():
    import torch
    n = 2 ** 31 + 300
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    p[-1], g[-1], g[2 ** 31], g[5] = 1, 1, -1, 1
    state = pk.head_adamw_state(p, 8)
    pk.head_adamw([p], [g], [state], 1, 1e-2, decay=0.0)
    np.testing.assert_allclose(_np(p[[5, 2 ** 31, n - 1, 6, n - 2]]), [-0.01, 0.01, 0.99, 0, 0], atol=1e-6)
    assert state.m.count_nonzero().item() == 3 and int(state.v[-1]) > 0


# ---------------------------------------------------------------- together

@pytest.mark.gpu
def test_calls_on_another_stream_and_from_a_graph():
    """The same bits on a stream of one's own, and on every replay of a captured step, with eager work between."""
    import torch
    rng = np.random.default_rng(2)
    n, t, vectors, dim, classes = 300, 20, 600, 48, 77
    ids, offsets = _leaf_ids(rng, n, t, vectors)
    ids, offsets = _torch(ids), _torch(offsets)
    table, nw, nb = (_torch(rng.standard_normal(s).astype(np.float32)) for s in ((vectors, dim), (dim,), (dim,)))
    w, b = (_torch(rng.standard_normal(s).astype(np.float32)) for s in ((classes, dim), (classes,)))
    targets = _torch(rng.integers(0, classes, n).astype(np.int32))
    share = torch.full((n,), 1 / n, device="cuda")

    def step(stream=None):
        k = dict(stream=stream)
        x = pk.head_embed(table, ids, offsets, 0.2, **k)
        y, mean, rstd = pk.head_layer_norm(x, nw, nb, **k)
        loss, lse = pk.head_cross_entropy(y, w, targets, b, **k)
        gy, gw, gb = pk.head_cross_entropy_grad(share, y, w, targets, lse, b, **k)
        gx, gnw, gnb = pk.head_layer_norm_grad(gy, x, nw, mean, rstd, **k)
        return [loss, gw, gb, gnw, gnb, pk.head_embed_grad(gx, ids, vectors, offsets, 0.2, **k)]

    want = [a.clone() for a in step()]
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    got = step(other)
    other.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    params, states = [table.clone(), w.clone()], None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for k in range(4):
        table.mul_(1.5)
        want = [a.clone() for a in step()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), k
    states = [pk.head_adamw_state(p) for p in params]
    fresh = [(p.clone(), pk.head_adamw_state(p)) for p in params]
    pk.head_adamw(params, [want[5], want[1]], states, 1, 1e-3, stream=other)
    other.synchronize()
    pk.head_adamw([p for p, _ in fresh], [want[5], want[1]], [s for _, s in fresh], 1, 1e-3)
    assert all(torch.equal(p, q) for p, (q, _) in zip(params, fresh))


@pytest.mark.gpu
def test_python_refuses_tensors_that_do_not_fit():
    import torch
    x, w = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    ids = torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in (lambda: pk.head_layer_norm(x.double(), w), lambda: pk.head_layer_norm(x.T, w), lambda: pk.head_layer_norm(x, w[:7]),
                 lambda: pk.head_layer_norm(x, w.bfloat16()), lambda: pk.head_layer_norm(x[0], w), lambda: pk.head_layer_norm(x, w, w.cpu()),
                 lambda: pk.head_embed(x, ids.long()), lambda: pk.head_embed(x, ids, torch.zeros(2, dtype=torch.int64, device="cuda")),
                 lambda: pk.head_embed(x, ids.T), lambda: pk.head_embed(x, ids[None]), lambda: pk.head_embed(x[:1].expand(4, 8), ids),
                 lambda: pk.head_embed_grad(x[:3], ids, 5), lambda: pk.head_cross_entropy(x, x.bfloat16(), t),
                 lambda: pk.head_cross_entropy(x, x[:, :7], t), lambda: pk.head_cross_entropy(x, x, t.long()),
                 lambda: pk.head_cross_entropy(x, x, t[:3]), lambda: pk.head_cross_entropy(x, x, t, w),
                 lambda: pk.head_adamw([x], [x[:3]], [pk.head_adamw_state(x)], 1, 0.1),
                 lambda: pk.head_adamw([x.bfloat16()], [x], [pk.head_adamw_state(x)], 1, 0.1),
                 lambda: pk.head_adamw([x, x], [x, x.bfloat16()], [pk.head_adamw_state(x)] * 2, 1, 0.1),
                 lambda: pk.head_adamw([x, x], [x, x], [pk.head_adamw_state(x), pk.head_adamw_state(x, 8)], 1, 0.1)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(pk.HeadError):
        pk.head_layer_norm(x, w, eps=-1.0)
    with pytest.raises(pk.HeadError):
        pk.head_adamw([x], [x], [pk.head_adamw_state(x)], 0, 0.1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,bits", [("float32", 32), ("bfloat16", 8)])
def test_a_head_over_a_forest_learns_other_labels(dtype, bits):
    """Labels that the forest was not made for, but that its leaves tell: the loss falls far below that of guessing, and the
    trained head, served by the framework's linear kernels, gives them back."""
    import torch
    import workloads as wl
    w = wl.make_workload("c1")
    model = pk.forest_load(w.forest)
    X = _torch(w.make_x(1000))
    leaves = model.predict_leaves(X)
    classes = 6
    targets = (leaves[:, 0] % classes).int().contiguous()
    head = pk.LeafHead(w.forest.tree_offset, classes, dim=32, dtype=getattr(torch, dtype), bits=bits, seed=4)
    first = last = None
    for _ in range(80):
        last = head.train_step(leaves, targets, rate=2e-2).item()
        first = last if first is None else first
    assert first > 1.2 and last < 0.4 * first
    probabilities, labels = head.predict(leaves)
    torch.cuda.synchronize()
    assert (labels == targets).float().mean() > 0.9
    assert torch.allclose(probabilities.sum(1), torch.ones(1000, device="cuda"), atol=1e-5)
    losses = head.losses(leaves, targets)
    picked = torch.log(probabilities.gather(1, targets.long()[:, None])[:, 0])
    assert (losses + picked).abs().max() < (0.3 if dtype == "bfloat16" else 1e-4)    # logits of some tens, rounded operands
    model.close()
