"""The head's layers and head_clip where their kernels change their ways: the largest tiles with rows, columns and sums that end inside them, and
what a call launches, which is asked for without a GPU.

Tolerances are bounds on rounding as in test_head_layers.py, element by element: n float32 terms differ from their exact sum by at most n * 2^-24 *
(sum of their magnitudes), and some more where a bias is added or parts are joined; a bfloat16 result by up to 2^-8 of itself; activations and slopes of
bfloat16 values are right to 2^-13, and slopes are at most 1.13.  References are computed in float64, on the GPU, by the formulas of head.h.
"""
import math
import os
import re

import pytest

import paper_2301_13441_amd as pk
from paper_2301_13441_amd import head_binding as hb

U = 2.0 ** -24
TINY = 1e-37
NEAR = {"float32": U, "bfloat16": 2.0 ** -8}  # what rounding to a type may change, relative to the value


def _within(got, want, bound, what=""):
    import torch
    off, bound = (got.double() - want).abs(), bound + TINY
    assert got.shape == want.shape, what
    assert (off <= bound).all(), (what, (off / bound).max().item(), torch.nonzero(~(off <= bound))[0].tolist())


def _act(name, x):
    import torch
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return x * torch.special.erfc(-x / math.sqrt(2)) / 2
    return x


def _slope(name, x):
    import torch
    if name == "silu":
        s = torch.sigmoid(x)
        return s + x * s * (1 - s)
    if name == "gelu":
        return torch.special.erfc(-x / math.sqrt(2)) / 2 + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(x)


def _act_off(name, x, dtype):
    if name is None:
        return _zeros(x)
    return _act(name, x).abs() * (2.0 ** -13 if dtype == "bfloat16" else U * (16 + 2 * x * x))


def _slope_off(name, x, dtype):
    return _zeros(x) if name is None else _zeros(x) + (2.0 ** -13 if dtype == "bfloat16" else 2.0 ** -19)


def _zeros(x):
    return x.new_zeros(x.shape)


def _z(x, w, b):
    """z and how far a float32 sum may be from it."""
    z, magnitude = x.double() @ w.double().T, x.double().abs() @ w.double().abs().T
    if b is not None:
        z, magnitude = z + b.double(), magnitude + b.double().abs()
    return z, (x.shape[1] + 64) * U * magnitude


def _check_forward(got, kept, x, w, b, act, residual, scale, gated, dtype):
    near = NEAR[dtype]
    z, off = _z(x, w, b)
    if kept is not None:
        _within(kept, z, off * (1 + near) + near * z.abs(), "z")
    if gated:
        (gate, value), (gate_off, value_off) = z.chunk(2, 1), off.chunk(2, 1)
        a, a_off = _act(act, gate), 1.13 * gate_off + _act_off(act, gate, dtype)
        want = a * value
        off = a_off * value.abs() + (a.abs() + a_off) * value_off + 4 * U * want.abs()
    else:
        rest = 0 if residual is None else residual.double()
        part = scale * _act(act, z)
        want = part + rest
        off = abs(scale) * (1.13 * off + _act_off(act, z, dtype)) + 4 * U * (part.abs() + (0 if residual is None else rest.abs()))
    _within(got, want, off * (1 + near) + near * want.abs(), "y")


def _check_gradients(got, grad, x, w, z, act, scale, gated, dtype):
    near, g, z = NEAR[dtype], grad.double(), None if z is None else z.double()
    if gated:
        import torch
        gate, value = z.chunk(2, 1)
        dz = torch.cat([g * value * _slope(act, gate), g * _act(act, gate)], 1)
        off = torch.cat([(g * value).abs() * (_slope_off(act, gate, dtype) + 4 * U * _slope(act, gate).abs()),
                         g.abs() * (_act_off(act, gate, dtype) + 2 * U * _act(act, gate).abs())], 1)
    elif act is None:
        dz, off = g, _zeros(g)
    else:
        dz = g * _slope(act, z)
        off = g.abs() * (_slope_off(act, z, dtype) + 2 * U * _slope(act, z).abs())
    if got[2] is not None:
        _within(got[2], scale * dz.sum(0), abs(scale) * (off.sum(0) + (len(dz) + 64) * U * dz.abs().sum(0)) + 2 * U * (scale * dz.sum(0)).abs(), "bias")
    off = off + near * (dz.abs() + off)  # dz is rounded to the type before it is multiplied
    size = dz.abs() + off
    for t, want, o, m, n, what in ((got[0], dz @ w.double(), off @ w.double().abs(), size @ w.double().abs(), dz.shape[1], "x"),
                                   (got[1], dz.T @ x.double(), off.T @ x.double().abs(), size.T @ x.double().abs(), len(dz), "weight")):
        want = scale * want
        _within(t, want, abs(scale) * (o + (n + 64) * U * m) * (1 + near) + (near + 2 * U) * want.abs(), what)


def _normal(seed, *shape, dtype="float32", scale=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(getattr(torch, dtype))


# ---------------------------------------------------------------- no GPU needed

def test_testing_header_declares_what_the_library_exports():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "head_testing.h")).read()
    code = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    assert set(re.findall(r"\b(head_[a-z_]+)\s*\(", code)) == set(hb.HEAD_TESTING_EXPORTS)
    assert re.findall(r"\b(\w+)[,;]", code[code.index("struct"):code.index("} head_layer_launch_t")]) == [name for name, _ in hb._LayerLaunch._fields_]
    lib = hb._lib()
    assert all(hasattr(lib, name) for name in hb.HEAD_TESTING_EXPORTS)
    for bad, code in (((0, 8, 8), -1), ((-1, 8, 8), -1), ((4, 0, 8), -1), ((4, 8, 0), -1), ((4, 16385, 8), -7), ((4, 8, 10 ** 9 + 1), -7)):
        with pytest.raises(pk.HeadError) as e:
            hb.head_layer_launch(*bad)
        assert e.value.code == code
    assert lib.head_layer_launch(None, 0, hb._LayerLaunch()) == lib.head_layer_launch(hb._Layer(0, 0, 4, 8, 8, 0, 8, 0, 8, None), 0, None) == -1


# Layers of bfloat16 values whose forward and gradients all go in tiles of 256: rows, columns and sums that end inside one and that fill it; widths
# that are whole in 16 bytes, in what a lane stores, and not; sums in one part and in three.
LARGE = [(False, 2049, 2049, 4101), (False, 4099, 2051, 2056), (False, 2049, 4099, 2051), (False, 4096, 4096, 4096),
         (True, 2049, 2051, 2051), (True, 4099, 2052, 1028), (True, 4096, 4096, 2048)]


@pytest.mark.parametrize("gated,n,dim,outs", LARGE)
def test_these_layers_go_in_the_largest_tiles(gated, n, dim, outs):
    """Whatever the rule that chooses tiles becomes, the shapes of the test below have to take the largest."""
    s = hb.head_layer_launch(n, dim, outs, "bfloat16", gated)
    assert (s["few"], s["tile"], s["to_x_tile"], s["to_weight_tile"]) == (0, 256, 256, 256), s


# Gated layers and the tile that was fastest by 8 % or more, z kept, of 64 x 128, 128 and 256 results.
FASTEST = [("bfloat16", 15_000, 1024, 4096, 256), ("bfloat16", 16_384, 1024, 4096, 256), ("bfloat16", 16_385, 1024, 4096, 256), ("bfloat16", 33_000, 512, 2048, 256),
           ("bfloat16", 8192, 2048, 1024, 256), ("bfloat16", 4096, 512, 2048, 256), ("bfloat16", 1000, 1024, 4096, 128), ("bfloat16", 2048, 512, 256, 64),
           ("bfloat16", 4096, 64, 128, 64), ("float32", 8192, 2048, 1024, 128), ("float32", 4096, 512, 2048, 128), ("float32", 16_384, 512, 2048, 128),
           ("float32", 1000, 1024, 4096, 128), ("float32", 4096, 64, 128, 64), ("float32", 1000, 128, 500, 64)]


@pytest.mark.parametrize("dtype,n,dim,outs,tile", FASTEST)
def test_a_gated_layer_goes_in_the_fastest_tiles(dtype, n, dim, outs, tile):
    s = hb.head_layer_launch(n, dim, outs, dtype, gated=True)
    assert (s["few"], s["tile"], s["splits"]) == (0, tile, 1), s


# Gated layers in tiles of 64 x 128 and 128 x 128.
GATED = [("bfloat16", 1003, 1027, 4093, 128), ("bfloat16", 9001, 336, 332, 128), ("float32", 4090, 515, 1021, 128), ("float32", 4090, 512, 1016, 128),
         ("bfloat16", 2050, 515, 257, 64), ("bfloat16", 2050, 512, 256, 64), ("float32", 4099, 67, 131, 64), ("float32", 4099, 64, 136, 64)]


@pytest.mark.parametrize("dtype,n,dim,outs,tile", GATED)
def test_these_gated_layers_go_in_these_tiles(dtype, n, dim, outs, tile):
    s = hb.head_layer_launch(n, dim, outs, dtype, gated=True)
    assert (s["few"], s["tile"], s["splits"]) == (0, tile, 1), s


# The kernel for few rows has a workgroup of 512 lanes for each 16 columns, and a grid's axis fewer than 2^32 lanes.
MANY = [("bfloat16", False, 140_000_003, 8), ("float32", False, 140_000_000, 3), ("bfloat16", True, 134_217_729, 7)]


@pytest.mark.parametrize("dtype,gated,outs,dim", MANY)
def test_few_rows_of_very_many_columns_fit_a_grid(dtype, gated, outs, dim):
    for n in (1, 16, 64):
        for columns in (outs, 10 ** 9 // (1 + gated)):
            s = hb.head_layer_launch(n, dim, columns, dtype, gated)
            assert s["few"] == 0 and s["tile"] and s["splits"] == 1 and s["to_x_tile"] == 0, s
        assert hb.head_layer_launch(n, dim, 4096, dtype, gated)["few"] == 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,gated,outs,dim", MANY)
def test_few_rows_of_very_many_columns(dtype, gated, outs, dim):
    import torch
    halves = 1 + gated
    g = torch.Generator(device="cuda").manual_seed(dim)
    w = torch.randn(halves * outs, dim, generator=g, device="cuda", dtype=getattr(torch, dtype))
    x = _normal(1, 1, dim, dtype=dtype)
    y = pk.head_gated(x, w, None, "gelu") if gated else pk.head_linear(x, w, None, "gelu")
    assert y.shape == (1, outs)
    at = torch.randint(0, outs, (200_000,), generator=g, device="cuda")
    at = torch.cat([at, torch.arange(5, device="cuda"), outs - 1 - torch.arange(5, device="cuda"), torch.arange(134_217_700, 134_217_729, device="cuda")])
    picked = torch.cat([w[at], w[at + outs]]) if gated else w[at]
    _check_forward(y[:, at], None, x, picked, None, "gelu", None, 1.0, gated, dtype)


# Layers of few rows that are not whole in 16 bytes, and how they were fastest by 15 % or more: parts of the kernel for few rows, which reads them value by
# value, or 0 for tiles.  `apart`: values between a row's end and the next row.
ODD = [("bfloat16", False, 1, 58, 256, 0, 1), ("bfloat16", False, 1, 2042, 8192, 0, 0), ("bfloat16", False, 16, 4090, 16_384, 0, 0), ("bfloat16", False, 5, 2048, 8192, 2, 0),
       ("bfloat16", False, 1, 249, 16_384, 0, 1), ("bfloat16", False, 16, 4089, 16_384, 0, 0), ("bfloat16", False, 16, 1018, 1000, 0, 4), ("bfloat16", False, 64, 8186, 64, 0, 0),
       ("bfloat16", False, 1, 8186, 64, 0, 16), ("float32", False, 16, 2041, 8192, 0, 0), ("float32", False, 1, 1017, 4096, 0, 1), ("float32", False, 64, 4089, 1000, 0, 0),
       ("bfloat16", False, 64, 90, 262_144, 0, 0), ("bfloat16", False, 16, 7, 32_768, 0, 1), ("float32", False, 1, 3, 32_768, 0, 1),
       ("bfloat16", True, 1, 2042, 8192, 0, 0), ("bfloat16", True, 1, 58, 128, 0, 1), ("float32", True, 64, 2041, 4096, 0, 0), ("float32", True, 5, 329, 45, 0, 1)]


@pytest.mark.parametrize("dtype,gated,n,dim,outs,apart,few", ODD)
def test_few_odd_rows_go_the_fastest_way(dtype, gated, n, dim, outs, apart, few):
    s = hb.head_layer_launch(n, dim, outs, dtype, gated, weight_stride=dim + apart)
    assert s["few"] == few and (few > 0) == (s["tile"] == 0), s


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,gated,n,dim,outs,apart,few", ODD)
def test_few_odd_rows(dtype, gated, n, dim, outs, apart, few):
    columns = outs * (1 + gated)
    x, b, rest = _normal(n, n, dim, dtype=dtype), _normal(outs, columns), _normal(1, n, outs, dtype=dtype)
    w = _normal(dim, columns, dim + apart, dtype=dtype, scale=dim ** -0.5)[:, :dim]
    y, z = pk.head_gated(x, w, b, "silu", keep=True) if gated else pk.head_linear(x, w, b, "silu", rest, 0.5, keep=True)
    _check_forward(y, z, x, w, b, "silu", rest, 0.5, gated, dtype)


# Rows that begin further apart than products read them where they are, 2 MB and 256 bytes, just as far, and in bfloat16 at odd values.
FAR = [(dtype, apart) for dtype, apart in (("float32", 1), ("float32", 0), ("bfloat16", 1), ("bfloat16", 2), ("bfloat16", 0))]


def _far_stride(dtype, apart):
    return ((1 << 21) + 256) // (4 if dtype == "float32" else 2) + apart


@pytest.mark.parametrize("dtype,apart", FAR)
def test_rows_too_far_apart_are_copied_first(dtype, apart):
    stride = _far_stride(dtype, apart)
    for gated in (False, True):
        s = hb.head_layer_launch(70, 41, 33, dtype, gated, x_stride=stride, weight_stride=stride)
        assert s["few"] == 0 and s["copies_x"] == s["copies_weight"] == (apart > 0), s
        s = hb.head_layer_launch(70, 40, 33, dtype, gated, x_stride=stride, weight_stride=40)
        assert s["copies_x"] == (apart > 0) and not s["copies_weight"], s


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,apart", FAR)
def test_rows_that_lie_megabytes_apart(dtype, apart):
    """All operands so, with NaN between their rows and behind the last."""
    import torch
    stride = _far_stride(dtype, apart)

    def far(t):
        whole = torch.full((len(t), stride), math.nan, device="cuda", dtype=t.dtype)
        whole[:, 2:2 + t.shape[1]] = t
        return whole[:, 2:2 + t.shape[1]]

    for n, dim, outs in ((70, 41, 34), (5, 40, 33)):
        x, b, rest, grad = far(_normal(1, n, dim, dtype=dtype)), _normal(2, 2 * outs), far(_normal(3, n, outs, dtype=dtype)), far(_normal(4, n, outs, dtype=dtype, scale=0.1))
        w = far(_normal(5, 2 * outs, dim, dtype=dtype, scale=dim ** -0.5))
        for act in ("silu", None):
            y, z = pk.head_linear(x, w[:outs], b[:outs], act, rest, 0.5, keep=True)
            _check_forward(y, z, x, w[:outs], b[:outs], act, rest, 0.5, False, dtype)
            got = pk.head_linear_grad(grad, x, w[:outs], far(z), act, 0.5)
            _check_gradients(got, grad, x, w[:outs], z, act, 0.5, False, dtype)
            y, z = pk.head_gated(x, w, b, act, keep=True)
            _check_forward(y, z, x, w, b, act, None, 1.0, True, dtype)
            _check_gradients(pk.head_gated_grad(grad, x, w, far(z), act), grad, x, w, z, act, 1.0, True, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [False, True])
def test_float32_gradients_of_the_most_outputs(gated):
    """Gated, rows of the gradient of z begin just as far apart as products read them."""
    n, dim, outs, dtype = 70, 9, 262_144, "float32"
    columns = outs * (1 + gated)
    x, w = _normal(1, n, dim), _normal(2, columns, dim, scale=dim ** -0.5)
    z, grad = _normal(3, n, columns), _normal(4, n, outs, scale=0.1)
    got = pk.head_gated_grad(grad, x, w, z, "silu") if gated else pk.head_linear_grad(grad, x, w, z, "silu")
    _check_gradients(got, grad, x, w, z, "silu", 1.0, gated, dtype)


# ---------------------------------------------------------------- tiles

@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,dim,outs,tile", GATED)
def test_gated_layers_in_each_tile(dtype, n, dim, outs, tile):
    import torch
    x, w, b = _normal(n, n, dim, dtype=dtype), _normal(dim, 2 * outs, dim, dtype=dtype, scale=dim ** -0.5), _normal(outs, 2 * outs)
    for act, bias in (("silu", b), ("gelu", None), (None, b)):
        y, z = pk.head_gated(x, w, bias, act, keep=True)
        _check_forward(y, z, x, w, bias, act, None, 1.0, True, dtype)
        assert torch.equal(pk.head_gated(x, w, bias, act), y)


@pytest.mark.gpu
@pytest.mark.parametrize("gated,n,dim,outs", LARGE)
def test_layers_in_the_largest_tiles(gated, n, dim, outs):
    import torch
    dtype, columns = "bfloat16", outs * (2 if gated else 1)
    x, w = _normal(n, n, dim, dtype=dtype), _normal(dim, columns, dim, dtype=dtype, scale=dim ** -0.5)
    b, residual, grad = _normal(outs, columns), _normal(1, n, outs, dtype=dtype), _normal(2, n, outs, dtype=dtype, scale=0.1)
    for act, bias, rest, scale in (("gelu", b, None, 1.0), ("silu", None, residual, 0.5), (None, b, residual, 0.75)):
        if gated:
            call = lambda keep: pk.head_gated(x, w, bias, act, keep=keep)  # noqa: E731
        else:
            call = lambda keep: pk.head_linear(x, w, bias, act, rest, scale, keep=keep)  # noqa: E731
        y, z = call(True)
        _check_forward(y, z, x, w, bias, act, rest, scale, gated, dtype)
        assert torch.equal(call(False), y)
        if gated:
            take = lambda: pk.head_gated_grad(grad, x, w, z, act, bias=bias is not None)  # noqa: E731
        else:
            take = lambda: pk.head_linear_grad(grad, x, w, z if act else None, act, scale, bias=bias is not None)  # noqa: E731
        got = take()
        _check_gradients(got, grad, x, w, z, act, 1.0 if gated else scale, gated, dtype)
        assert all(p is None or torch.equal(p, q) for p, q in zip(take(), got))  # the same call gives the same bits


# ---------------------------------------------------------------- clipping

@pytest.mark.gpu
@pytest.mark.parametrize("n", [100, 300_001])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_clip_by_a_share_that_float32_does_not_hold(dtype, n):
    """Values near the end of float32 and limits far below them: the share is subnormal in float32, or below that, and the results are ordinary."""
    import torch
    for limit in (1e-6, 1e-20, 1e-33, 2.0 ** -100 * 3e38):
        g = _normal(n, n).clamp_(-4, 4).mul_(5e37).to(getattr(torch, dtype))
        norm64 = g.double().square().sum().sqrt()
        want = g.double() * (limit / norm64)
        for in_place in (False, True):
            norm, (got,) = pk.head_clip([g], limit, in_place=in_place)
            assert norm.item() == math.inf or abs(norm.item() / norm64.item() - 1) <= 5 * U
            # the norm's and the factor's rounding, the product's and that to the type; results below the smallest normal ones in steps of the type's last
            off = (got.double() - want).abs()
            assert (off <= (NEAR[dtype] + 8 * U) * want.abs() + 2.0 ** -125 * NEAR[dtype]).all(), (limit, in_place, (off / want.abs()).max().item())


@pytest.mark.gpu
@pytest.mark.parametrize("n", [100, 300_001])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_norm_alone(dtype, n):
    """The C call whose tensors have no results: nothing but the norm is written, whatever the limit is."""
    import torch
    lib, tensors = hb._lib(), [_normal(1, n, dtype=dtype), _normal(2, 33), _normal(3, 0)]
    before = [t.clone() for t in tensors]
    want = math.sqrt(sum(t.double().square().sum().item() for t in tensors))
    rows = (hb._ClipTensor * 3)(*(hb._ClipTensor(t.data_ptr() or None, None, t.numel(), int(t.dtype == torch.bfloat16)) for t in tensors))
    size = lib.head_clip_bytes(rows, 3)
    assert (size > 0) == (n > 100)
    work, norm = torch.empty(max(16, size), dtype=torch.uint8, device="cuda"), torch.full((3,), -1.0, device="cuda")
    for limit in (0.5, 1e9, math.inf):
        norm.fill_(-1)
        assert lib.head_clip(rows, 3, limit, norm.data_ptr() + 4, work.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
        got = norm.tolist()
        assert abs(got[1] - want) <= 5 * U * want and got[0] == got[2] == -1
        assert all(torch.equal(a, b) for a, b in zip(tensors, before))
