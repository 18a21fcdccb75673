"""ctypes binding of the trainable head over leaf ids, same names as include/head.h (argument checks and marshalling only;
every step runs in the HIP kernels).

All tensors of a call are on one device, the current one.  A 2-D tensor may have any row stride of at least its row's length;
its rows' elements are adjacent.  Results are new tensors (of the stream's pool) unless the call says that it updates
its arguments.  `stream`: the torch stream to work on, the current one by default; a tensor that belongs to another stream
is kept from being reused until this one is done with it, but the streams are the caller's to order.

Autograd records none of the calls: a gradient is a call of its own (`*_grad`).  So that none is lost without a word, tensors that require a
gradient are refused unless recording is off (torch.no_grad(), an autograd Function's methods), and tensors with a tangent always; head_adamw, like any
optimizer's step, takes its tensors either way.
"""
from __future__ import annotations

import contextlib
import ctypes
import warnings
from typing import NamedTuple, Optional

from .binding import entry_point, load_library

_p = ctypes.c_void_p
_i32, _i64, _u32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32
_f32, _f64 = ctypes.c_float, ctypes.c_double

HEAD_EXPORTS = ["head_embed", "head_embed_grad_bytes", "head_embed_grad", "head_layer_norm", "head_layer_norm_grad_bytes",
                "head_layer_norm_grad", "head_cross_entropy_bytes", "head_cross_entropy_grad_bytes", "head_cross_entropy",
                "head_cross_entropy_grad", "head_adamw", "head_adamw_values", "head_linear_bytes", "head_linear", "head_linear_grad_bytes",
                "head_linear_grad", "head_gated_bytes", "head_gated", "head_gated_grad_bytes", "head_gated_grad", "head_clip_bytes",
                "head_clip", "head_strerror"]
HEAD_TESTING_EXPORTS = ["head_layer_launch"]
ACTIVATIONS = {None: 0, "relu": 1, "gelu": 2, "silu": 3}  # HEAD_IDENTITY, HEAD_RELU, HEAD_GELU, HEAD_SILU
BLOCK = 128  # HEAD_BLOCK


class _Ids(ctypes.Structure):
    _fields_ = [("n_rows", _i64), ("n_ids", _i64), ("n_vectors", _i64), ("ids", _p), ("ids_stride", _i64), ("offset", _p)]


class _Classes(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("n_rows", _i64), ("dim", _i64), ("n_classes", _i64), ("hidden", _p), ("hidden_stride", _i64),
                ("weight", _p), ("weight_stride", _i64), ("bias", _p), ("target", _p)]


class _AdamwTensor(ctypes.Structure):
    _fields_ = [("param", _p), ("grad", _p), ("m", _p), ("v", _p), ("m_scale", _p), ("v_scale", _p), ("copy", _p), ("n", _i64)]


class _AdamwRule(ctypes.Structure):
    _fields_ = [("grad_dtype", _i32), ("bits", _i32), ("step", _i64), ("rate", _f64), ("beta1", _f64), ("beta2", _f64),
                ("eps", _f64), ("decay", _f64), ("seed", _u32)]


class _Layer(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("activation", _i32), ("n_rows", _i64), ("dim", _i64), ("n_outputs", _i64), ("x", _p), ("x_stride", _i64),
                ("weight", _p), ("weight_stride", _i64), ("bias", _p)]


class _ClipTensor(ctypes.Structure):
    _fields_ = [("grad", _p), ("out", _p), ("n", _i64), ("dtype", _i32)]


class _LayerLaunch(ctypes.Structure):
    _fields_ = [(name, _i32) for name in ("few", "copies_x", "copies_weight", "tile", "splits", "to_x_tile", "to_x_splits", "to_weight_tile",
                                          "to_weight_splits")]


class HeadError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {code} ({_lib().head_strerror(int(code)).decode()})")
        self.code = code


_ready = None


def _lib():
    global _ready
    if _ready is not None:
        return _ready
    lib = load_library()
    ids, classes, layer, clips = (ctypes.POINTER(t) for t in (_Ids, _Classes, _Layer, _ClipTensor))
    for name, result, *args in (
            ("head_embed", _i32, ids, _i32, _i64, _p, _i64, _f32, _p, _p),
            ("head_embed_grad_bytes", _i64, ids, _i32, _i64),
            ("head_embed_grad", _i32, ids, _i32, _i64, _p, _i64, _f32, _p, _p, _p),
            ("head_layer_norm", _i32, _i32, _i64, _i64, _p, _i64, _p, _p, _f32, _p, _p, _p, _p),
            ("head_layer_norm_grad_bytes", _i64, _i32, _i64, _i64),
            ("head_layer_norm_grad", _i32, _i32, _i64, _i64, _p, _i64, _p, _i64, _p, _p, _p, _p, _p, _p, _p, _p),
            ("head_cross_entropy_bytes", _i64, classes),
            ("head_cross_entropy_grad_bytes", _i64, classes),
            ("head_cross_entropy", _i32, classes, _p, _p, _p, _p),
            ("head_cross_entropy_grad", _i32, classes, _p, _p, _p, _p, _p, _p, _p),
            ("head_adamw", _i32, ctypes.POINTER(_AdamwRule), ctypes.POINTER(_AdamwTensor), _i32, _p),
            ("head_adamw_values", _i32, ctypes.POINTER(_AdamwTensor), ctypes.POINTER(_p), ctypes.POINTER(_p), _i32, _p),
            ("head_linear_bytes", _i64, layer),
            ("head_linear", _i32, layer, _p, _i64, _f32, _p, _p, _p, _p),
            ("head_linear_grad_bytes", _i64, layer),
            ("head_linear_grad", _i32, layer, _p, _i64, _p, _i64, _f32, _p, _p, _p, _p, _p),
            ("head_gated_bytes", _i64, layer),
            ("head_gated", _i32, layer, _p, _p, _p, _p),
            ("head_gated_grad_bytes", _i64, layer),
            ("head_gated_grad", _i32, layer, _p, _i64, _p, _i64, _p, _p, _p, _p, _p),
            ("head_clip_bytes", _i64, clips, _i32),
            ("head_clip", _i32, clips, _i32, _f64, _p, _p, _p),
            ("head_layer_launch", _i32, layer, _i32, ctypes.POINTER(_LayerLaunch)),
            ("head_strerror", ctypes.c_char_p, _i32)):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = result, args
    _ready = lib
    return lib


class _Declines:
    """In the native calls' place where the extension is missing: the general way is complete without them."""
    def __getattr__(self, name):
        return lambda *args: None


_calls = None


def _native():
    """The calls as one native call each (csrc/head_call.cpp), for plain contiguous tensors on the current stream; None from one of
    them: it goes the general way."""
    global _calls
    if _calls is None:
        lib = _lib()
        try:
            import torch  # noqa: F401 - the extension is linked against its libraries
            from . import _head_call
            _head_call.bind(*(entry_point(getattr(lib, name)) for name in (
                "head_embed", "head_embed_grad_bytes", "head_embed_grad", "head_layer_norm", "head_layer_norm_grad_bytes",
                "head_layer_norm_grad", "head_cross_entropy_bytes", "head_cross_entropy", "head_cross_entropy_grad_bytes",
                "head_cross_entropy_grad", "head_adamw", "head_adamw_values", "head_linear_bytes", "head_linear", "head_linear_grad_bytes",
                "head_linear_grad", "head_gated_bytes", "head_gated", "head_gated_grad_bytes", "head_gated_grad", "head_clip_bytes",
                "head_clip")))
            _calls = _head_call
        except ImportError as exc:
            warnings.warn(f"the native calls of the head cannot be imported ({exc}): calls take some microseconds more; "
                          "build them with `python -m paper_2301_13441_amd.build`", RuntimeWarning, stacklevel=4)
            _calls = _Declines()
    return _calls


def _done(got, what: str):
    """What a native call returned, which did not decline."""
    if type(got) is int:
        raise HeadError(got, what)
    return got


def _check(code: int, what: str) -> int:
    if code < 0:
        raise HeadError(code, what)
    return code


def _dtype(t, what: str) -> int:
    import torch
    if t.dtype == torch.float32:
        return 0
    if t.dtype == torch.bfloat16:
        return 1
    raise ValueError(f"{what} must be float32 or bfloat16, not {t.dtype}")


def _tensor(t, what: str, dtype=None, shape=None, like=None):
    """`t` as a device tensor of that type and shape (None in a shape: any length) whose rows' elements are adjacent."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if like is not None and t.device != like.device:
        raise ValueError(f"{what} is on {t.device}, the other tensors on {like.device}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, not {t.dtype}")
    if shape is not None and (t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape))):
        raise ValueError(f"{what} must have shape {list(shape)}, not {list(t.shape)}")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient, which this call does not record: make it under torch.no_grad(), and take the gradient "
                         "from the operator's own call for it")
    if t.is_floating_point() and torch.autograd.forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{what} has a tangent, which this call does not carry on")
    if t.is_contiguous() or (t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1) and t.stride(0) >= t.shape[1]):
        return t
    raise ValueError(f"{what} must be contiguous" + (" along its rows, which must not overlap" if t.dim() == 2 else ""))


def _stride(t) -> int:
    return max(t.stride(0), t.shape[1]) if t.dim() == 2 else 1


@contextlib.contextmanager
def _other_stream(stream, tensors):
    """Work on `stream`: new tensors come from its pool, and `tensors` of other streams outlive its use of them."""
    import torch
    with torch.cuda.stream(stream):
        yield stream.cuda_stream
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


class _CurrentStream:
    """The same for the current stream, whose tensors they are."""
    def __init__(self, device):
        self.device = device

    def __enter__(self):
        import torch
        return torch.cuda.current_stream(self.device).cuda_stream

    def __exit__(self, *args):
        return False


def _on(stream, first, tensors):
    import torch
    if first.device.index != torch.cuda.current_device():
        raise ValueError(f"the tensors are on {first.device}, but the current device is {torch.cuda.current_device()}")
    if stream is None:
        return _CurrentStream(first.device)
    if stream.device != first.device:
        raise ValueError(f"the tensors are on {first.device}, but the stream is on {stream.device}")
    return _other_stream(stream, tensors)


def _workspace(nbytes: int, like):
    import torch
    return torch.empty(nbytes, dtype=torch.uint8, device=like.device) if nbytes else None


def _at(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _ids(ids, offsets, n_vectors: int, like):
    import torch
    _tensor(ids, "ids", torch.int32, like=like)
    if ids.dim() not in (1, 2):
        raise ValueError(f"ids must have shape [n_rows, n_ids] or [n_rows], not {list(ids.shape)}")
    n_ids = ids.shape[1] if ids.dim() == 2 else 1
    if offsets is not None:
        _tensor(offsets, "offsets", torch.int64, (n_ids,), like=like)
    return _Ids(ids.shape[0], n_ids, n_vectors, ids.data_ptr(), _stride(ids), _at(offsets))


def head_embed(table, ids, offsets=None, scale: float = 1.0, stream=None):
    """out[r] = scale * sum_t table[ids[r, t] + offsets[t]].

    table: [n_vectors, dim] float32 or bfloat16.  ids: int32 [n_rows, n_ids], or [n_rows] for a lookup of one vector each.
    offsets: int64 [n_ids] or None (zeros); with the ids of Forest.predict_leaves, the forest's tree_offset[:-1].  A
    negative id, or one without a vector, adds nothing.  Returns [n_rows, dim] of the table's type.
    """
    if stream is None:
        got = _native().embed(table, ids, offsets, scale)
        if got is not None:
            return _done(got, "head_embed")
    import torch
    _tensor(table, "table", shape=(None, None))
    dtype = _dtype(table, "table")
    desc = _ids(ids, offsets, table.shape[0], table)
    with _on(stream, table, (table, ids, offsets)) as s:
        out = torch.empty((ids.shape[0], table.shape[1]), dtype=table.dtype, device=table.device)
        _check(_lib().head_embed(desc, dtype, table.shape[1], table.data_ptr(), _stride(table), scale, out.data_ptr(), s), "head_embed")
    return out


def head_embed_grad(grad, ids, n_vectors: int, offsets=None, scale: float = 1.0, stream=None):
    """The gradient of head_embed's table: [n_vectors, dim] of the type of grad, [n_rows, dim]; zero for vectors that no id
    stands for."""
    if stream is None:
        got = _native().embed_grad(grad, ids, n_vectors, offsets, scale)
        if got is not None:
            return _done(got, "head_embed_grad")
    import torch
    _tensor(grad, "grad", shape=(None, None))
    dtype = _dtype(grad, "grad")
    desc = _ids(ids, offsets, n_vectors, grad)
    if ids.shape[0] != grad.shape[0]:
        raise ValueError(f"ids has {ids.shape[0]} rows, grad {grad.shape[0]}")
    lib = _lib()
    nbytes = _check(lib.head_embed_grad_bytes(desc, dtype, grad.shape[1]), "head_embed_grad")
    with _on(stream, grad, (grad, ids, offsets)) as s:
        out = torch.empty((n_vectors, grad.shape[1]), dtype=grad.dtype, device=grad.device)
        work = _workspace(nbytes, grad)
        _check(lib.head_embed_grad(desc, dtype, grad.shape[1], grad.data_ptr(), _stride(grad), scale, out.data_ptr(), _at(work), s),
               "head_embed_grad")
    return out


def head_layer_norm(x, weight, bias=None, eps: float = 1e-5, stream=None):
    """Layer norm of the rows of x, [n_rows, dim] float32 or bfloat16, with weight and bias (or None) float32 [dim].
    Returns (y, mean, rstd): y like x, mean and rstd float32 [n_rows], which the gradient needs."""
    if stream is None:
        got = _native().layer_norm(x, weight, bias, eps)
        if got is not None:
            return _done(got, "head_layer_norm")
    import torch
    _tensor(x, "x", shape=(None, None))
    dtype, (n, dim) = _dtype(x, "x"), x.shape
    _tensor(weight, "weight", torch.float32, (dim,), x)
    if bias is not None:
        _tensor(bias, "bias", torch.float32, (dim,), x)
    with _on(stream, x, (x, weight, bias)) as s:
        y = torch.empty((n, dim), dtype=x.dtype, device=x.device)
        mean = torch.empty(n, dtype=torch.float32, device=x.device)
        rstd = torch.empty(n, dtype=torch.float32, device=x.device)
        _check(_lib().head_layer_norm(dtype, n, dim, x.data_ptr(), _stride(x), weight.data_ptr(), _at(bias), eps, y.data_ptr(),
                                      mean.data_ptr(), rstd.data_ptr(), s), "head_layer_norm")
    return y, mean, rstd


def head_layer_norm_grad(grad, x, weight, mean, rstd, stream=None):
    """The gradients of head_layer_norm from grad, that of y.  Returns (grad_x, grad_weight, grad_bias): grad_x like x, the others
    float32 [dim]."""
    if stream is None:
        got = _native().layer_norm_grad(grad, x, weight, mean, rstd)
        if got is not None:
            return _done(got, "head_layer_norm_grad")
    import torch
    _tensor(x, "x", shape=(None, None))
    dtype, (n, dim) = _dtype(x, "x"), x.shape
    _tensor(grad, "grad", x.dtype, (n, dim), x)
    _tensor(weight, "weight", torch.float32, (dim,), x)
    _tensor(mean, "mean", torch.float32, (n,), x)
    _tensor(rstd, "rstd", torch.float32, (n,), x)
    lib = _lib()
    nbytes = _check(lib.head_layer_norm_grad_bytes(dtype, n, dim), "head_layer_norm_grad")
    with _on(stream, x, (grad, x, weight, mean, rstd)) as s:
        grad_x = torch.empty((n, dim), dtype=x.dtype, device=x.device)
        grad_weight = torch.empty(dim, dtype=torch.float32, device=x.device)
        grad_bias = torch.empty(dim, dtype=torch.float32, device=x.device)
        work = _workspace(nbytes, x)
        _check(lib.head_layer_norm_grad(dtype, n, dim, grad.data_ptr(), _stride(grad), x.data_ptr(), _stride(x), weight.data_ptr(),
                                        mean.data_ptr(), rstd.data_ptr(), grad_x.data_ptr(), grad_weight.data_ptr(),
                                        grad_bias.data_ptr(), _at(work), s), "head_layer_norm_grad")
    return grad_x, grad_weight, grad_bias


def _classes(hidden, weight, targets, bias):
    import torch
    _tensor(hidden, "hidden", shape=(None, None))
    dtype, (n, dim) = _dtype(hidden, "hidden"), hidden.shape
    _tensor(weight, "weight", hidden.dtype, (None, dim), hidden)
    _tensor(targets, "targets", torch.int32, (n,), hidden)
    if bias is not None:
        _tensor(bias, "bias", torch.float32, (weight.shape[0],), hidden)
    return _Classes(dtype, n, dim, weight.shape[0], hidden.data_ptr(), _stride(hidden), weight.data_ptr(), _stride(weight), _at(bias),
                    targets.data_ptr())


def head_cross_entropy(hidden, weight, targets, bias=None, stream=None):
    """Softmax cross entropy of the classes' logits hidden @ weight.T + bias, which are never kept.

    hidden: [n_rows, dim], weight: [n_classes, dim], both float32 or both bfloat16.  bias: float32 [n_classes] or None.
    targets: int32 [n_rows]; a row whose target is no class (-1, say) has loss 0 and no gradient.  Returns (loss, lse),
    float32 [n_rows]: a row's loss, and the logarithm of the sum of its logits' exponentials, which the gradient needs.
    """
    if stream is None:
        got = _native().cross_entropy(hidden, weight, targets, bias)
        if got is not None:
            return _done(got, "head_cross_entropy")
    import torch
    desc = _classes(hidden, weight, targets, bias)
    lib = _lib()
    nbytes = _check(lib.head_cross_entropy_bytes(desc), "head_cross_entropy")
    with _on(stream, hidden, (hidden, weight, targets, bias)) as s:
        loss = torch.empty(hidden.shape[0], dtype=torch.float32, device=hidden.device)
        lse = torch.empty(hidden.shape[0], dtype=torch.float32, device=hidden.device)
        work = _workspace(nbytes, hidden)
        _check(lib.head_cross_entropy(desc, loss.data_ptr(), lse.data_ptr(), _at(work), s), "head_cross_entropy")
    return loss, lse


def head_cross_entropy_grad(grad_loss, hidden, weight, targets, lse, bias=None, stream=None):
    """The gradients of sum_r grad_loss[r] * loss[r] (for the mean loss: 1 / the number of rows with a target), given
    head_cross_entropy's lse for the same arguments.  Returns (grad_hidden, grad_weight, grad_bias): like hidden, like weight,
    and float32 [n_classes], None without a bias."""
    if stream is None:
        got = _native().cross_entropy_grad(grad_loss, hidden, weight, targets, lse, bias)
        if got is not None:
            return _done(got, "head_cross_entropy_grad")
    import torch
    desc = _classes(hidden, weight, targets, bias)
    n = hidden.shape[0]
    _tensor(grad_loss, "grad_loss", torch.float32, (n,), hidden)
    _tensor(lse, "lse", torch.float32, (n,), hidden)
    lib = _lib()
    nbytes = _check(lib.head_cross_entropy_grad_bytes(desc), "head_cross_entropy_grad")
    with _on(stream, hidden, (grad_loss, hidden, weight, targets, lse, bias)) as s:
        grad_hidden = torch.empty((n, hidden.shape[1]), dtype=hidden.dtype, device=hidden.device)
        grad_weight = torch.empty((weight.shape[0], hidden.shape[1]), dtype=hidden.dtype, device=hidden.device)
        grad_bias = None if bias is None else torch.empty(weight.shape[0], dtype=torch.float32, device=hidden.device)
        work = _workspace(nbytes, hidden)
        _check(lib.head_cross_entropy_grad(desc, lse.data_ptr(), grad_loss.data_ptr(), grad_hidden.data_ptr(), grad_weight.data_ptr(),
                                           _at(grad_bias), _at(work), s), "head_cross_entropy_grad")
    return grad_hidden, grad_weight, grad_bias


class AdamwState32(NamedTuple):
    """Float32 states, of the parameter's shape."""
    m: object
    v: object


class AdamwState8(NamedTuple):
    """8-bit states: codes, one for each value, and scale bytes, one for each BLOCK values (include/head.h)."""
    m: object
    m_scale: object
    v: object
    v_scale: object


def head_adamw_state(param, bits: int = 32):
    """The states of a parameter before its first step: AdamwState32 or AdamwState8."""
    import torch
    if bits == 32:
        return AdamwState32(torch.zeros_like(param, dtype=torch.float32), torch.zeros_like(param, dtype=torch.float32))
    if bits != 8:
        raise ValueError(f"bits must be 32 or 8, not {bits}")
    n = param.numel()
    code, scale = ((n,), (-(-n // BLOCK),))
    return AdamwState8(*(torch.zeros(shape, dtype=torch.uint8, device=param.device) for shape in (code, scale, code, scale)))


def _flat(t, what: str, dtype, n: int, like):
    """`t` as n adjacent values."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype or t.numel() != n or not t.is_contiguous() or t.device != like.device:
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of {n} values on {like.device}")
    return t.data_ptr()


def _state(s, k: int, n: int, like):
    """(m, v, m_scale, v_scale) as addresses."""
    import torch
    if len(s) == 2:
        return (_flat(s[0], f"m of state {k}", torch.float32, n, like), _flat(s[1], f"v of state {k}", torch.float32, n, like), None, None)
    if len(s) != 4:
        raise ValueError(f"state {k} must be (m, v) or (m, m_scale, v, v_scale)")
    blocks = -(-n // BLOCK)
    m, ms, v, vs = (_flat(t, f"{what} of state {k}", torch.uint8, count, like)
                    for t, what, count in zip(s, ("m", "m_scale", "v", "v_scale"), (n, blocks, n, blocks)))
    return m, v, ms, vs


def head_adamw(params, grads, states, step: int, rate: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
               decay: float = 0.01, copies=None, seed: int = 0, stream=None) -> None:
    """One AdamW step over all tensors; updates params, states and copies.

    params: float32, contiguous.  grads: all float32 or all bfloat16.  states: what head_adamw_state gives, of one
    kind for all.  step: 1 for the first step.  copies: None, or a bfloat16 tensor or None for each parameter, which becomes a
    copy of the new parameter.  seed: of the 8-bit states' rounding.  No tensor may be in the lists twice.
    """
    if stream is None:
        got = _native().adamw(params, grads, states, copies, step, rate, beta1, beta2, eps, decay, seed)
        if got is not None:
            _done(got, "head_adamw")
            return
    import torch
    n = len(params)
    if len(grads) != n or len(states) != n or (copies is not None and len(copies) != n):
        raise ValueError("params, grads, states and copies must be of one length")
    if n == 0:
        return
    if not isinstance(params[0], torch.Tensor) or not params[0].is_cuda:
        raise ValueError("parameter 0 must be a CUDA tensor")
    first, kind = params[0], len(states[0])
    grad_dtype = _dtype(grads[0], "grads")
    rows = (_AdamwTensor * n)()
    for k, (p, g, s) in enumerate(zip(params, grads, states)):
        count = p.numel()
        if len(s) != kind:
            raise ValueError("states must be of one kind")
        m, v, ms, vs = _state(s, k, count, first)
        copy = None if copies is None or copies[k] is None else _flat(copies[k], f"copy {k}", torch.bfloat16, count, first)
        rows[k] = _AdamwTensor(_flat(p, f"parameter {k}", torch.float32, count, first),
                               _flat(g, f"gradient {k}", grads[0].dtype, count, first), m, v, ms, vs, copy, count)
    rule = _AdamwRule(grad_dtype, 32 if kind == 2 else 8, step, rate, beta1, beta2, eps, decay, seed & 0xFFFFFFFF)
    used = [] if stream is None else [*params, *grads, *(t for s in states for t in s), *(copies or [])]
    with _on(stream, first, used) as s:
        written = [*params, *(t for s in states for t in s), *(c for c in copies or [] if c is not None)]
        torch.autograd.graph.increment_version([t for t in written if not t.is_inference()])  # what autograd has kept of them is out of date
        _check(_lib().head_adamw(rule, rows, n, s), "head_adamw")


def head_adamw_values(states, params, stream=None):
    """What 8-bit states stand for: a list of (m, v), bfloat16 tensors of the shapes of params."""
    if stream is None:
        got = _native().adamw_values(states, params)
        if got is not None:
            return _done(got, "head_adamw_values")
    import torch
    if len(states) != len(params):
        raise ValueError("states and params must be of one length")
    n = len(params)
    if n == 0:
        return []
    if not isinstance(params[0], torch.Tensor) or not params[0].is_cuda:
        raise ValueError("parameter 0 must be a CUDA tensor")
    first = params[0]
    rows, at_m, at_v = (_AdamwTensor * n)(), (_p * n)(), (_p * n)()
    for k, (s, p) in enumerate(zip(states, params)):
        if len(s) != 4:
            raise ValueError(f"state {k} is not one of 8 bits")
        m, v, ms, vs = _state(s, k, p.numel(), first)
        rows[k] = _AdamwTensor(None, None, m, v, ms, vs, None, p.numel())
    used = [] if stream is None else [t for s in states for t in s]
    with _on(stream, first, used) as s:
        out = [tuple(torch.empty(p.shape, dtype=torch.bfloat16, device=first.device) for _ in range(2)) for p in params]
        for k, (m, v) in enumerate(out):
            at_m[k], at_v[k] = m.data_ptr(), v.data_ptr()
        _check(_lib().head_adamw_values(rows, at_m, at_v, n, s), "head_adamw_values")
    return out


def _activation(name) -> int:
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"activation must be one of {list(ACTIVATIONS)}, not {name!r}") from None


def _layer(x, weight, bias, activation: int, halves: int):
    import torch
    _tensor(x, "x", shape=(None, None))
    dtype = _dtype(x, "x")
    _tensor(weight, "weight", x.dtype, (None, x.shape[1]), x)
    if weight.shape[0] % halves:
        raise ValueError(f"weight must have as many rows of gates as of values, not {weight.shape[0]} in all")
    if bias is not None:
        _tensor(bias, "bias", torch.float32, (weight.shape[0],), x)
    return _Layer(dtype, activation, x.shape[0], x.shape[1], weight.shape[0] // halves, x.data_ptr(), _stride(x), weight.data_ptr(),
                  _stride(weight), _at(bias))


def head_layer_launch(n_rows: int, dim: int, n_outputs: int, dtype: str = "float32", gated: bool = False, x: int = 0, x_stride: Optional[int] = None,
                      weight: int = 0, weight_stride: Optional[int] = None) -> dict:
    """What calls on a layer launch whose x and weight are at these addresses, their rows so many values apart (include/head_testing.h); no GPU
    needed."""
    s = _LayerLaunch()
    layer = _Layer({"float32": 0, "bfloat16": 1}[dtype], 0, n_rows, dim, n_outputs, x, dim if x_stride is None else x_stride, weight,
                   dim if weight_stride is None else weight_stride, None)
    _check(_lib().head_layer_launch(layer, gated, s), "head_layer_launch")
    return {name: int(getattr(s, name)) for name, _ in _LayerLaunch._fields_}


def head_linear(x, weight, bias=None, activation: Optional[str] = None, residual=None, scale: float = 1.0, keep: bool = False, stream=None):
    """y = residual + scale * activation(z) with z = x weight^T + bias.

    x: [n_rows, dim] float32 or bfloat16, weight: [n_outputs, dim] of the same type, bias: float32 [n_outputs] or None.  activation:
    None, "relu", "gelu" (x times the normal distribution's integral up to x) or "silu".  residual: [n_rows, n_outputs] of the same type, or
    None.  Returns y, [n_rows, n_outputs] of the same type, and with keep (y, z): z, which the gradients of a layer with an
    activation need.

    float32 products of many rows, and those of the gradients, take a value below 2^-109 to 2^-133 (include/head.h); a row's last bits may depend on how
    many rows its call has.
    """
    act = _activation(activation)
    if stream is None:
        got = _native().linear(x, weight, bias, act, residual, scale, keep)
        if got is not None:
            return _done(got, "head_linear")
    import torch
    layer = _layer(x, weight, bias, act, 1)
    shape = (layer.n_rows, layer.n_outputs)
    if residual is not None:
        _tensor(residual, "residual", x.dtype, shape, x)
    nbytes = _check(_lib().head_linear_bytes(layer), "head_linear")
    with _on(stream, x, (x, weight, bias, residual)) as s:
        y = torch.empty(shape, dtype=x.dtype, device=x.device)
        z = torch.empty(shape, dtype=x.dtype, device=x.device) if keep else None
        work = _workspace(nbytes, x)
        _check(_lib().head_linear(layer, _at(residual), 0 if residual is None else _stride(residual), scale, y.data_ptr(), _at(z), _at(work), s),
               "head_linear")
    return (y, z) if keep else y


def _layer_grad(what, call, nbytes, layer, halves, grad, x, weight, z, bias, stream):
    """The checks, outputs and workspace of a layer's gradient; call(z and its stride, grad and its stride, outputs, workspace, stream)."""
    import torch
    _tensor(grad, "grad", x.dtype, (layer.n_rows, layer.n_outputs), x)
    if z is not None:
        _tensor(z, "z", x.dtype, (layer.n_rows, weight.shape[0]), x)
    elif halves == 2 or layer.activation:
        raise ValueError("z is what the layer gave with keep=True, and is needed where there is an activation")
    nbytes = _check(nbytes(layer), what)
    with _on(stream, x, (grad, x, weight, z)) as s:
        grad_x = torch.empty((layer.n_rows, layer.dim), dtype=x.dtype, device=x.device)
        grad_weight = torch.empty(weight.shape, dtype=x.dtype, device=x.device)
        grad_bias = torch.empty(weight.shape[0], dtype=torch.float32, device=x.device) if bias else None
        work = _workspace(nbytes, x)
        _check(call(_at(z), 0 if z is None else _stride(z), grad.data_ptr(), _stride(grad), grad_x.data_ptr(), grad_weight.data_ptr(),
                    _at(grad_bias), _at(work), s), what)
    return grad_x, grad_weight, grad_bias


def head_linear_grad(grad, x, weight, z=None, activation: Optional[str] = None, scale: float = 1.0, bias: bool = True, stream=None):
    """The gradients of head_linear from grad, that of y.  z: what head_linear gave with keep=True; without an activation it is not needed.
    Returns (grad_x, grad_weight, grad_bias): the first two like x and weight, grad_bias float32 [n_outputs], or None without `bias`.  The
    residual's gradient is grad itself."""
    act = _activation(activation)
    if stream is None:
        got = _native().linear_grad(grad, x, weight, z, act, scale, bias)
        if got is not None:
            return _done(got, "head_linear_grad")
    layer = _layer(x, weight, None, act, 1)

    def call(z_at, z_stride, grad_at, grad_stride, *rest):
        return _lib().head_linear_grad(layer, z_at, z_stride, grad_at, grad_stride, scale, *rest)
    return _layer_grad("head_linear_grad", call, _lib().head_linear_grad_bytes, layer, 1, grad, x, weight, z, bias, stream)


def head_gated(x, weight, bias=None, activation: Optional[str] = "silu", keep: bool = False, stream=None):
    """y = activation(gates) * values, where z = x weight^T + bias is the gates, its first half of columns, and the values.

    x: [n_rows, dim] float32 or bfloat16, weight: [2 * n_outputs, dim] of the same type, bias: float32 [2 * n_outputs] or None, activation: as
    in head_linear.  Returns y, [n_rows, n_outputs] of the same type, and with keep (y, z): z, [n_rows, 2 * n_outputs], which
    the gradients need.  Products are as in head_linear.
    """
    act = _activation(activation)
    if stream is None:
        got = _native().gated(x, weight, bias, act, keep)
        if got is not None:
            return _done(got, "head_gated")
    import torch
    layer = _layer(x, weight, bias, act, 2)
    nbytes = _check(_lib().head_gated_bytes(layer), "head_gated")
    with _on(stream, x, (x, weight, bias)) as s:
        y = torch.empty((layer.n_rows, layer.n_outputs), dtype=x.dtype, device=x.device)
        z = torch.empty((layer.n_rows, weight.shape[0]), dtype=x.dtype, device=x.device) if keep else None
        work = _workspace(nbytes, x)
        _check(_lib().head_gated(layer, y.data_ptr(), _at(z), _at(work), s), "head_gated")
    return (y, z) if keep else y


def head_gated_grad(grad, x, weight, z, activation: Optional[str] = "silu", bias: bool = True, stream=None):
    """The gradients of head_gated from grad, that of y, and z, which head_gated gave with keep=True.  Returns (grad_x, grad_weight, grad_bias):
    the first two like x and weight, grad_bias float32 [2 * n_outputs], or None without `bias`."""
    act = _activation(activation)
    if stream is None:
        got = _native().gated_grad(grad, x, weight, z, act, bias)
        if got is not None:
            return _done(got, "head_gated_grad")
    layer = _layer(x, weight, None, act, 2)

    def call(*args):
        return _lib().head_gated_grad(layer, *args)
    return _layer_grad("head_gated_grad", call, _lib().head_gated_grad_bytes, layer, 2, grad, x, weight, z, bias, stream)


def head_clip(grads, max_norm: float, in_place: bool = False, stream=None):
    """The 2-norm of all tensors' values together, and the tensors times min(1, max_norm / norm).

    grads: contiguous float32 and bfloat16 tensors of any shape, a list.  max_norm: above 0; math.inf for no limit.  Returns (norm, clipped): norm a
    float32 tensor of no dimensions, clipped a list of new tensors like grads, or with in_place of grads themselves, whose values are
    replaced: they must not overlap.  A NaN among the values makes the norm and, unless there is no limit, all of them NaN.
    """
    if stream is None:
        got = _native().clip(grads, max_norm, in_place)
        if got is not None:
            return _done(got, "head_clip")
    import torch
    grads = list(grads)
    if not grads:
        raise ValueError("there are no tensors")
    if not max_norm > 0:
        raise ValueError(f"max_norm must be above 0, not {max_norm}")
    for k, t in enumerate(grads):
        _tensor(t, f"grads[{k}]", like=grads[0] if k else None)
        _dtype(t, f"grads[{k}]")
        if not t.is_contiguous():
            raise ValueError(f"grads[{k}] must be contiguous")
    if in_place:
        ends = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in grads if t.numel())
        if any(end > begin for (_, end), (begin, _) in zip(ends, ends[1:])):
            raise ValueError("tensors that are replaced must not overlap")
    with _on(stream, grads[0], grads) as s:
        norm = torch.empty((), dtype=torch.float32, device=grads[0].device)
        out = grads if in_place else [torch.empty_like(t, memory_format=torch.contiguous_format) for t in grads]
        tensors = (_ClipTensor * len(grads))(*(_ClipTensor(t.data_ptr(), o.data_ptr(), t.numel(), _dtype(t, "grads")) for t, o in zip(grads, out)))
        work = _workspace(_check(_lib().head_clip_bytes(tensors, len(grads)), "head_clip"), grads[0])
        if in_place:
            torch.autograd.graph.increment_version([t for t in grads if not t.is_inference()])  # what autograd has kept of them is out of date
        _check(_lib().head_clip(tensors, len(grads), max_norm, norm.data_ptr(), _at(work), s), "head_clip")
    return norm, list(out)
