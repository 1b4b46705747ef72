"""The feed-forward operators of ``include/spingtp.h``: norm, 8-bit blocks, 8-bit product, gated block, linear layer.

Argument checks, outputs and the calls are in ``csrc/binding.cpp``, every step of the computation in the HIP
kernels of ``libspingtp.so``.  Matrices are 2-D device tensors whose rows are contiguous (``stride(1) == 1``),
at any row stride; the gated block's bf16 x and weights start on 16 bytes (a tensor of its own does, a slice may
not: SpinGTPError).  Every operator runs on the current stream of its tensors' device, or on ``stream=``.

The operators are no part of autograd's graph: what they make requires no gradient, whatever the operands do, and
gradients are the ``*_backward`` functions' to give (from a ``torch.autograd.Function``, for instance).
"""

import functools
import importlib.util
import os

import torch

from . import _lib

_ACTS = {"silu": 0, "gelu": 1}
_SAVES = {None: 0, "same": 1, "8bit": 2}
_LINEAR_ACTS = {**_ACTS, None: 2}
_LINEAR_SAVES = {None: False, "same": True}
_TRANSPOSE = {False: 0, True: 1, "both": 2}
_DTYPES = {torch.float32: False, torch.bfloat16: True}

_BINDING_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_binding.so")
# in the order of Entries in csrc/binding.cpp
_ENTRIES = ("spingtp_pack8", "spingtp_unpack8", "spingtp_rms_norm", "spingtp_rms_norm_backward",
            "spingtp_rms_norm_backward_workspace_size", "spingtp_matmul8", "spingtp_gated_forward",
            "spingtp_gated_forward_workspace_size", "spingtp_gated_forward8", "spingtp_gated_forward8_workspace_size",
            "spingtp_gated_backward", "spingtp_gated_backward_workspace_size", "spingtp_linear_forward",
            "spingtp_linear_forward_workspace_size", "spingtp_linear_forward8", "spingtp_linear_forward8_workspace_size",
            "spingtp_linear_backward", "spingtp_linear_backward_workspace_size", "spingtp_embedding", "spingtp_sort_index",
            "spingtp_sort_index_workspace_size", "spingtp_embedding_backward",
            "spingtp_embedding_backward_workspace_size", "spingtp_adamw")


def _load():
    if not os.path.exists(_BINDING_PATH):
        raise RuntimeError(f"{_BINDING_PATH} is not built; run __graft_entry__.build() "
                           "(or python paper_2607_01408_amd/build.py)")
    import ctypes

    spec = importlib.util.spec_from_file_location("paper_2607_01408_amd._binding", _BINDING_PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    lib = _lib.lib()
    module.bind(tuple(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in _ENTRIES), _lib.SpinGTPError)
    return module


_ops = _load()
_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch.cuda.current_device


def _on_stream(op):
    """``stream=``: the call and what it allocates are that stream's, as under ``torch.cuda.stream(stream)``."""

    name = op.__code__.co_varnames[0]  # the first operand's, whose device the stream must be of

    @functools.wraps(op)
    def call(*args, stream=None, **kwargs):
        if stream is None:
            return op(*args, **kwargs)
        first = args[0] if args else kwargs.get(name)
        if isinstance(first, (list, tuple)) and first:
            first = first[0]
        if stream.device != getattr(first, "device", stream.device):
            raise ValueError(f"the stream is of {stream.device}, the tensors are on {first.device}")
        with torch.cuda.stream(stream):
            return op(*args, **kwargs)

    return call


def _run(op, first, *args):
    """The call on the device of `first` and that device's current stream."""
    index = getattr(first, "device", torch.device("cpu")).index
    if index is None:
        raise ValueError(f"tensors on a GPU are wanted, not {first!r}")
    if index == _current_device():
        return op(*args, _raw_stream(index))
    with torch.cuda.device(index):
        return op(*args, _raw_stream(index))


def _choice(table, value, name):
    try:
        return table[value]
    except (KeyError, TypeError):
        raise ValueError(f"{name} must be one of {list(table)}, not {value!r}") from None


class Block8:
    """A matrix in the 8-bit block format (``spingtp.h``): ``values`` [R, Dp] float8_e4m3fn, ``scales``
    [R, Sp] float8_e8m0fnu, ``shape`` (R, D).  Columns of ``values`` from D on must be zero.  D = 0 is the transpose of a
    matrix of no rows."""

    __slots__ = ("values", "scales", "shape")

    def __init__(self, values, scales, shape):
        R, D = shape
        _ops.check_block(values, scales, R, D)
        self.values, self.scales, self.shape = values, scales, (R, D)

    @property
    def device(self):
        return self.values.device

    @classmethod
    def empty(cls, R, D, device):
        """A matrix with values and scales still to be written."""
        return cls(torch.empty((R, -(-D // 128) * 128), dtype=torch.float8_e4m3fn, device=device),
                   torch.empty((R, -(-D // 512) * 4), dtype=torch.float8_e8m0fnu, device=device), (R, D))


def _made(pair, R, D):
    """What the library made: nothing to check."""
    b = Block8.__new__(Block8)
    b.values, b.scales = pair
    b.shape = (R, D)
    return b


def _block(b, name, rows=None, columns=None):
    if not isinstance(b, Block8):
        raise ValueError(f"{name} must be a Block8")
    R, D = b.shape
    if (rows is not None and R != rows) or (columns is not None and D != columns):
        raise ValueError(f"{name} must be [{'any' if rows is None else rows}, {'any' if columns is None else columns}], "
                         f"not {list(b.shape)}")
    return b.values, b.scales


@_on_stream
def pack8(x, transpose=False):
    """spingtp_pack8: ``x`` [R, D] as a Block8; with ``transpose=True`` its transpose [D, R] (packed along x's
    columns), with ``transpose="both"`` the pair, x read once."""
    how = _choice(_TRANSPOSE, transpose, "transpose")
    made = _run(_ops.pack8, x, x, how)
    R, D = x.shape
    if how == 2:
        return _made(made[0], R, D), _made(made[1], D, R)
    return _made(made, D, R) if how else _made(made, R, D)


@_on_stream
def unpack8(b, dtype=torch.bfloat16, out=None):
    """spingtp_unpack8: the matrix [R, D] that a Block8 stands for."""
    return _run(_ops.unpack8, b, *_block(b, "b"), *b.shape, _choice(_DTYPES, dtype, "dtype"), out)


@_on_stream
def rms_norm(x, gain, residual=None, eps=1e-6, out8=False):
    """spingtp_rms_norm: (y, h, rstd) with h = x + residual, y = h rstd gain.

    y is of x's dtype or, with ``out8``, a Block8; h is x itself where there is no residual."""
    y, h, rstd = _run(_ops.rms_norm, x, x, gain, residual, eps, out8)
    return _made(y, *x.shape) if out8 else y, x if h is None else h, rstd


@_on_stream
def rms_norm_backward(grad_y, h, rstd, gain, grad_h=None, need_gain=True):
    """spingtp_rms_norm_backward: (grad_x, grad_gain); grad_x is also the residual's gradient.

    ``grad_h`` is the gradient that reaches h directly (the residual stream's); grad_gain is None where not
    needed."""
    return _run(_ops.rms_norm_backward, grad_y, grad_y, h, rstd, gain, grad_h, need_gain)


@_on_stream
def matmul8(a, b, dtype=torch.bfloat16, out=None):
    """spingtp_matmul8: a [M, K] times b [N, K] transposed, both Block8; [M, N] in bf16 or fp32."""
    pa = _block(a, "a")
    M, K = a.shape
    pb = _block(b, "b", None, K)
    return _run(_ops.matmul8, a, *pa, *pb, M, b.shape[0], K, _choice(_DTYPES, dtype, "dtype"), out)


@_on_stream
def matmul8_backward(grad_out, a_t, b_t):
    """Gradients (grad_a [M, K], grad_b [N, K]) of ``matmul8``, in grad_out's dtype.

    grad_out [M, N] is packed along its rows and its columns, read once; ``a_t`` [K, M] and ``b_t`` [K, N] are the
    operands packed along the axis that each gradient sums over (``pack8(..., transpose=True)`` of the matrices that
    ``a`` and ``b`` were packed from)."""
    rows, cols = pack8(grad_out, transpose="both")
    M, N = grad_out.shape
    _block(a_t, "a_t", None, M)
    _block(b_t, "b_t", a_t.shape[0], N)
    return matmul8(rows, b_t, grad_out.dtype), matmul8(cols, a_t, grad_out.dtype)


class GatedSaved:
    """What ``gated`` keeps for ``gated_backward``: ``x``, and the pre-activations ``g`` and ``u``; bf16 tensors or
    Block8."""

    __slots__ = ("x", "g", "u", "act", "save")

    def __init__(self, x, g, u, act, save):
        self.x, self.g, self.u, self.act, self.save = x, g, u, act, save


@_on_stream
def gated(x, w_gate, w_up, act="silu", save=None, out8=False):
    """spingtp_gated_forward / spingtp_gated_forward8: (h [M, F], saved) with h = act(x w_gate^T) (x w_up^T).

    bf16 x [M, K] and weights [F, K]: h is bf16.  ``save`` keeps what the backward pass needs: ``"same"`` x as it is
    and the pre-activations in bf16, ``"8bit"`` all three as Block8.  Block8 operands (inference): h is bf16 or, with
    ``out8``, a Block8.  saved is None without ``save``."""
    code, keep = _choice(_ACTS, act, "act"), _choice(_SAVES, save, "save")
    if isinstance(x, Block8):
        if keep:
            raise ValueError("save needs bf16 operands")
        M, K = x.shape
        pg = _block(w_gate, "w_gate", None, K)
        F = w_gate.shape[0]
        pu = _block(w_up, "w_up", F, K)
        if F < 1 or K < 1:
            raise ValueError("the weights are empty")
        h = _run(_ops.gated8, x, x.values, x.scales, *pg, *pu, M, K, F, code, out8)
        return _made(h, M, F) if out8 else h, None
    if out8:
        raise ValueError("out8 needs Block8 operands")
    h, x8, g, u = _run(_ops.gated, x, x, w_gate, w_up, code, keep)
    if keep == 0:
        return h, None
    if keep == 1:
        return h, GatedSaved(x, g, u, act, save)
    (M, K), F = x.shape, w_gate.shape[0]
    return h, GatedSaved(_made(x8, M, K), _made(g, M, F), _made(u, M, F), act, save)


@_on_stream
def gated_backward(grad_h, saved, w_gate, w_up, need_x=True, need_w=True):
    """spingtp_gated_backward: (grad_x [M, K], grad_w_gate [F, K], grad_w_up [F, K]) in bf16 (None where not
    needed; the two weight gradients are halves of one tensor)."""
    if not isinstance(saved, GatedSaved):
        raise ValueError("saved must be what gated returned with save")
    keep = _choice(_SAVES, saved.save, "saved.save")
    kept = saved.x, saved.g, saved.u
    if keep == 2:
        # with their widths: blocks of another width may have the same padded one
        kept = tuple((*_block(b, n), b.shape[1]) for b, n in zip(kept, ("saved.x", "saved.g", "saved.u")))
    grad_x, grad_w = _run(_ops.gated_backward, grad_h, grad_h, keep, *kept, w_gate, w_up,
                          _choice(_ACTS, saved.act, "saved.act"), need_x, need_w)
    if grad_w is None:
        return grad_x, None, None
    return (grad_x, *grad_w.chunk(2))


class LinearSaved:
    """What ``linear`` keeps for ``linear_backward``: ``x`` [M, K] as it is and, where there is an activation ``act``,
    ``z`` [M, N], x w^T + bias in bf16."""

    __slots__ = ("x", "z", "act")

    def __init__(self, x, z=None, act=None):
        self.x, self.z, self.act = x, z, act


@_on_stream
def linear(x, w, bias=None, act=None, residual=None, save=None, dtype=torch.bfloat16, out=None):
    """spingtp_linear_forward / spingtp_linear_forward8: (y [M, N], saved) with y = act(x w^T + bias) + residual.

    x [M, K] and w [N, K] in bf16 (any alignment; rows that do not start and end on 16 bytes are copied) or, for
    inference, both Block8; bias [N] fp32; act None, ``"silu"`` or ``"gelu"``; residual and y of ``dtype``, bf16 or fp32;
    ``out`` may be the residual itself, and overlaps no operand otherwise.
    ``save="same"`` (bf16) keeps what the backward pass needs; saved is None without it."""
    code, keep = _choice(_LINEAR_ACTS, act, "act"), _choice(_LINEAR_SAVES, save, "save")
    bf16 = _choice(_DTYPES, dtype, "dtype")
    if isinstance(x, Block8):
        if keep:
            raise ValueError("save needs bf16 operands")
        M, K = x.shape
        pw = _block(w, "w", None, K)
        return _run(_ops.linear8, x, x.values, x.scales, *pw, M, K, w.shape[0], bias, code, residual, bf16, out), None
    y, z = _run(_ops.linear, x, x, w, bias, code, residual, keep, bf16, out)
    return y, LinearSaved(x, z, act) if keep else None


@_on_stream
def linear_backward(grad_y, saved, w, need_x=True, need_w=True, need_bias=True, dtype=torch.bfloat16):
    """spingtp_linear_backward: (grad_x [M, K] bf16, grad_w [N, K] of ``dtype``, grad_bias [N] fp32), None where not
    needed.  grad_y is bf16 or fp32; it is also the residual's gradient."""
    if not isinstance(saved, LinearSaved):
        raise ValueError("saved must be what linear returned with save, or a LinearSaved")
    return _run(_ops.linear_backward, grad_y, grad_y, saved.x, saved.z, _choice(_LINEAR_ACTS, saved.act, "saved.act"), w,
                need_x, need_w, need_bias, _choice(_DTYPES, dtype, "dtype"))
