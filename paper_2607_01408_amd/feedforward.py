"""The feed-forward operators of ``include/spingtp.h``: norm, 8-bit blocks, 8-bit product, gated block.

Argument checks and marshalling only; every step runs in the HIP kernels of ``libspingtp.so``.
Matrices are 2-D device tensors whose rows are contiguous (``stride(1) == 1``), at any row stride.
Every operator runs on the current stream of its tensors' device, or on ``stream=``.
"""

import ctypes
import functools

import torch

from . import _lib

_DTYPES = {torch.float32: 0, torch.bfloat16: 1}
_ACTS = {"silu": 0, "gelu": 1}
_SAVES = {None: 0, "same": 1, "8bit": 2}


def _up(n, m):
    return -(-n // m) * m


@functools.lru_cache(maxsize=None)
def _call(name):
    return getattr(_lib.lib(), name)


def _on_stream(op):
    """``stream=``: the call and what it allocates are that stream's, as under ``torch.cuda.stream(stream)``."""

    @functools.wraps(op)
    def call(first, *args, stream=None, **kwargs):
        if stream is None:
            return op(first, *args, **kwargs)
        if stream.device != getattr(first, "device", stream.device):
            raise ValueError(f"the stream is of {stream.device}, the tensors are on {first.device}")
        with torch.cuda.stream(stream):
            return op(first, *args, **kwargs)

    return call


def _run(name, device, *args):
    """The C call on `device` and its current stream."""
    index = device.index
    stream = torch.cuda.current_stream(index).cuda_stream
    if index == torch.cuda.current_device():
        status = _call(name)(*args, stream)
    else:
        with torch.cuda.device(index):
            status = _call(name)(*args, stream)
    if status:
        _lib.check(status, name)


def _matrix(t, name, shape=None, dtypes=(torch.float32, torch.bfloat16), device=None):
    """Checks a [rows, columns] operand and gives (address, row stride)."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, not {t.dtype}")
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} must be on {device or 'a GPU'}, not on {t.device}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, not {list(t.shape)}")
    rows, columns = t.shape
    ld, step = t.stride()
    if columns > 1 and step != 1:
        raise ValueError(f"{name} must have contiguous rows")
    if rows <= 1:
        ld = columns  # the stride of a single row says nothing
    elif ld < columns:
        raise ValueError(f"{name} has overlapping rows")
    return t.data_ptr(), max(ld, 1)


def _vector(t, name, n, device):
    if not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or tuple(t.shape) != (n,) or t.device != device or (
            n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous fp32 [{n}] tensor on {device}")
    return t.data_ptr()


class Block8:
    """A matrix in the 8-bit block format (``spingtp.h``): ``values`` [R, Dp] float8_e4m3fn, ``scales``
    [R, Sp] float8_e8m0fnu, ``shape`` (R, D).  Columns of ``values`` from D on must be zero."""

    __slots__ = ("values", "scales", "shape")

    def __init__(self, values, scales, shape):
        R, D = int(shape[0]), int(shape[1])
        if R < 0 or D < 1:
            raise ValueError(f"no matrix has the shape {(R, D)}")
        pitch, spitch = _up(D, 128), _up(D, 512) // 128
        if (values.dtype != torch.float8_e4m3fn or tuple(values.shape) != (R, pitch) or not values.is_contiguous()
                or not values.is_cuda):
            raise ValueError(f"values must be a contiguous float8_e4m3fn [{R}, {pitch}] device tensor")
        if (scales.dtype != torch.float8_e8m0fnu or tuple(scales.shape) != (R, spitch) or not scales.is_contiguous()
                or scales.device != values.device):
            raise ValueError(f"scales must be a contiguous float8_e8m0fnu [{R}, {spitch}] tensor beside the values")
        self.values, self.scales, self.shape = values, scales, (R, D)

    @property
    def device(self):
        return self.values.device

    @classmethod
    def empty(cls, R, D, device):
        """A matrix with values and scales still to be written."""
        b = cls.__new__(cls)
        b.values = torch.empty((R, _up(D, 128)), dtype=torch.float8_e4m3fn, device=device)
        b.scales = torch.empty((R, _up(D, 512) // 128), dtype=torch.float8_e8m0fnu, device=device)
        b.shape = (R, D)
        return b


def _block(b, name, shape=None, device=None):
    if not isinstance(b, Block8):
        raise ValueError(f"{name} must be a Block8")
    if shape is not None and tuple(b.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, not {list(b.shape)}")
    if device is not None and b.device != device:
        raise ValueError(f"{name} must be on {device}, not on {b.device}")
    return b.values.data_ptr(), b.scales.data_ptr()


def _result(out, shape, dtype, device, name="out"):
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _matrix(out, name, shape, (dtype,), device)
    return out


@_on_stream
def pack8(x, transpose=False):
    """spingtp_pack8: ``x`` [R, D] as a Block8; with ``transpose=True`` its transpose [D, R] (packed along x's
    columns), with ``transpose="both"`` the pair, x read once."""
    if transpose not in (False, True, "both"):
        raise ValueError('transpose must be False, True or "both"')
    p, ld = _matrix(x, "x")
    R, D = x.shape
    if D < 1 or (transpose and R < 1):
        raise ValueError(f"no blocks in a matrix of shape {(R, D)}")
    rows = Block8.empty(R, D, x.device) if transpose is not True else None
    cols = Block8.empty(D, R, x.device) if transpose else None
    a = (rows.values.data_ptr(), rows.scales.data_ptr()) if rows else (None, None)
    b = (cols.values.data_ptr(), cols.scales.data_ptr()) if cols else (None, None)
    _run("spingtp_pack8", x.device, _DTYPES[x.dtype], p, ld, *a, *b, R, D)
    return (rows, cols) if transpose == "both" else (cols if transpose else rows)


@_on_stream
def unpack8(b, dtype=torch.bfloat16, out=None):
    """spingtp_unpack8: the matrix [R, D] that a Block8 stands for."""
    v, s = _block(b, "b")
    if dtype not in _DTYPES:
        raise ValueError(f"dtype must be torch.float32 or torch.bfloat16, not {dtype}")
    out = _result(out, b.shape, dtype, b.device)
    p, ld = _matrix(out, "out")
    _run("spingtp_unpack8", b.device, v, s, _DTYPES[dtype], p, ld, *b.shape)
    return out


@_on_stream
def rms_norm(x, gain, residual=None, eps=1e-6, out8=False):
    """spingtp_rms_norm: (y, h, rstd) with h = x + residual, y = h rstd gain.

    y is of x's dtype or, with ``out8``, a Block8; h is x itself where there is no residual."""
    p, ld = _matrix(x, "x")
    R, D = x.shape
    dev = x.device
    if D < 1:
        raise ValueError("x has no columns")
    g = _vector(gain, "gain", D, dev)
    if not eps >= 0:
        raise ValueError(f"eps must not be negative: {eps}")
    h, pr, ldr, ph, ldh = x, None, 0, None, 0
    if residual is not None:
        pr, ldr = _matrix(residual, "residual", (R, D), (x.dtype,), dev)
        h = torch.empty((R, D), dtype=x.dtype, device=dev)
        ph, ldh = h.data_ptr(), D
    rstd = torch.empty(R, dtype=torch.float32, device=dev)
    if out8:
        y = Block8.empty(R, D, dev)
        out = (None, 0, y.values.data_ptr(), y.scales.data_ptr())
    else:
        y = torch.empty((R, D), dtype=x.dtype, device=dev)
        out = (y.data_ptr(), D, None, None)
    _run("spingtp_rms_norm", dev, _DTYPES[x.dtype], p, ld, pr, ldr, g, float(eps), ph, ldh, *out,
         rstd.data_ptr(), R, D)
    return y, h, rstd


@_on_stream
def rms_norm_backward(grad_y, h, rstd, gain, grad_h=None, need_gain=True):
    """spingtp_rms_norm_backward: (grad_x, grad_gain); grad_x is also the residual's gradient.

    ``grad_h`` is the gradient that reaches h directly (the residual stream's); grad_gain is None where not
    needed."""
    pd, ldd = _matrix(grad_y, "grad_y")
    R, D = grad_y.shape
    dev = grad_y.device
    if D < 1:
        raise ValueError("grad_y has no columns")
    ph, ldh = _matrix(h, "h", (R, D), (grad_y.dtype,), dev)
    pr, pg = _vector(rstd, "rstd", R, dev), _vector(gain, "gain", D, dev)
    pgh, ldgh = _matrix(grad_h, "grad_h", (R, D), (grad_y.dtype,), dev) if grad_h is not None else (None, 0)
    grad_x = torch.empty((R, D), dtype=grad_y.dtype, device=dev)
    grad_gain = workspace = None
    n = ctypes.c_size_t(0)
    if need_gain:
        grad_gain = torch.empty(D, dtype=torch.float32, device=dev)
        _lib.check(_call("spingtp_rms_norm_backward_workspace_size")(R, D, ctypes.byref(n)),
                   "spingtp_rms_norm_backward_workspace_size")
        workspace = torch.empty(n.value, dtype=torch.uint8, device=dev)
    _run("spingtp_rms_norm_backward", dev, _DTYPES[grad_y.dtype], pd, ldd, ph, ldh, pr, pg, pgh, ldgh,
         grad_x.data_ptr(), D, grad_gain.data_ptr() if need_gain else None,
         workspace.data_ptr() if need_gain else None, n.value, R, D)
    return grad_x, grad_gain


@_on_stream
def matmul8(a, b, dtype=torch.bfloat16, out=None):
    """spingtp_matmul8: a [M, K] times b [N, K] transposed, both Block8; [M, N] in bf16 or fp32."""
    pa = _block(a, "a")
    M, K = a.shape
    pb = _block(b, "b", (b.shape[0], K) if isinstance(b, Block8) else None, a.device)
    N = b.shape[0]
    if dtype not in _DTYPES:
        raise ValueError(f"dtype must be torch.float32 or torch.bfloat16, not {dtype}")
    out = _result(out, (M, N), dtype, a.device)
    p, ld = _matrix(out, "out")
    _run("spingtp_matmul8", a.device, *pa, *pb, _DTYPES[dtype], p, ld, M, N, K)
    return out


@_on_stream
def matmul8_backward(grad_out, a_t, b_t):
    """Gradients (grad_a [M, K], grad_b [N, K]) of ``matmul8``, in grad_out's dtype.

    grad_out [M, N] is packed along its rows and its columns, x read once; ``a_t`` [K, M] and ``b_t`` [K, N] are the
    operands packed along the axis that each gradient sums over (``pack8(..., transpose=True)`` of the matrices that
    ``a`` and ``b`` were packed from)."""
    _matrix(grad_out, "grad_out")
    M, N = grad_out.shape
    _block(a_t, "a_t", (a_t.shape[0], M) if isinstance(a_t, Block8) else None, grad_out.device)
    _block(b_t, "b_t", (a_t.shape[0], N), grad_out.device)
    rows, cols = pack8(grad_out, transpose="both")
    return (matmul8(rows, b_t, grad_out.dtype), matmul8(cols, a_t, grad_out.dtype))


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
    if act not in _ACTS:
        raise ValueError(f"act must be one of {sorted(_ACTS)}, not {act!r}")
    if save not in _SAVES:
        raise ValueError(f'save must be None, "same" or "8bit", not {save!r}')
    if isinstance(x, Block8):
        if save is not None:
            raise ValueError("save needs bf16 operands")
        dev, (M, K) = x.device, x.shape
        F = w_gate.shape[0] if isinstance(w_gate, Block8) else 0
        px = _block(x, "x")
        pg, pu = _block(w_gate, "w_gate", (F, K), dev), _block(w_up, "w_up", (F, K), dev)
        if F < 1:
            raise ValueError("the weights have no rows")
        n, ws = ctypes.c_size_t(0), None
        if out8:
            h = Block8.empty(M, F, dev)
            o = (h.values.data_ptr(), 0, h.scales.data_ptr())
            _lib.check(_call("spingtp_gated_forward8_workspace_size")(M, K, F, 1, ctypes.byref(n)),
                       "spingtp_gated_forward8_workspace_size")
            if n.value:
                ws = torch.empty(n.value, dtype=torch.uint8, device=dev)
        else:
            h = torch.empty((M, F), dtype=torch.bfloat16, device=dev)
            o = (h.data_ptr(), F, None)
        _run("spingtp_gated_forward8", dev, _ACTS[act], *px, *pg, *pu, *o, ws.data_ptr() if ws is not None else None,
             n.value, M, K, F)
        return h, None
    if out8:
        raise ValueError("out8 needs Block8 operands")
    bf16 = (torch.bfloat16,)
    px, ldx = _matrix(x, "x", None, bf16)
    M, K = x.shape
    dev = x.device
    pg, ldw = _matrix(w_gate, "w_gate", None, bf16, dev)
    F = w_gate.shape[0]
    pu, ldw2 = _matrix(w_up, "w_up", w_gate.shape, bf16, dev)
    if w_gate.shape[1] != K or K < 1 or F < 1:
        raise ValueError(f"the weights must be [F, {K}], not {list(w_gate.shape)}")
    if ldw != ldw2:
        raise ValueError("w_gate and w_up must have the same row stride")
    h = torch.empty((M, F), dtype=torch.bfloat16, device=dev)
    saved, g = None, (None, None, None, None)
    if save == "same":
        saved = GatedSaved(x, torch.empty_like(h), torch.empty_like(h), act, save)
        g = (saved.g.data_ptr(), None, saved.u.data_ptr(), None)
    elif save == "8bit":
        saved = GatedSaved(pack8(x), Block8.empty(M, F, dev), Block8.empty(M, F, dev), act, save)
        g = (saved.g.values.data_ptr(), saved.g.scales.data_ptr(), saved.u.values.data_ptr(), saved.u.scales.data_ptr())
    n, ws = ctypes.c_size_t(0), None
    if K % 8 or ldx % 8 or ldw % 8 or (M <= 32 and save == "8bit"):  # otherwise none is needed
        _lib.check(_call("spingtp_gated_forward_workspace_size")(M, K, F, ldx, ldw, _SAVES[save], ctypes.byref(n)),
                   "spingtp_gated_forward_workspace_size")
        ws = torch.empty(n.value, dtype=torch.uint8, device=dev)
    _run("spingtp_gated_forward", dev, _ACTS[act], px, ldx, pg, pu, ldw, h.data_ptr(), F, _SAVES[save], *g,
         ws.data_ptr() if ws is not None else None, n.value, M, K, F)
    return h, saved


@_on_stream
def gated_backward(grad_h, saved, w_gate, w_up, need_x=True, need_w=True):
    """spingtp_gated_backward: (grad_x [M, K], grad_w_gate [F, K], grad_w_up [F, K]) in bf16 (None where not
    needed; the two weight gradients are halves of one tensor)."""
    if not isinstance(saved, GatedSaved):
        raise ValueError("saved must be what gated returned with save")
    bf16 = (torch.bfloat16,)
    ph, ldh = _matrix(grad_h, "grad_h", None, bf16)
    M, F = grad_h.shape
    dev = grad_h.device
    pg, ldw = _matrix(w_gate, "w_gate", None, bf16, dev)
    K = w_gate.shape[1]
    if w_gate.shape[0] != F:
        raise ValueError(f"w_gate must be [{F}, K], not {list(w_gate.shape)}")
    pu, ldw2 = _matrix(w_up, "w_up", (F, K), bf16, dev)
    if ldw != ldw2:
        raise ValueError("w_gate and w_up must have the same row stride")
    if saved.save == "8bit":
        x, sx = _block(saved.x, "saved.x", (M, K), dev)
        ldx = K
        g, gs = _block(saved.g, "saved.g", (M, F), dev)
        u, us = _block(saved.u, "saved.u", (M, F), dev)
    else:
        x, ldx = _matrix(saved.x, "saved.x", (M, K), bf16, dev)
        sx = gs = us = None
        (g, ldg), (u, ldu) = _matrix(saved.g, "saved.g", (M, F), bf16, dev), _matrix(saved.u, "saved.u", (M, F), bf16, dev)
        if ldg != F or ldu != F:
            raise ValueError("saved.g and saved.u must be dense")
    grad_x = torch.empty((M, K), dtype=torch.bfloat16, device=dev) if need_x else None
    grad_w = torch.empty((2 * F, K), dtype=torch.bfloat16, device=dev) if need_w else None
    n = ctypes.c_size_t(0)
    _lib.check(_call("spingtp_gated_backward_workspace_size")(M, K, F, ctypes.byref(n)),
               "spingtp_gated_backward_workspace_size")
    ws = torch.empty(n.value, dtype=torch.uint8, device=dev)
    _run("spingtp_gated_backward", dev, _ACTS[saved.act], ph, ldh, _SAVES[saved.save], g, gs, u, us, x, ldx, sx,
         pg, pu, ldw, grad_x.data_ptr() if need_x else None, K, grad_w.data_ptr() if need_w else None, ws.data_ptr(),
         n.value, M, K, F)
    return grad_x, grad_w[:F] if need_w else None, grad_w[F:] if need_w else None
