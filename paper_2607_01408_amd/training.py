"""The operators of a training step around the layers (``include/spingtp.h``): lookup of embeddings and its gradient
by sorted indexes, AdamW over many tensors.

As the feed-forward operators they take device tensors, run on the current stream of their device or on ``stream=``,
and are no part of autograd's graph; argument checks, outputs and the calls are in ``csrc/binding.cpp``, every step of
the computation in the HIP kernels of ``libspingtp.so``.
"""

import torch

from .feedforward import _DTYPES, Block8, _choice, _on_stream, _ops, _run


class SortedIndex:
    """What ``sort_index`` makes of an index: its places by the rows that they name (``order``, int32, equal rows in the
    index's order), those rows (``rows``, int32; ``V`` for entries outside the table) and the table's number of
    rows ``V``."""

    __slots__ = ("order", "rows", "V")

    def __init__(self, order, rows, V):
        self.order, self.rows, self.V = order, rows, V

    @property
    def device(self):
        return self.order.device


@_on_stream
def embedding(table, index, scale=1.0):
    """spingtp_embedding: ``scale`` times the rows of ``table`` [V, D] that ``index`` [n] (int64 or int32) names, [n, D] in the
    table's dtype.  An entry outside [0, V) names no row: zeros."""
    return _run(_ops.embedding, table, table, index, scale)


@_on_stream
def sort_index(index, V):
    """spingtp_sort_index: the SortedIndex of ``index`` [n] (int64 or int32) into a table of ``V`` rows, for the gradients of
    as many lookups as take this index."""
    return SortedIndex(*_run(_ops.sort_index, index, index, V), V)


@_on_stream
def embedding_backward(grad, index, V, scale=1.0, dtype=None):
    """spingtp_embedding_backward: [V, D], row v the sum of ``scale`` times the rows of ``grad`` [n, D] where ``index`` is v
    (zeros where it nowhere is), in ``dtype`` (grad's).  ``index`` is the lookup's or its SortedIndex; entries
    outside [0, V) add to no row.  Sums are fp32 and in the same order in every call."""
    if isinstance(index, SortedIndex):
        if index.V != V:
            raise ValueError(f"the index was sorted for {index.V} rows, not {V}")
        pair = index.order, index.rows
    else:
        pair = index, None
    return _run(_ops.embedding_backward, grad, grad, *pair, V, scale,
                None if dtype is None else _choice(_DTYPES, dtype, "dtype"))


def _list(x):
    return x if type(x) is list else list(x)


@_on_stream
def adamw(params, grads, m, v, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_scale=None, copies=None,
          seed=0):
    """spingtp_adamw: one step over the tensors of ``params`` (fp32 or bf16), in place, from ``grads`` (fp32 or bf16) and
    the states ``m`` and ``v``, lists of as many.  All tensors are contiguous and on one device, a gradient in its
    param's shape.

    A state is an fp32 tensor of as many elements or a Block8 of shape (1, elements), both of a tensor alike; in 8
    bits ``v`` holds its root, and values are rounded by random bits from ``seed``, the step and the element's place
    (zeros to begin with: ``adamw_state``).  ``copies``: bf16 tensors (or None) that receive fp32 params rounded, the weights
    that layers read.  ``grad_scale``: a device fp32 tensor of one element, a factor of all gradients.  ``step`` (1 for the
    first) and ``lr`` are numbers or, for captured steps, device tensors of one element, int64 and fp32."""
    params = _list(params)
    if params:
        _run(_ops.adamw, params[0], params, _list(grads), _list(m), _list(v), None if copies is None else _list(copies), step,
             lr, *betas, eps, weight_decay, grad_scale, seed)


def adamw_state(param, bits=32):
    """(m, v) for ``adamw`` before the first step: zeros beside ``param``, fp32 or, with ``bits=8``, Block8."""
    if bits == 32:
        return tuple(torch.zeros(param.shape, dtype=torch.float32, device=param.device) for _ in range(2))
    if bits != 8:
        raise ValueError(f"bits must be 8 or 32, not {bits!r}")
    made = tuple(Block8.empty(1, param.numel(), param.device) for _ in range(2))
    for b in made:
        b.values.view(torch.uint8).zero_()
        b.scales.view(torch.uint8).fill_(127)
    return made
