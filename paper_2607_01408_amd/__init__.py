"""SpinGTP on AMD MI355X: the spin-weighted Gaunt tensor product as a C-ABI HIP library.

``Plan`` wraps ``spingtp_plan_create`` / ``spingtp_forward`` (``include/spingtp.h``).
``rms_norm``, ``matmul8``, ``gated``, ``linear``, ``pack8`` and their kin are the feed-forward operators on
invariant channels (``feedforward``), ``Block8`` their 8-bit block format; ``embedding``, ``sort_index``, ``adamw`` and
theirs the operators of a training step around the layers (``training``).
``workloads`` holds the seeded synthetic input generators.
"""

from ._lib import SpinGTPError, LIB_PATH
from .spingtp import Plan, plan_tables_host, dense_tensor_host, mfma_operands_host, pre_table_host, conj_map_host, direct_table_host, paths_host, uvw_table_host, BASIS_PAPER, BASIS_M0_PAIRED, BASIS_PARITY

_FEEDFORWARD = ("Block8", "GatedSaved", "pack8", "unpack8", "rms_norm", "rms_norm_backward", "matmul8",
                "matmul8_backward", "gated", "gated_backward", "LinearSaved", "linear", "linear_backward")
_TRAINING = ("SortedIndex", "sort_index", "embedding", "embedding_backward", "adamw", "adamw_state")


def __getattr__(name):  # torch is imported with the first operator that needs it
    if name in _FEEDFORWARD:
        from . import feedforward
        globals().update({n: getattr(feedforward, n) for n in _FEEDFORWARD})
        return globals()[name]
    if name in _TRAINING:
        from . import training
        globals().update({n: getattr(training, n) for n in _TRAINING})
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")


def __dir__():
    return sorted({*globals(), *_FEEDFORWARD, *_TRAINING})


# without the operators: what an import of all names asks of a machine is what the plans need
__all__ = ["Plan", "plan_tables_host", "dense_tensor_host", "mfma_operands_host", "pre_table_host", "conj_map_host", "direct_table_host", "paths_host", "uvw_table_host", "SpinGTPError", "LIB_PATH", "BASIS_PAPER", "BASIS_M0_PAIRED", "BASIS_PARITY"]
