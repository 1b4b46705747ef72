"""The argument checks and workspace sizes of the training step's entry points (no GPU needed): each refusal comes before
any launch.  And the same, with those of the linear layer, under the sanitizers."""

import ctypes
import os
import subprocess
import sys

import pytest

from paper_2607_01408_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BUF = ctypes.create_string_buffer(4096 + 16)
P = (ctypes.addressof(BUF) + 15) // 16 * 16  # 16-byte aligned; never read: every call here is refused or empty
INVALID, OK = 1, 0
BIG = 1 << 31

LOOKUP = dict(dtype=0, table=P, ldt=8, index=P, index_bytes=8, scale=1.0, out=P, ldo=8, n=2, V=4, D=8, stream=None)
SORT = dict(index=P, index_bytes=8, order=P, rows=P, workspace=P, workspace_bytes=1 << 40, n=20_000, V=4, stream=None)
GRADIENT = dict(dtype=0, grad=P, ldg=8, order=P, rows=P, scale=1.0, table_dtype=1, grad_table=P, ldt=8, workspace=P,
                workspace_bytes=1 << 40, n=2, V=4, D=8, stream=None)
WIDE = 65535 * 512 + 1

REFUSED = [
    ("spingtp_embedding", LOOKUP, [
        dict(dtype=2), dict(index_bytes=2), dict(ldt=7), dict(ldo=7), dict(n=-1), dict(n=BIG), dict(V=0), dict(V=BIG - 1), dict(D=0),
        dict(table=None), dict(table=P + 2), dict(out=None), dict(out=P + 1), dict(index=None), dict(index=P + 4),
        dict(index=P + 2, index_bytes=4), dict(ldt=1 << 47), dict(ldo=(1 << 63) - 1), dict(D=WIDE, ldt=BIG, ldo=BIG)]),
    ("spingtp_sort_index", SORT, [
        dict(index_bytes=1), dict(n=-1), dict(n=BIG), dict(V=0), dict(V=BIG - 1), dict(index=None), dict(index=P + 4),
        dict(order=None), dict(order=P + 2), dict(rows=None), dict(rows=P + 1), dict(workspace=None), dict(workspace=P + 8),
        dict(workspace_bytes=64)]),
    ("spingtp_embedding_backward", GRADIENT, [
        dict(dtype=-1), dict(table_dtype=2), dict(ldg=7), dict(ldt=7), dict(n=-1), dict(n=BIG), dict(V=0), dict(V=BIG - 1),
        dict(D=0), dict(grad=None), dict(grad=P + 2), dict(order=None), dict(order=P + 2), dict(rows=None), dict(grad_table=None),
        dict(grad_table=P + 1), dict(n=0, grad_table=None), dict(workspace=None), dict(workspace=P + 4), dict(workspace_bytes=8),
        dict(ldg=1 << 62), dict(ldt=1 << 62), dict(D=WIDE, ldg=BIG, ldt=BIG)]),
]


def call(name, args):
    return getattr(_lib.lib(), name)(*args.values())


@pytest.mark.parametrize("name,good,change", [(n, g, c) for n, g, cs in REFUSED for c in cs])
def test_refusals(name, good, change):
    assert call(name, {**good, **change}) == INVALID


@pytest.mark.parametrize("name,good,none", [
    ("spingtp_embedding", LOOKUP, dict(n=0, index=None, out=None)),
    ("spingtp_sort_index", SORT, dict(n=0, index=None, order=None, rows=None, workspace=None, workspace_bytes=0)),
])
def test_nothing_to_do(name, good, none):
    assert call(name, {**good, **none}) == OK


def test_workspace_sizes():
    n = ctypes.c_size_t(0)
    sort, gradient = _lib.lib().spingtp_sort_index_workspace_size, _lib.lib().spingtp_embedding_backward_workspace_size
    assert sort(8192, 1 << 30, ctypes.byref(n)) == OK and n.value == 0  # one workgroup's LDS
    assert sort(8193, 511, ctypes.byref(n)) == OK and n.value == 4 * 512 * 512  # one digit: counts alone
    assert sort(8193, 512, ctypes.byref(n)) == OK and n.value == 4 * (512 * 512 + 2 * 8196)
    assert gradient(0, 8, ctypes.byref(n)) == OK and n.value == 0
    assert gradient(100, 8, ctypes.byref(n)) == OK and n.value > 0
    for bad in ((-1, 4), (BIG, 4), (4, 0), (4, BIG)):
        assert sort(*bad, ctypes.byref(n)) == INVALID
        assert gradient(*bad, ctypes.byref(n)) == INVALID
    assert sort(4, 4, None) == INVALID and gradient(4, 4, None) == INVALID


class Tensor(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("param", "grad", "m", "v", "m_scales", "v_scales", "copy")] + [
        ("n", ctypes.c_int64), ("param_dtype", ctypes.c_int), ("grad_dtype", ctypes.c_int)]


class Options(ctypes.Structure):
    _fields_ = [(k, ctypes.c_double) for k in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [("step", ctypes.c_int64)] + [
        (k, ctypes.c_void_p) for k in ("device_step", "device_lr", "grad_scale")] + [("seed", ctypes.c_uint64)]


TENSOR = dict(param=P, grad=P, m=P, v=P, m_scales=None, v_scales=None, copy=None, n=8, param_dtype=0, grad_dtype=0)
EIGHT = dict(m_scales=P, v_scales=P)
OPTIONS = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1)
NAN, INF = float("nan"), float("inf")


def adamw(tensors, options, count=None):
    table = (Tensor * max(1, len(tensors)))(*(Tensor(**{**TENSOR, **t}) for t in tensors))
    o = Options(**{**OPTIONS, **options})
    return _lib.lib().spingtp_adamw(ctypes.byref(table), len(tensors) if count is None else count, ctypes.byref(o), None)


@pytest.mark.parametrize("change", [
    dict(param=None), dict(param=P + 2), dict(grad=None), dict(grad=P + 1), dict(m=None), dict(m=P + 2), dict(v=None), dict(v=P + 1),
    dict(n=-1), dict(n=(1 << 46) + 1), dict(param_dtype=2), dict(grad_dtype=-1), dict(m_scales=P), dict(v_scales=P),
    dict(EIGHT, m=P + 8), dict(EIGHT, v=P + 4), dict(copy=P + 1), dict(copy=P, param_dtype=1)])
def test_adamw_refuses_tensors(change):
    assert adamw([dict(n=0), change], {}) == INVALID


@pytest.mark.parametrize("change", [
    dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=NAN), dict(eps=-1.0), dict(eps=INF), dict(lr=NAN), dict(lr=INF),
    dict(weight_decay=INF), dict(step=0), dict(step=-5), dict(device_step=P + 4), dict(device_lr=P + 2), dict(grad_scale=P + 1)])
def test_adamw_refuses_options(change):
    assert adamw([{}], change) == INVALID


def test_adamw_of_nothing():
    assert adamw([], {}) == OK and adamw([dict(n=0, param=None, grad=None, m=None, v=None)] * 3, {}) == OK
    assert adamw([{}], {}, count=-1) == INVALID
    o = Options(**OPTIONS)
    assert _lib.lib().spingtp_adamw(None, 1, ctypes.byref(o), None) == INVALID
    assert _lib.lib().spingtp_adamw(None, 0, ctypes.byref(o), None) == OK
    assert _lib.lib().spingtp_adamw(None, 0, None, None) == INVALID


@pytest.mark.slow
def test_the_checks_pass_under_sanitizers():
    if os.environ.get("SPINGTP_LIBRARY"):
        pytest.skip("already under them")
    from paper_2607_01408_amd import build

    env = dict(os.environ)
    env.update({
        "LD_PRELOAD": build.sanitizer_runtime(),
        "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=1",
        "UBSAN_OPTIONS": "print_stacktrace=1:halt_on_error=1",
        "SPINGTP_LIBRARY": build.build_sanitized(),
    })
    files = [os.path.join(ROOT, "tests", f) for f in ("test_training_host.py", "test_linear_host.py")]
    r = subprocess.run([sys.executable, "-m", "pytest", *files, "-q", "-x", "-p", "no:cacheprovider", "-m", "not gpu"], cwd=ROOT,
                       env=env, capture_output=True, text=True, timeout=1500)
    tail = (r.stdout + r.stderr)[-3000:]
    assert r.returncode == 0, tail
    assert "AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, tail
    assert " passed" in r.stdout, tail
