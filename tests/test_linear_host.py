"""The argument checks and workspace sizes of the linear layer's entry points (no GPU needed): each refusal comes
before any launch."""

import ctypes

import pytest

from paper_2607_01408_amd import _lib

BUF = ctypes.create_string_buffer(4096 + 16)
P = (ctypes.addressof(BUF) + 15) // 16 * 16  # 16-byte aligned; never read: every call here is refused or empty
INVALID, OK = 1, 0
BIG = 1 << 31

FORWARD = dict(act=0, x=P, ldx=8, w=P, ldw=8, bias=P, dtype=0, residual=P, ldr=4, y=P, ldy=4, z=P, workspace=P,
               workspace_bytes=1 << 40, M=2, K=8, N=4, stream=None)
FORWARD8 = dict(act=0, x=P, x_scales=P, w=P, w_scales=P, bias=P, dtype=1, residual=P, ldr=4, y=P, ldy=4, workspace=P,
                workspace_bytes=1 << 40, M=2, K=8, N=4, stream=None)
BACKWARD = dict(act=0, dtype=1, grad_y=P, ldg=4, z=P, x=P, ldx=8, w=P, ldw=8, grad_x=P, ldgx=8, w_dtype=0, grad_w=P,
                grad_bias=P, workspace=P, workspace_bytes=1 << 40, M=2, K=8, N=4, stream=None)
LONG = 64 * 65535 + 1

REFUSED = [
    ("spingtp_linear_forward", FORWARD, [
        dict(act=3), dict(act=-1), dict(dtype=2), dict(M=-1), dict(K=0), dict(N=0), dict(M=BIG), dict(ldx=7), dict(ldw=7),
        dict(ldr=3), dict(ldy=3), dict(x=None), dict(x=P + 1), dict(w=None), dict(w=P + 1), dict(bias=P + 2), dict(y=None),
        dict(y=P + 2), dict(residual=P + 2), dict(z=P + 1), dict(K=LONG, ldx=BIG, ldw=BIG), dict(N=LONG, ldy=BIG, ldr=BIG),
        dict(ldx=1 << 47), dict(ldw=(1 << 63) - 1), dict(ldy=1 << 62), dict(ldr=1 << 62), dict(M=(1 << 30) + 1),
        dict(M=100, K=7, workspace=None), dict(M=100, K=7, workspace=P + 8), dict(M=100, K=7, workspace_bytes=64)]),
    ("spingtp_linear_forward8", FORWARD8, [
        dict(act=3), dict(dtype=-1), dict(M=-1), dict(K=0), dict(N=0), dict(N=BIG), dict(ldr=3), dict(ldy=3), dict(x=None),
        dict(x=P + 8), dict(x_scales=None), dict(x_scales=P + 2), dict(w=P + 8), dict(w_scales=None), dict(bias=P + 1),
        dict(y=None), dict(y=P + 1), dict(residual=P + 1), dict(K=128 * 65535 + 1), dict(N=LONG, ldy=BIG, ldr=BIG),
        dict(M=(1 << 30) + 1), dict(K=65536, workspace=None), dict(K=65536, workspace_bytes=64)]),
    ("spingtp_linear_backward", BACKWARD, [
        dict(act=3), dict(dtype=2), dict(w_dtype=2), dict(M=-1), dict(K=0), dict(N=0), dict(ldg=3), dict(ldx=7), dict(ldw=7),
        dict(ldgx=7), dict(grad_y=None), dict(grad_y=P + 1), dict(z=None), dict(z=P + 1), dict(x=None), dict(x=P + 1),
        dict(w=None), dict(w=P + 1), dict(grad_x=P + 1), dict(grad_w=P + 2), dict(grad_bias=P + 2), dict(workspace=None),
        dict(workspace=P + 4), dict(workspace_bytes=64), dict(ldg=1 << 62), dict(ldgx=1 << 62), dict(M=(1 << 30) + 1),
        dict(N=LONG, ldg=BIG), dict(K=LONG, ldx=BIG, ldw=BIG, ldgx=BIG)]),
]


def call(name, args):
    return getattr(_lib.lib(), name)(*args.values())


@pytest.mark.parametrize("name,good,change", [(n, g, c) for n, g, cs in REFUSED for c in cs])
def test_refusals(name, good, change):
    assert call(name, {**good, **change}) == INVALID


@pytest.mark.parametrize("name,good,none", [
    ("spingtp_linear_forward", FORWARD, dict(M=0, x=None, y=None, workspace=None, workspace_bytes=0)),
    ("spingtp_linear_forward8", FORWARD8, dict(M=0, x=None, y=None, workspace=None, workspace_bytes=0)),
    ("spingtp_linear_backward", BACKWARD, dict(grad_x=None, grad_w=None, grad_bias=None, z=None, grad_y=None)),
])
def test_nothing_to_do(name, good, none):
    assert call(name, {**good, **none}) == OK


def size(name, *args):
    n = ctypes.c_size_t(0)
    assert getattr(_lib.lib(), name)(*args, ctypes.byref(n)) == OK
    return n.value


def test_workspace_sizes():
    forward, backward = "spingtp_linear_forward_workspace_size", "spingtp_linear_backward_workspace_size"
    assert size(forward, P, 64, P, 64, 100, 64, 32) == 0  # rows on 16 bytes: read as they are
    assert size(forward, P, 63, P, 63, 100, 63, 32) == 2 * 64 * (100 + 32)
    assert size(forward, P + 2, 64, P, 64, 100, 64, 32) == 2 * 64 * 100
    assert size(forward, P, 64, P + 2, 64, 100, 64, 32) == 2 * 64 * 32
    assert size(forward, P + 2, 63, P, 63, 10, 63, 32) == 0  # few rows: as they are
    assert size(forward, P, 65536, P, 65536, 1, 65536, 16) % (4 * 16) == 0  # slices' sums
    assert size(forward, P, 65536, P, 65536, 1, 65536, 16) > 0
    assert size(forward, None, 64, None, 64, 0, 64, 32) == 0
    assert size("spingtp_linear_forward8_workspace_size", 100, 64, 32) == 0
    args = [2, 1, P, 104, P, 64, P, 64, P, None, None, 100, 64, 104]
    assert size(backward, *args) == 0  # the gradient as it is
    args[2] = P + 2
    assert size(backward, *args) == 2 * 100 * 128
    args[2], args[0] = P, 0
    assert size(backward, *args) == 2 * 100 * 128
    args[10] = P
    assert size(backward, *args) > 2 * 100 * 128
    n = ctypes.c_size_t(0)
    for bad in ([3] + args[1:], args[:3] + [103] + args[4:], args[:7] + [63] + args[8:]):
        assert getattr(_lib.lib(), backward)(*bad, ctypes.byref(n)) == INVALID
    assert getattr(_lib.lib(), backward)(*args, None) == INVALID
    assert getattr(_lib.lib(), forward)(P, 64, P, 64, 100, 64, 32, None) == INVALID
