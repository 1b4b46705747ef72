"""The argument checks of the feed-forward entry points (no GPU needed): each refusal comes before any launch."""

import ctypes

import pytest

from paper_2607_01408_amd import _lib

BUF = ctypes.create_string_buffer(4096 + 16)
P = (ctypes.addressof(BUF) + 15) // 16 * 16  # 16-byte aligned; never read: every call here is refused or empty
INVALID, OK = 1, 0

PACK = dict(dtype=0, x=P, ldx=8, values=P, scales=P, t_values=None, t_scales=None, R=2, D=8, stream=None)
UNPACK = dict(values=P, scales=P, dtype=0, x=P, ldx=8, R=2, D=8, stream=None)
NORM = dict(dtype=1, x=P, ldx=8, residual=None, ldr=0, gain=P, eps=1e-6, h=None, ldh=0, y=P, ldy=8, values=None,
            scales=None, rstd=P, R=2, D=8, stream=None)
NORM_BWD = dict(dtype=1, grad_y=P, ldg=8, h=P, ldh=8, rstd=P, gain=P, grad_h=None, ldgh=0, grad_x=P, ldx=8, grad_gain=P,
                workspace=P, workspace_bytes=4096, R=2, D=8, stream=None)
MATMUL = dict(a_values=P, a_scales=P, b_values=P, b_scales=P, dtype=0, c=P, ldc=4, M=2, N=4, K=8, stream=None)
GATED = dict(act=0, x=P, ldx=8, w_gate=P, w_up=P, ldw=8, h=P, ldh=4, save=0, g=None, g_scales=None, u=None, u_scales=None,
             workspace=None, workspace_bytes=0, M=2, K=8, F=4, stream=None)
GATED8 = dict(act=0, x=P, x_scales=P, w_gate=P, w_gate_scales=P, w_up=P, w_up_scales=P, h=P, ldh=4, h_scales=None,
              workspace=P, workspace_bytes=4096, M=2, K=8, F=4, stream=None)
GATED_BWD = dict(act=0, grad_h=P, ldgh=4, save=1, g=P, g_scales=None, u=P, u_scales=None, x=P, ldx=8, x_scales=None,
                 w_gate=P, w_up=P, ldw=8, grad_x=P, ldgx=8, grad_w=P, workspace=P, workspace_bytes=1 << 30, M=2, K=8, F=4,
                 stream=None)
BIG = 1 << 31

REFUSED = [
    ("spingtp_pack8", PACK, [dict(dtype=2), dict(D=0), dict(R=-1), dict(R=BIG), dict(ldx=7), dict(x=None), dict(x=P + 1),
                             dict(values=None), dict(values=None, scales=None), dict(scales=None), dict(values=P + 8),
                             dict(t_values=P), dict(t_values=P, t_scales=P, D=128 * 65535 + 1, ldx=BIG), dict(ldx=1 << 47)]),
    ("spingtp_unpack8", UNPACK, [dict(dtype=-1), dict(D=0), dict(ldx=7), dict(values=None), dict(scales=P + 2), dict(x=P + 2),
                                 dict(R=BIG)]),
    ("spingtp_rms_norm", NORM, [dict(dtype=3), dict(D=0), dict(ldx=7), dict(x=None), dict(x=P + 1), dict(gain=None),
                                dict(eps=-1.0), dict(eps=float("nan")), dict(y=None), dict(values=P, scales=P),
                                dict(y=None, values=P), dict(residual=P, ldr=8), dict(residual=P, ldr=7, h=P, ldh=8),
                                dict(h=P, ldh=7), dict(ldy=7), dict(rstd=P + 1), dict(y=None, values=P + 8, scales=P)]),
    ("spingtp_rms_norm_backward", NORM_BWD, [dict(dtype=2), dict(D=0), dict(ldg=7), dict(ldh=7), dict(ldx=7), dict(h=None),
                                             dict(grad_y=None), dict(rstd=None), dict(gain=None), dict(grad_x=None),
                                             dict(grad_h=P, ldgh=7), dict(workspace=None), dict(workspace_bytes=8)]),
    ("spingtp_matmul8", MATMUL, [dict(dtype=2), dict(K=0), dict(M=-1), dict(N=BIG), dict(ldc=3), dict(a_values=None),
                                 dict(a_values=P + 8), dict(a_scales=None), dict(b_scales=P + 1), dict(b_values=None),
                                 dict(c=None), dict(c=P + 2), dict(K=128 * 65535 + 1)]),
    ("spingtp_gated_forward", GATED, [dict(act=2), dict(K=0), dict(F=0), dict(M=-1), dict(ldx=7), dict(ldw=7), dict(ldh=3),
                                      dict(x=P + 2), dict(w_gate=None), dict(w_up=P + 8), dict(h=None), dict(save=3),
                                      dict(save=1), dict(save=1, g=P), dict(save=2, g=P, u=P),
                                      dict(save=2, g=P, u=P, g_scales=P, u_scales=P),
                                      dict(K=7, M=65), dict(ldx=9, M=65), dict(K=7, M=65, workspace=P, workspace_bytes=16), dict(F=32 * 65535 + 1, ldh=BIG), dict(K=64 * 65535 + 1, ldx=BIG, ldw=BIG)]),
    ("spingtp_gated_forward8", GATED8, [dict(act=-1), dict(K=0), dict(F=0), dict(ldh=3), dict(x=None), dict(x_scales=None),
                                        dict(w_gate=P + 8), dict(w_gate_scales=None), dict(w_up=None),
                                        dict(w_up_scales=P + 2), dict(h=None), dict(h=P + 2, h_scales=P),
                                        dict(h_scales=P, workspace=None), dict(h_scales=P, workspace_bytes=16)]),
    ("spingtp_gated_backward", GATED_BWD, [dict(act=2), dict(save=0), dict(save=2), dict(ldgh=3), dict(ldx=7), dict(ldw=7),
                                           dict(ldgx=7), dict(g=None), dict(u=P + 8), dict(x=None), dict(w_gate=None),
                                           dict(grad_h=None), dict(workspace=None), dict(workspace_bytes=64),
                                           dict(x_scales=P + 1), dict(w_gate=P + 2), dict(x=P + 2)]),
]


def call(name, args):
    return getattr(_lib.lib(), name)(*args.values())


@pytest.mark.parametrize("name,good,change", [(n, g, c) for n, g, cs in REFUSED for c in cs])
def test_refusals(name, good, change):
    assert call(name, {**good, **change}) == INVALID


@pytest.mark.parametrize("name,good,none", [
    ("spingtp_pack8", PACK, dict(R=0, x=None)), ("spingtp_unpack8", UNPACK, dict(R=0, x=None, values=None, scales=None)),
    ("spingtp_rms_norm", NORM, dict(R=0, x=None)), ("spingtp_matmul8", MATMUL, dict(M=0, a_values=None, c=None)),
    ("spingtp_matmul8", MATMUL, dict(N=0, b_values=None, c=None, ldc=1)), ("spingtp_gated_forward", GATED, dict(M=0, x=None)),
    ("spingtp_gated_forward8", GATED8, dict(M=0, x=None)),
    ("spingtp_gated_backward", GATED_BWD, dict(grad_x=None, grad_w=None)),
])
def test_nothing_to_do(name, good, none):
    assert call(name, {**good, **none}) == OK


@pytest.mark.parametrize("name,sizes", [("spingtp_rms_norm_backward_workspace_size", (2, 0)),
                                        ("spingtp_gated_forward_workspace_size", (65, 8, 4, 7, 8, 0)),
                                        ("spingtp_gated_forward8_workspace_size", (0, 0, 4, 1)),
                                        ("spingtp_gated_backward_workspace_size", (2, 8, 0, 8, 8, 0))])
def test_workspace_sizes(name, sizes):
    n = ctypes.c_size_t(0)
    fn = getattr(_lib.lib(), name)
    assert fn(*sizes, ctypes.byref(n)) == INVALID
    good = tuple(max(s, 9) if i < 5 else s for i, s in enumerate(sizes))
    assert fn(*good, None) == INVALID
    assert fn(*good, ctypes.byref(n)) == OK and n.value > 0


def test_workspace_grows_with_the_operands():
    n = ctypes.c_size_t(0)
    fn = _lib.lib().spingtp_gated_forward_workspace_size
    assert fn(100, 64, 32, 64, 64, 0, ctypes.byref(n)) == OK and n.value == 0  # rows on 16 bytes: read as they are
    assert fn(100, 63, 32, 63, 63, 1, ctypes.byref(n)) == OK and n.value == 2 * 64 * (100 + 2 * 32)
    assert fn(100, 64, 32, 65, 64, 2, ctypes.byref(n)) == OK and n.value == 2 * 64 * 100
    assert fn(32, 63, 32, 63, 63, 1, ctypes.byref(n)) == OK and n.value == 0  # few rows: as they are
    assert fn(32, 63, 32, 63, 63, 2, ctypes.byref(n)) == OK and n.value == 4 * 2 * 32 * 32  # g and u in fp32
    assert fn(32, 63, 32, 63, 63, 3, ctypes.byref(n)) == INVALID
    fn = _lib.lib().spingtp_gated_forward8_workspace_size
    assert fn(32, 64, 100, 1, ctypes.byref(n)) == OK and n.value == 4 * 32 * 100
    assert fn(65, 64, 100, 1, ctypes.byref(n)) == OK and n.value == 0
    assert fn(1, 64, 100, 0, ctypes.byref(n)) == OK and n.value == 0
    fn = _lib.lib().spingtp_gated_backward_workspace_size
    assert fn(100, 64, 100, 64, 72, 0, ctypes.byref(n)) == OK and n.value == 2 * 100 * 256  # g and u alone
    assert fn(100, 64, 100, 65, 72, 0, ctypes.byref(n)) == OK and n.value == 2 * 100 * (256 + 64)
    assert fn(100, 64, 100, 0, 72, 1, ctypes.byref(n)) == OK and n.value == 2 * 100 * (256 + 64)
    assert fn(100, 63, 100, 63, 63, 0, ctypes.byref(n)) == OK and n.value == 2 * (100 * (256 + 64) + 2 * 100 * 64)
    assert fn(100, 64, 100, 63, 64, 0, ctypes.byref(n)) == INVALID


@pytest.mark.parametrize("name,good,change", [
    ("spingtp_matmul8", MATMUL, dict(M=(1 << 30) + 1, N=4)), ("spingtp_matmul8", MATMUL, dict(M=2, N=(1 << 30) + 1, ldc=BIG)),
    ("spingtp_gated_forward", GATED, dict(M=(1 << 30) + 1)), ("spingtp_gated_forward8", GATED8, dict(M=(1 << 30) + 1)),
    ("spingtp_gated_backward", GATED_BWD, dict(M=(1 << 30) + 1, workspace_bytes=1 << 60)),
    ("spingtp_gated_backward", GATED_BWD, dict(M=(1 << 23), K=1 << 18, ldx=1 << 18, ldw=1 << 18, ldgx=1 << 18, workspace_bytes=1 << 60)),
])
def test_more_tiles_than_a_launch_holds_are_refused(name, good, change):
    assert call(name, {**good, **change}) == INVALID


@pytest.mark.parametrize("ld", [(1 << 46) + 1, 1 << 62, (1 << 63) - 1])
def test_strides_out_of_range_have_no_workspace_size(ld):
    n = ctypes.c_size_t(0)
    forward, backward = (getattr(_lib.lib(), f"spingtp_gated_{d}_workspace_size") for d in ("forward", "backward"))
    for M in (1, 100):
        assert forward(M, 64, 32, ld, 64, 0, ctypes.byref(n)) == INVALID
        assert forward(M, 64, 32, 64, ld, 0, ctypes.byref(n)) == INVALID
        assert backward(M, 64, 32, ld, 64, 0, ctypes.byref(n)) == INVALID
        assert backward(M, 64, 32, 64, ld, 0, ctypes.byref(n)) == INVALID
        assert backward(M, 64, 32, ld, 64, 1, ctypes.byref(n)) == OK  # x in 8 bits: its stride is not used
    for name, good, change in (("spingtp_gated_forward", GATED, dict(ldx=ld)), ("spingtp_gated_forward", GATED, dict(ldw=ld)),
                               ("spingtp_gated_backward", GATED_BWD, dict(ldx=ld)),
                               ("spingtp_gated_backward", GATED_BWD, dict(ldw=ld))):
        assert call(name, {**good, **change}) == INVALID
