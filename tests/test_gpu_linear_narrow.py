"""The linear layer's gradients for many rows and few channels, whose dz and grad_x are made in one launch (GPU); bounds as in
test_gpu_linear.py."""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2607_01408_amd as sg  # noqa: E402
from tests.test_gpu_linear import test_backward as backward  # noqa: E402
from tests.test_gpu_linear import (ACTS, BF16, F32, HALF, INF, NAN, amid, backward64, rand, within)  # noqa: E402

# one tile of rows a workgroup and more; sums that end inside a step; channels from a chunk of 8 to all 128; the fewest rows,
# the most outputs
SHAPES = [(40_000, 128, 512), (40_001, 8, 8), (66_000, 128, 64), (45_011, 64, 200), (65_537, 120, 72), (70_001, 16, 520),
          (100_003, 128, 136), (41_001, 72, 2048), (43_007, 100, 264), (50_001, 3, 40)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_gradients(M, K, N, act):
    backward(M, K, N, act)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K,N", [(40_000, 128, 64), (45_011, 40, 200)])
def test_rows_with_others_beside_them(M, K, N, dtype):
    x, w, z, dy = rand((M, K), BF16, 1), rand((N, K), BF16, 2, K**-0.5), rand((M, N), BF16, 3), rand((M, N), dtype, 4)
    for act in ("silu", "gelu"):
        want = sg.linear_backward(dy, sg.LinearSaved(x, z, act), w)
        got = sg.linear_backward(amid(dy), sg.LinearSaved(amid(x), z, act), amid(w))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("shift", [1, 4])
def test_rows_off_16_bytes_take_the_other_way(shift):
    M, K, N = 41_000, 128, 96
    x, w, z, dy = rand((M, K), BF16, 1), rand((N, K), BF16, 2, K**-0.5), rand((M, N), BF16, 3), rand((M, N), BF16, 4)
    (rx, ex), (rw, ew), (rb, eb) = backward64(dy, z, "silu", x.double(), w.double())
    gx, gw, gb = sg.linear_backward(amid(dy, shift=shift), sg.LinearSaved(x, z, "silu"), w)
    within(gx, rx, ex + HALF[BF16] * (rx.abs() + ex) + 1e-38)
    within(gw, rw, ew + HALF[BF16] * (rw.abs() + ew) + 1e-38)
    within(gb, rb, eb + 1e-38)


def test_values_that_are_not_numbers_stay_in_their_rows():
    M, K, N = 50_003, 120, 200
    x, w, z, dy = rand((M, K), BF16, 1), rand((N, K), BF16, 2), rand((M, N), BF16, 3), rand((M, N), BF16, 4)
    for at in (0, 127, 128, 9_999, M - 1):
        for value in (NAN, INF):
            bad = dy.clone()
            bad[at, 7] = value
            gx, gw, gb = sg.linear_backward(bad, sg.LinearSaved(x, z, "silu"), w)
            others = torch.arange(M, device="cuda") != at
            assert not bool(torch.isfinite(gx[at]).any()) and bool(torch.isfinite(gx[others]).all())
            others = torch.arange(N, device="cuda") != 7
            assert not bool(torch.isfinite(gw[7]).any()) and bool(torch.isfinite(gw[others]).all())
            assert not bool(torch.isfinite(gb[7])) and bool(torch.isfinite(gb[others]).all())


@pytest.mark.parametrize("K,lddx,shift", [(128, 136, 0), (128, 129, 0), (96, 104, 1), (100, 100, 0), (37, 40, 0)])
def test_from_c_without_weights_and_onto_any_rows(K, lddx, shift):
    """Without grad_x there need not be weights, and grad_bias and grad_w have the same bits as with it; grad_x onto rows with
    others beside them."""
    import ctypes

    from paper_2607_01408_amd import _lib

    C = _lib.lib()
    M, N = 42_003, 72
    x, w, z, dy = rand((M, K), BF16, 1), rand((N, K), BF16, 2, K**-0.5), rand((M, N), BF16, 3), rand((M, N), BF16, 4)
    want = sg.linear_backward(dy, sg.LinearSaved(x, z, "silu"), w)
    wide = torch.full((M * lddx + 16,), 9.0, dtype=BF16, device="cuda")
    gx = wide[shift : shift + M * lddx].view(M, lddx)
    gw, gb = torch.empty((N, K), dtype=BF16, device="cuda"), torch.empty(N, device="cuda")

    def p(t):
        return None if t is None else ctypes.c_void_p(t.data_ptr())

    def run(w, gx):
        n = ctypes.c_size_t()
        head = (ctypes.c_int(0), ctypes.c_int(1), p(dy), ctypes.c_int64(N))
        tail = tuple(ctypes.c_int64(v) for v in (M, K, N))
        size = C.spingtp_linear_backward_workspace_size
        assert size(*head, p(x), ctypes.c_int64(K), p(w), ctypes.c_int64(K), p(gx), p(gw), p(gb), *tail, ctypes.byref(n)) == 0
        ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
        stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        assert C.spingtp_linear_backward(*head, p(z), p(x), ctypes.c_int64(K), p(w), ctypes.c_int64(K), p(gx),
                                         ctypes.c_int64(lddx), ctypes.c_int(1), p(gw), p(gb), p(ws),
                                         ctypes.c_size_t(n.value), *tail, stream) == 0
        torch.cuda.synchronize()

    run(w, gx)
    assert all(torch.equal(a, b) for a, b in zip((gx[:, :K], gw, gb), want))
    assert bool((gx[:, K:] == 9).all()) and bool((wide[:shift] == 9).all()) and bool((wide[shift + M * lddx :] == 9).all())
    gw.fill_(0), gb.fill_(0)
    run(None, None)
    assert torch.equal(gw, want[1]) and torch.equal(gb, want[2])


def test_a_captured_backward_replays():
    M, K, N = 48_000, 96, 264
    x, w, z, dy = rand((M, K), BF16, 1), rand((N, K), BF16, 2, K**-0.5), rand((M, N), BF16, 3), rand((M, N), BF16, 4)
    saved = sg.LinearSaved(x, z, "gelu")
    sg.linear_backward(dy, saved, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = sg.linear_backward(dy, saved, w)
    for i in range(3):
        dy.copy_(rand((M, N), BF16, 10 + i))
        graph.replay()
        want = sg.linear_backward(dy, saved, w)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
