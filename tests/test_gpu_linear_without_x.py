"""The linear layer's gradients of many rows and few channels where grad_x is not wanted, a first layer (GPU)."""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2607_01408_amd as sg  # noqa: E402
from tests.test_gpu_linear import ACTS, BF16, F32, amid, rand  # noqa: E402


# columns of every width of a row's lanes, at its ends and between; rows that fill a workgroup's tiles and do not
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M", [40_000, 65_536, 70_001])
@pytest.mark.parametrize("N", [8, 64, 72, 128, 136, 256, 264, 512, 520, 1024, 1032, 2040, 2048])
def test_the_same_bits_as_with_it(M, N, act):
    K = 16
    x, w, z = rand((M, K), BF16, 1), rand((N, K), BF16, 2), rand((M, N), BF16, 3, 2.0) if act else None
    for dtype in (BF16, F32):
        dy = rand((M, N), dtype, 4)
        for g in (dy, amid(dy)):
            saved = sg.LinearSaved(x, z, act)
            _, gw, gb = sg.linear_backward(g, saved, w, dtype=F32)
            for need_w, need_bias in ((True, True), (True, False), (False, True)):
                none, a, b = sg.linear_backward(g, saved, w, False, need_w, need_bias, F32)
                assert none is None and (not need_w or torch.equal(a, gw)) and (not need_bias or torch.equal(b, gb))


def test_it_takes_less_time_than_with_it():
    """200,000 x 2,048 by 128, silu: all gradients 820 us, without grad_x 680; 788 where its product's steps and barriers are
    gone through all the same."""
    M, K, N = 200_000, 128, 2048
    x, w, z, dy = rand((M, K), BF16, 1), rand((N, K), BF16, 2), rand((M, N), BF16, 3), rand((M, N), BF16, 4)
    saved = sg.LinearSaved(x, z, "silu")

    def least(need_x):
        times = []
        for _ in range(20):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(3):
                sg.linear_backward(dy, saved, w, need_x=need_x)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    assert least(False) <= 0.91 * least(True)
