"""The activations' derivatives in the linear layer's gradients, in fp32 (GPU).

grad_bias of a column with a single row whose grad_y is 1, all others 0, is the derivative itself.  silu' = t (1 + z (1 - t)) and
gelu' = Phi + z phi are off by at most 2^-20 of the magnitudes of their terms, t (1 + |z|) and Phi + |z| phi: the exponential
and the reciprocal are off by 2^-23 each, gelu's polynomial by 6 2^-24, and five other operations by 2^-24 each; arguments and
their squares are exact (bf16)."""

import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2607_01408_amd as sg  # noqa: E402
from tests.test_gpu_linear import BF16, F32, act64, rand  # noqa: E402


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act,least", [("silu", -84.0), ("gelu", -12.5)])
@pytest.mark.parametrize("M", [5, 300, 40_000])  # dz by itself, and in one launch with grad_x
def test_slopes(M, act, least, dtype):
    K, N = 8, 1024
    at = torch.linspace(least, 12.0, N, device="cuda").to(BF16)
    z = rand((M, N), BF16, 1)
    dy = torch.zeros((M, N), dtype=dtype, device="cuda")
    row = torch.arange(N, device="cuda") * 7919 % M
    z[row, torch.arange(N)] = at
    dy[row, torch.arange(N)] = 1
    x, w = rand((M, K), BF16, 2), rand((N, K), BF16, 3)
    want = act64(at.double(), act)[1]
    if act == "silu":
        size = torch.sigmoid(at.double()) * (1 + at.double().abs())
    else:
        g = at.double()
        size = 0.5 * torch.erfc(-g / math.sqrt(2)) + g.abs() * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    for need_x in (True, False):
        got = sg.linear_backward(dy, sg.LinearSaved(x, z, act), w, need_x=need_x, need_w=False)[2]
        off = ((got.double() - want).abs() / size).max()
        assert float(off) <= 2.0**-20, float(off) * 2.0**20
