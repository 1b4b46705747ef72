"""Where the linear layer may write its output (GPU)."""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2607_01408_amd as sg  # noqa: E402
from tests.test_gpu_linear import BF16, F32, rand  # noqa: E402

M, K, N = 40, 64, 64


def test_outputs_over_other_operands_are_refused():
    x, w, b = rand((M, K), BF16, 1), rand((N, K), BF16, 2), rand((N,), F32, 3)
    x8, w8 = sg.pack8(rand((M, 256), BF16, 4)), sg.pack8(rand((N, 256), BF16, 5))
    r = rand((M + 2, N + 8), BF16, 6)
    wide = rand((M, N), F32, 7)
    keep = [t.clone() for t in (x, w, b, r, wide)]
    blocks = [t.view(torch.uint8).clone() for t in (x8.values, w8.values, x8.scales, w8.scales)]
    over = {
        "the residual a row further": lambda: sg.linear(x, w, residual=r[:M, :N], out=r[1 : M + 1, :N]),
        "a column further": lambda: sg.linear(x, w, residual=r[:M, :N], out=r[:M, 1 : N + 1]),
        "its last column": lambda: sg.linear(x, w, residual=r[:M, :N], out=r.view(-1)[N - 1 : N - 1 + M * (N + 8)].view(M, N + 8)[:, :N]),
        "the same start at another stride": lambda: sg.linear(x, w, residual=r.view(-1)[: M * N].view(M, N), out=r[:M, :N]),
        "x": lambda: sg.linear(x, w, out=x),
        "w": lambda: sg.linear(x, w, out=w[:M, :]),
        "a bias in it": lambda: sg.linear(x, w, bias=wide[M - 1], out=wide, dtype=F32),
        "x's blocks": lambda: sg.linear(x8, w8, out=x8.values.view(BF16)[:, :N]),
        "w's blocks": lambda: sg.linear(x8, w8, out=w8.values.view(BF16)[:M, 3 : N + 3]),
        "a residual beside 8 bits": lambda: sg.linear(x8, w8, residual=r[:M, :N], out=r[2:, :N]),
    }
    for name, call in over.items():
        with pytest.raises(ValueError, match="overlap"):
            call()
            pytest.fail(f"{name} was not refused")
    assert all(torch.equal(a, k) for a, k in zip((x, w, b, r, wide), keep))
    assert all(torch.equal(t.view(torch.uint8), k) for t, k in zip((x8.values, w8.values, x8.scales, w8.scales), blocks))


def test_outputs_beside_other_operands_are_written():
    x, w = rand((M, K), BF16, 1), rand((N, K), BF16, 2)
    x8, w8 = sg.pack8(x), sg.pack8(w)
    buffer = rand((M, 2 * N + K), BF16, 3)
    left, right, inside = buffer[:, :N], buffer[:, N : 2 * N], buffer[:, 2 * N :]
    inside.copy_(x)
    want, want8 = sg.linear(x, w, residual=left)[0], sg.linear(x8, w8, residual=left)[0]
    assert sg.linear(inside, w, residual=left, out=right)[0] is right and torch.equal(right, want)
    sg.linear(x8, w8, residual=left, out=right)
    assert torch.equal(right, want8)
    # rows of a residual between the output's, at half their stride
    pairs = rand((2 * M, N), BF16, 4)
    odd = pairs.view(M, 2 * N)[:, N:]
    want = sg.linear(x[:1], w, residual=pairs[:1])[0]
    sg.linear(x[:1], w, residual=pairs[:1], out=odd[:1])
    assert torch.equal(odd[:1], want)
    r = rand((M, N), BF16, 5)
    want = sg.linear(x, w, residual=r)[0]
    assert sg.linear(x, w, residual=r, out=r)[0] is r and torch.equal(r, want)


def test_a_given_output_is_seen_by_autograd():
    x, w = rand((M, K), BF16, 1), rand((N, K), BF16, 2)
    x8, w8 = sg.pack8(x), sg.pack8(w)
    for call in (lambda out: sg.linear(x, w, residual=out, out=out), lambda out: sg.linear(x8, w8, out=out),
                 lambda out: sg.matmul8(x8, w8, out=out), lambda out: sg.unpack8(x8, out=out)):
        out = rand((M, N), BF16, 3)
        factor = torch.ones((M, N), dtype=BF16, device="cuda", requires_grad=True)
        kept = (out * factor).sum()
        before = out._version
        call(out)
        assert out._version > before
        with pytest.raises(RuntimeError, match="inplace"):
            kept.backward()
