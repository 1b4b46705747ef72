"""The linear layer against float64 (GPU).

Bounds, from the number formats alone:
  * a rounding is off by at most half a step: bf16 2^-8, fp32 2^-24 of the value;
  * a sum of K products in fp32 is off by at most K 2^-24 of the sum of their magnitudes, however it is cut into
    parts; products of bf16 numbers are exact;
  * an activation is off by 2^-20 of its argument, and has a derivative of at most 1.13.
"""

import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)

from tests import linear_shapes as shapes  # noqa: E402
import paper_2607_01408_amd as sg  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0**-24, BF16: 2.0**-8}
NAN, INF = float("nan"), float("inf")
ACTS = [None, "silu", "gelu"]


def rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def within(got, ref, bound, what=""):
    """|got - ref| <= bound everywhere; non-finite values in the same places."""
    got = got.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), fine), what
    over = ((got - ref).abs() - bound)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, (what, float(over.max()))


def act64(z, name):
    """(a(z), a'(z))."""
    if name is None:
        return z, torch.ones_like(z)
    if name == "silu":
        t = torch.sigmoid(z)
        return z * t, t * (1 + z * (1 - t))
    p = 0.5 * torch.erfc(-z / math.sqrt(2))
    return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def as64(b):
    s = torch.exp2(b.scales.view(torch.uint8).double() - 127).repeat_interleave(128, 1)
    return (b.values.double() * s[:, : b.values.shape[1]])[:, : b.shape[1]]


def forward64(x, w, bias, act, residual, dtype):
    """(z, its bound in fp32, y, its bound)."""
    K = x.shape[1]
    z, size = x @ w.t(), x.abs() @ w.abs().t()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    ez = (K + 64) * 2.0**-24 * size
    y = act64(z, act)[0]
    ey = 1.13 * ez + (2.0**-20 * z.abs() if act else 0)
    if residual is not None:
        y = y + residual.double()
        ey = ey + 2.0**-24 * (y.abs() + ey)
    return z, ez, y, ey + HALF[dtype] * (y.abs() + ey) + 1e-38


# few rows; every tile, with the sum in one piece and in slices; odd sizes and copied rows
SHAPES = [(1, 1, 1), (1, 64, 16), (1, 2048, 301), (3, 130, 70), (7, 5003, 20), (16, 640, 200), (17, 96, 129), (33, 100, 130),
          (64, 72, 300), (64, 4000, 31), (65, 257, 64), (70, 8200, 65), (130, 1100, 130), (300, 72, 500), (257, 2100, 300),
          (999, 200, 273), (2001, 1160, 2100), (513, 1000, 1100), (4090, 700, 8189), (5000, 129, 70)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_forward(M, K, N, act):
    x, w = rand((M, K), BF16, 1), rand((N, K), BF16, 2, K**-0.5)
    bias = rand((N,), F32, 3) if (M + N) % 3 else None
    for dtype in (BF16, F32):
        residual = rand((M, N), dtype, 4) if (K + N) % 2 or dtype == F32 else None
        z, ez, y, ey = forward64(x.double(), w.double(), bias, act, residual, dtype)
        got, saved = sg.linear(x, w, bias=bias, act=act, residual=residual, dtype=dtype)
        assert saved is None and got.dtype == dtype and got.shape == (M, N)
        within(got, y, ey)
        again, saved = sg.linear(x, w, bias=bias, act=act, residual=residual, dtype=dtype, save="same")
        assert torch.equal(got, again) and saved.x is x and saved.act == act
        if act is None:
            assert saved.z is None
        else:
            within(saved.z, z, ez + HALF[BF16] * (z.abs() + ez))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_forward_from_8_bits(M, K, N, act):
    x, w = sg.pack8(rand((M, K), BF16, 1)), sg.pack8(rand((N, K), F32, 2, K**-0.5))
    bias = rand((N,), F32, 3) if (M + N) % 3 else None
    for dtype in (BF16, F32):
        residual = rand((M, N), dtype, 4) if (K + N) % 2 or dtype == F32 else None
        y, ey = forward64(as64(x), as64(w), bias, act, residual, dtype)[2:]
        got, saved = sg.linear(x, w, bias=bias, act=act, residual=residual, dtype=dtype)
        assert saved is None and got.dtype == dtype
        within(got, y, ey)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", list(shapes.FORWARD16))
def test_forward_in_every_tile(M, K, N, act):
    test_forward(M, K, N, act)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", list(shapes.FORWARD8))
def test_forward_from_8_bits_in_every_tile(M, K, N, act):
    test_forward_from_8_bits(M, K, N, act)


def backward64(dy, z, act, x, w):
    """((grad_x, bound), (grad_w, bound before its rounding), (grad_bias, bound)); dz is rounded to bf16."""
    (M, K), N = x.shape, w.shape[0]
    d = act64(z.double(), act)[1] if act else torch.ones_like(dy, dtype=torch.float64)
    dz = dy.double() * d
    # a' in fp32: off by 2^-20 (1 + |z|); the operand's rounding to bf16
    e32 = dy.double().abs() * 2.0**-20 * (1 + z.double().abs()) if act else torch.zeros_like(dz)
    e = e32 + (2.0**-8 * (dz.abs() + e32) if act or dy.dtype == F32 else 0)
    size = dz.abs() + e
    gx = dz @ w, e @ w.abs() + (N + 64) * 2.0**-24 * (size @ w.abs())
    gw = dz.t() @ x, e.t() @ x.abs() + (M + 64) * 2.0**-24 * (size.t() @ x.abs())
    return gx, gw, (dz.sum(0), e32.sum(0) + (M + 64) * 2.0**-24 * size.sum(0))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_backward(M, K, N, act):
    x, w = rand((M, K), BF16, 1), rand((N, K), BF16, 2, K**-0.5)
    z = rand((M, N), BF16, 3, 2.0) if act else None
    for dtype in (BF16, F32):
        dy = rand((M, N), dtype, 4)
        saved = sg.LinearSaved(x, z, act)
        (rx, ex), (rw, ew), (rb, eb) = backward64(dy, z, act, x.double(), w.double())
        gx, gw, gb = sg.linear_backward(dy, saved, w, dtype=dtype)
        assert gx.dtype == BF16 and gw.dtype == dtype and gb.dtype == F32
        within(gx, rx, ex + HALF[BF16] * (rx.abs() + ex) + 1e-38)
        within(gw, rw, ew + HALF[dtype] * (rw.abs() + ew) + 1e-38)
        within(gb, rb, eb + 1e-38)
        for need in range(8):  # each alone and with others: the same bits
            some = sg.linear_backward(dy, saved, w, bool(need & 1), bool(need & 2), bool(need & 4), dtype)
            for i, (a, b) in enumerate(zip(some, (gx, gw, gb))):
                assert torch.equal(a, b) if need >> i & 1 else a is None


@pytest.mark.parametrize("act", [None, "gelu"])
@pytest.mark.parametrize("M,K,N", list(shapes.BACKWARD))
def test_backward_in_every_tile(M, K, N, act):
    test_backward(M, K, N, act)


@pytest.mark.parametrize("act", ACTS)
def test_backward_against_differences(act):
    M, K, N = 70, 96, 130
    x, w, bias = rand((M, K), BF16, 1), rand((N, K), BF16, 2, K**-0.5), rand((N,), F32, 3)
    dy = rand((M, N), BF16, 4)
    grads = sg.linear_backward(dy, sg.linear(x, w, bias=bias, act=act, save="same")[1], w)
    at = [t.double() for t in (x, w, bias)]

    def loss(i, s, v):
        p = [t + s * v if j == i else t for j, t in enumerate(at)]
        return float((act64(p[0] @ p[1].t() + p[2], act)[0] * dy.double()).sum())

    for i, grad in enumerate(grads):
        v = rand(at[i].shape, F32, 20 + i).double()
        along = (loss(i, 1e-5, v) - loss(i, -1e-5, v)) / 2e-5
        terms = grad.double() * v
        # three roundings to bf16 on the way (z, dz, the result), 2^-8 of a term each, signs not aligned
        assert abs(float(terms.sum()) - along) <= 3 * 2.0**-8 * float(terms.abs().sum())


def amid(t, fill=NAN, shift=0):
    """The same numbers with others before and behind every row and below the last; `shift` elements off 16 bytes."""
    wide = torch.full((t.shape[0] + 70, (t.shape[1] + shift + 23) // 8 * 8), fill, dtype=t.dtype, device="cuda")
    wide[: t.shape[0], shift : shift + t.shape[1]] = t
    return wide[: t.shape[0], shift : shift + t.shape[1]]


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("M,K,N", [(1, 8, 1), (40, 72, 99), (70, 72, 104), (70, 2056, 100), (65, 24, 65), (257, 264, 200),
                                   (129, 65, 64), (9, 130, 2056), (300, 1100, 300), (999, 1096, 2730), (1300, 1001, 1500)])
def test_nothing_beside_the_rows_is_read_or_written(M, K, N, shift):
    x, w, bias = rand((M, K), BF16, 1), rand((N, K), BF16, 2, K**-0.5), rand((N,), F32, 3)
    r, z, dy = rand((M, N), BF16, 4), rand((M, N), BF16, 5), rand((M, N), BF16, 6)
    far_x, far_w, far_r, far_dy = (amid(t, shift=shift) for t in (x, w, r, dy))
    out = amid(r, 9.0, shift)
    got, _ = sg.linear(far_x, far_w, bias=bias, act="gelu", residual=far_r, out=out)
    assert got is out and torch.equal(got, sg.linear(x, w, bias=bias, act="gelu", residual=r)[0])
    wide = out._base
    wide[:M, shift : shift + N] = 9
    assert bool((wide == 9).all())
    for act in (None, "silu"):  # dy as its own dz, and not
        want = sg.linear_backward(dy, sg.LinearSaved(x, z, act), w)
        got = sg.linear_backward(far_dy, sg.LinearSaved(far_x, z, act), far_w)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K,N", [(1, 72, 40), (70, 8200, 65), (300, 1100, 301), (2050, 1064, 3000), (3000, 3000, 3001)])
def test_onto_the_residual_in_place(M, K, N, dtype):
    x, w, r = rand((M, K), BF16, 1), rand((N, K), BF16, 2, K**-0.5), rand((M, N), dtype, 3)
    for a, b in ((x, w), (sg.pack8(x), sg.pack8(w))):
        want, there = sg.linear(a, b, residual=r, act="silu", dtype=dtype)[0], r.clone()
        got = sg.linear(a, b, residual=there, act="silu", dtype=dtype, out=there)[0]
        assert got is there and torch.equal(there, want)


@pytest.mark.parametrize("M", [1, 100, 700])
def test_values_that_are_not_numbers_stay_in_their_rows(M):
    K, N = 300, 200
    x, w, dy = rand((M, K), BF16, 1), rand((N, K), BF16, 2), rand((M, N), BF16, 3)
    x[0, 5], dy[0, 7] = NAN, INF
    y = sg.linear(x, w)[0]
    assert bool(torch.isnan(y[0]).all()) and bool(torch.isfinite(y[1:]).all())
    gx, gw, gb = sg.linear_backward(dy, sg.LinearSaved(x), w)
    assert not bool(torch.isfinite(gx[0]).any()) and bool(torch.isfinite(gx[1:]).all())
    assert bool(torch.isnan(gw[:, 5]).all()) and not bool(torch.isfinite(gw[7]).any()) and float(gb[7]) == INF
    fine = torch.ones((N, K), dtype=torch.bool, device="cuda")
    fine[:, 5] = fine[7] = False
    assert bool(torch.isfinite(gw[fine]).all()) and bool(torch.isfinite(gb[torch.arange(N) != 7]).all())


def test_no_rows():
    x, w = torch.empty((0, 40), dtype=BF16, device="cuda"), rand((30, 40), BF16, 2)
    y, saved = sg.linear(x, w, act="silu", save="same")
    assert y.shape == (0, 30)
    for dtype in (BF16, F32):
        gx, gw, gb = sg.linear_backward(y, saved, w, dtype=dtype)
        assert gx.shape == (0, 40) and bool((gw == 0).all()) and bool((gb == 0).all()) and gw.dtype == dtype


def test_many_rows():
    """More than 2^31 elements in y, and a sum of a million rows."""
    M, K, N = 1_050_007, 16, 2_056
    x, w, bias = rand((M, K), BF16, 1), rand((N, K), BF16, 2), rand((N,), F32, 3)
    y, saved = sg.linear(x, w, bias=bias, act="silu", save="same")
    for rows in (slice(0, 300), slice(M - 300, M)):
        ref, bound = forward64(x[rows].double(), w.double(), bias, "silu", None, BF16)[2:]
        within(y[rows], ref, bound)
    gx, gw, gb = sg.linear_backward(y, saved, w)
    last = slice(M - 300, M)
    (rx, ex), _, _ = backward64(y[last], saved.z[last], "silu", x[last].double(), w.double())
    within(gx[last], rx, ex + HALF[BF16] * (rx.abs() + ex) + 1e-38)
    sums = [torch.zeros((N, K), dtype=torch.float64, device="cuda") for _ in range(2)]
    bias64 = [torch.zeros(N, dtype=torch.float64, device="cuda") for _ in range(2)]
    for at in range(0, M, 50_000):
        part = slice(at, min(M, at + 50_000))
        _, rw, rb = backward64(y[part], saved.z[part], "silu", x[part].double(), w.double())
        for total, p in zip(sums, rw):
            total += p
        for total, p in zip(bias64, rb):
            total += p
    # the parts' bounds count a sum of 50,000 rows; of all rows it is 21 times that
    within(gw, sums[0], 21 * sums[1] + HALF[BF16] * (sums[0].abs() + 21 * sums[1]))
    within(gb, bias64[0], 21 * bias64[1])


def chain(x, w, bias, residual, dy):
    h, kept = sg.linear(x, w[0], bias=bias, act="gelu", save="same")
    y, last = sg.linear(h, w[1], residual=residual, save="same")
    gh, gw1, _ = sg.linear_backward(dy, last, w[1], need_bias=False)
    gx, gw0, gb = sg.linear_backward(gh, kept, w[0], dtype=F32)
    return y, gx, gw0, gw1, gb


@pytest.mark.parametrize("M", [1, 50, 700])
def test_a_captured_training_step_replays(M):
    D, F = 256, 1160
    w, bias = [rand((F, D), BF16, 1, 0.06), rand((D, F), BF16, 2, 0.03)], rand((F,), F32, 3)
    x, r, dy = rand((M, D), BF16, 6), rand((M, D), BF16, 7), rand((M, D), BF16, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(x, w, bias, r, dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = chain(x, w, bias, r, dy)
    for seed in range(3):
        x.copy_(rand((M, D), BF16, 30 + seed))
        graph.replay()
        want = chain(x, w, bias, r, dy)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_arguments_by_their_names_and_another_stream():
    x, w, b = rand((80, 64), BF16, 1), rand((16, 64), BF16, 2), rand((16,), F32, 3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def step(**on):
        y, saved = sg.linear(x=x, w=w, bias=b, act="silu", residual=None, save="same", dtype=F32, out=None, **on)
        x8, w8 = sg.pack8(x, **on), sg.pack8(w, **on)
        return (y, sg.linear(x=x8, w=w8, bias=b, **on)[0],
                *sg.linear_backward(grad_y=y, saved=saved, w=w, need_x=True, need_w=True, need_bias=True, dtype=F32, **on))

    here, there = step(), step(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(here, there))
    assert not any(t.requires_grad for t in here)


def test_refusals():
    x, w, b = rand((8, 64), BF16, 1), rand((16, 64), BF16, 2), rand((16,), F32, 3)
    y, saved = sg.linear(x, w, act="silu", save="same")
    x8, w8 = sg.pack8(x), sg.pack8(w)
    plain = sg.LinearSaved(x)
    bad = [
        lambda: sg.linear(x.float(), w), lambda: sg.linear(x, w.float()), lambda: sg.linear(x, w[:, :63]),
        lambda: sg.linear(x.cpu(), w), lambda: sg.linear(x, w.t()), lambda: sg.linear(x[0], w),
        lambda: sg.linear(x, w, bias=b[:15]), lambda: sg.linear(x, w, bias=b.bfloat16()), lambda: sg.linear(x, w, act="relu"),
        lambda: sg.linear(x, w, save="8bit"), lambda: sg.linear(x, w, dtype=torch.float16),
        lambda: sg.linear(x, w, residual=y.float()), lambda: sg.linear(x, w, residual=y[:7]),
        lambda: sg.linear(x, w, out=y[:, :15]), lambda: sg.linear(x, w, out=y, dtype=F32), lambda: sg.linear(x, w[:0]),
        lambda: sg.linear(x[:, :0], w[:, :0]), lambda: sg.linear(x8, w), lambda: sg.linear(x, w8),
        lambda: sg.linear(x8, w8, save="same"), lambda: sg.linear(x8, sg.pack8(w[:, :63])),
        lambda: sg.linear(x8, w8, residual=y.float()), lambda: sg.linear_backward(y, None, w),
        lambda: sg.linear_backward(y[:, :15], plain, w), lambda: sg.linear_backward(y[:7], plain, w),
        lambda: sg.linear_backward(y, sg.LinearSaved(x, None, "silu"), w),
        lambda: sg.linear_backward(y, sg.LinearSaved(x, y.float(), "silu"), w),
        lambda: sg.linear_backward(y, sg.LinearSaved(x, amid(y), "silu"), w),
        lambda: sg.linear_backward(y, sg.LinearSaved(x.float()), w), lambda: sg.linear_backward(y, plain, w[:, :63]),
        lambda: sg.linear_backward(y, saved, w, dtype=torch.float16), lambda: sg.linear_backward(y.half(), plain, w),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
