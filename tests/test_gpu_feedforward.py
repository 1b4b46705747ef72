"""The feed-forward operators against float64 (GPU).

Bounds, from the number formats alone:
  * bf16 rounds to nearest: relative error 2^-9, taken as 2^-8; fp32 2^-24;
  * a sum of K products in fp32 is off by at most K 2^-24 of the sum of their magnitudes;
  * e4m3 rounds to nearest: relative error 2^-4, and 2^-10 of the block's scale below its smallest
    normal number.
"""

import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)

from tests import feedforward_shapes as shapes  # noqa: E402
import paper_2607_01408_amd as sg  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
UNIT = {F32: 2.0**-24, BF16: 2.0**-8}
NAN, INF = float("nan"), float("inf")


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


# ------------------------------------------------------------------ the 8-bit format

def ref_blocks(x):
    """(values [R, Dp] e4m3, scale bytes [R, blocks]) of x, from the format's definition in float64 on the CPU."""
    x = x.double().cpu()
    R, D = x.shape
    nb = -(-D // 128)
    v = torch.zeros((R, nb * 128), dtype=torch.float64)
    v[:, :D] = x
    v = v.view(R, nb, 128)
    top = torch.where(torch.isfinite(v), v.abs(), torch.zeros_like(v)).amax(-1)
    e = torch.zeros_like(top)
    for i in range(R):
        for j in range(nb):
            t = float(top[i, j])
            if t > 0:
                k = math.frexp(t)[1] - 9  # t / 2^k in [256, 512)
                e[i, j] = max(-126, k if t <= 448 * 2.0**k else k + 1)
    t = v / torch.exp2(e)[..., None]
    t = torch.where(torch.isfinite(t), t, torch.full_like(t, NAN))
    return t.float().to(torch.float8_e4m3fn).view(R, -1), (e + 127).to(torch.uint8)


def same_blocks(b, x):
    q, e = ref_blocks(x)
    assert torch.equal(b.values.view(torch.uint8).cpu() & 0x7F, q.view(torch.uint8) & 0x7F)
    a, c = b.values.float().cpu(), q.float()
    fine = ~torch.isnan(c)
    assert torch.equal(torch.isnan(a), ~fine) and torch.equal(a[fine], c[fine])
    assert torch.equal(b.scales.view(torch.uint8).cpu()[:, : e.shape[1]], e)


def special(R, D, dtype, seed):
    """Normal values with blocks of zeros, tiny and huge ones, and non-finite elements."""
    x = rand((R, D), F32, seed)
    x[0, : min(D, 128)] = 0
    x[R // 2] *= 1e-36
    x[R - 1] *= 1e36
    if R > 2:
        x[1, D // 2] = INF
        x[1, D - 1] = NAN
        x[2, 0] = -INF
        x[2, D // 3] = 1.75 * 2.0**9  # the largest with its scale
    return x.to(dtype)


SHAPES = [(1, 1), (3, 7), (5, 128), (4, 129), (7, 500), (130, 260), (257, 640), (2, 4800)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,D", SHAPES)
def test_pack_is_the_format(R, D, dtype):
    x = special(R, D, dtype, 7 * R + D)
    same_blocks(sg.pack8(x), x)
    same_blocks(sg.pack8(x, transpose=True), x.t())
    rows, cols = sg.pack8(x, transpose="both")
    same_blocks(rows, x)
    same_blocks(cols, x.t())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,D", SHAPES)
def test_unpack_is_values_times_scales(R, D, dtype):
    b = sg.pack8(special(R, D, F32, R + D))
    y = sg.unpack8(b, dtype=dtype)
    assert y.dtype == dtype and tuple(y.shape) == (R, D)
    s = torch.exp2(b.scales.view(torch.uint8).double() - 127).repeat_interleave(128, 1)[:, :D]
    ref = (b.values.double()[:, :D] * s).to(dtype)
    ok = torch.isnan(ref)
    assert torch.equal(torch.isnan(y), ok) and torch.equal(y[~ok], ref[~ok])


def test_pack_takes_strided_rows_and_keeps_its_neighbours():
    big = rand((40, 1000), BF16, 3)
    x = big[3:20, 5:302]  # rows at odd element addresses
    same_blocks(sg.pack8(x), x)
    same_blocks(sg.pack8(x, transpose=True), x.t())
    out = torch.full((17, 400), 9.0, dtype=F32, device="cuda")
    sg.unpack8(sg.pack8(x), dtype=F32, out=out[:, 50:347])
    assert bool((out[:, :50] == 9).all()) and bool((out[:, 347:] == 9).all())


def test_past_two_to_the_31_elements():
    R, D = 66_001, 32_800  # 2.16e9 elements
    x = torch.empty((R, D), dtype=BF16, device="cuda")
    x.fill_(0.5)
    tail = rand((3, D), BF16, 11)
    x[-3:] = tail
    b = sg.pack8(x)
    small = sg.Block8(b.values[-3:].contiguous(), b.scales[-3:].contiguous(), (3, D))
    same_blocks(small, tail)
    y = sg.unpack8(b, dtype=BF16)
    assert torch.equal(y[-3:], sg.unpack8(small, dtype=BF16)) and bool((y[: R - 3] == 0.5).all())
    del y, b
    gain = torch.ones(D, device="cuda")
    n, _, rstd = sg.rms_norm(x, gain)
    ref = tail.double() * (tail.double().pow(2).mean(-1, keepdim=True) + 1e-6).rsqrt()
    within(n[-3:], ref, 2.0**-8 * ref.abs() + 1e-6)
    assert abs(float(rstd[R // 2]) - 2) < 1e-4


@pytest.mark.parametrize("M", [1, 40, 100, 300])  # few rows, and the tiles
def test_a_scale_that_is_nan(M):
    K, N = 300, 50
    a, b = sg.pack8(rand((M, K), F32, 1)), sg.pack8(rand((N, K), F32, 2))
    a.scales.view(torch.uint8)[0, 0] = 255
    for dtype in (F32, BF16):
        y = sg.unpack8(a, dtype=dtype)
        assert bool(torch.isnan(y[0, :128]).all()) and int(torch.isnan(y).sum()) == 128
        assert bool(torch.isfinite(y[0, 128:]).all()) and bool(torch.isfinite(y[1:]).all())
        c = sg.matmul8(a, b, dtype=dtype)
        assert bool(torch.isnan(c[0]).all()) and bool(torch.isfinite(c[1:]).all())
    x, w, dh = rand((M, K), BF16, 1), rand((N, K), BF16, 2), rand((M, N), BF16, 3)
    _, saved = sg.gated(x, w, w, save="8bit")
    saved.u.scales.view(torch.uint8)[0, 0] = 255
    dx = sg.gated_backward(dh, saved, w, w)[0]
    assert bool(torch.isnan(dx[0]).all()) and bool(torch.isfinite(dx[1:]).all())


def test_the_smallest_scale():
    a = sg.pack8(rand((5, 300), F32, 1))
    a.scales.view(torch.uint8)[:] = 0
    assert torch.equal(sg.unpack8(a, dtype=F32).double(), a.values.double()[:, :300] * 2.0**-127)


def test_transposed_packing_of_more_rows_than_one_launch():
    R, D = (1 << 27) + 900, 2
    x = rand((R, D), BF16, 1)
    x[-3:] = NAN
    t, want = sg.pack8(x, transpose=True), sg.pack8(x.t().contiguous())
    assert torch.equal(t.values.view(torch.uint8), want.values.view(torch.uint8))
    assert torch.equal(t.scales.view(torch.uint8), want.scales.view(torch.uint8))


# ------------------------------------------------------------------ norm

def ref_norm(x, r, gain, eps):
    h = x.double() if r is None else (x.double() + r.double()).to(x.dtype).double()
    rstd = 1 / torch.sqrt(h.pow(2).mean(-1) + eps)
    return h * rstd[:, None] * gain.double(), h, rstd


NORM_SHAPES = [(1, 1), (3, 5), (2, 128), (33, 100), (300, 128), (5000, 130), (17, 513), (4, 1000), (3000, 1024),
               (2, 2048), (520, 2056), (3, 4096), (600, 7001), (2, 16384), (2, 33000), (300, 33000)]


@pytest.mark.parametrize("out8", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,D", NORM_SHAPES)
def test_norm(R, D, dtype, out8):
    residual = (R + D) % 3 != 0
    x = rand((R, D), dtype, R + D, 3.0)
    r = rand((R, D), dtype, R + D + 1) if residual else None
    gain = 1 + rand((D,), F32, 5, 0.3)
    y, h, rstd = sg.rms_norm(x, gain, residual=r, eps=1e-5, out8=out8)
    ref, rh, rr = ref_norm(x, r, gain, 1e-5)
    assert torch.equal(h.double(), rh)
    # the sum of squares is a sum of D positive terms, in at most D / 4 steps of each lane and the tree
    within(rstd, rr, rr * (D + 64) * 2.0**-24, "rstd")
    slack = (D + 64) * 2.0**-24 + 4 * 2.0**-24
    if out8:
        got = sg.unpack8(y, dtype=F32)
        scale = torch.exp2(y.scales.view(torch.uint8).double() - 127).repeat_interleave(128, 1)[:, :D]
        within(got, ref, ref.abs() * (2.0**-4 + slack) + scale * 2.0**-10, "y8")
        assert bool((y.values.float()[:, D:] == 0).all())
        e = ref_blocks(ref)[1]
        assert float((y.scales.view(torch.uint8).cpu()[:, : e.shape[1]].int() - e.int()).abs().max()) <= 1
    else:
        assert y.dtype == dtype
        within(y, ref, ref.abs() * (UNIT[dtype] + slack) + 1e-38, "y")


@pytest.mark.parametrize("out8", [False, True])
def test_norm_of_zeros_and_non_finite_rows(out8):
    x = rand((4, 300), F32, 1)
    x[0] = 0
    x[1, 7] = INF
    x[2, 9] = NAN
    gain = torch.ones(300, device="cuda")
    y, _, rstd = sg.rms_norm(x, gain, eps=1e-6, out8=out8)
    if out8:
        y = sg.unpack8(y, dtype=F32)
    assert bool((y[0] == 0).all()) and abs(float(rstd[0]) - 1000) < 0.01
    # an infinite element makes its row's rstd 0: zeros, and NaN (inf * 0) in its place
    assert float(rstd[1]) == 0 and bool(torch.isnan(y[1, 7])) and int(torch.isnan(y[1]).sum()) == 1
    assert bool(torch.isnan(y[2]).all())
    ref = ref_norm(x[3:], None, gain, 1e-6)[0]
    within(y[3:], ref, ref.abs() * (2.0**-4 if out8 else 1e-5) + (0.01 if out8 else 0))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [7, 100, 300, 1001, 2050, 33000])
def test_norm_pads_with_zeros_whatever_the_row_holds(D, dtype):
    x = rand((6, D), dtype, D)
    x[1, D // 2], x[2, 0], x[3] = NAN, INF, 0
    for eps in (0.0, 1e-6):
        y, _, _ = sg.rms_norm(x, torch.ones(D, device="cuda"), eps=eps, out8=True)
        assert bool((y.values.float()[:, D:] == 0).all())


def test_norm_takes_strided_rows():
    big = rand((50, 700), BF16, 2)
    x, r = big[1:30, 3:404], big[20:49, 101:502]
    gain = 1 + rand((401,), F32, 5, 0.3)
    y, h, rstd = sg.rms_norm(x, gain, residual=r)
    y2, h2, rstd2 = sg.rms_norm(x.contiguous(), gain, residual=r.contiguous())
    assert torch.equal(y, y2) and torch.equal(h, h2) and torch.equal(rstd, rstd2)
    dx, dg = sg.rms_norm_backward(big[2:31, 7:408], h, rstd, gain, grad_h=r)
    dx2, dg2 = sg.rms_norm_backward(big[2:31, 7:408].contiguous(), h, rstd, gain, grad_h=r.contiguous())
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,D", NORM_SHAPES)
def test_norm_backward(R, D, dtype):
    with_h = (R + D) % 2 == 0
    x, dy = rand((R, D), dtype, R + D, 2.0), rand((R, D), dtype, R + D + 1)
    gain = 1 + rand((D,), F32, 5, 0.3)
    gh = rand((R, D), dtype, 9) if with_h else None
    _, h, rstd = sg.rms_norm(x, gain)
    dx, dgain = sg.rms_norm_backward(dy, h, rstd, gain, grad_h=gh)
    hd, dd, gd = h.double(), dy.double(), gain.double()
    rr = 1 / torch.sqrt(hd.pow(2).mean(-1, keepdim=True) + 1e-6)
    xhat, t = hd * rr, dd * gd
    ref = rr * (t - xhat * (t * xhat).mean(-1, keepdim=True))
    size = rr * (t.abs() + xhat.abs() * (t * xhat).abs().mean(-1, keepdim=True))
    if gh is not None:
        ref = ref + gh.double()
    within(dx, ref, UNIT[dtype] * ref.abs() + (2 * D + 128) * 2.0**-24 * size + 1e-38, "dx")
    # the gain's gradient: R products, each with a factor rstd of relative error (D + 64) 2^-24
    within(dgain, (dd * xhat).sum(0), (R + D + 128) * 2.0**-24 * (dd * xhat).abs().sum(0) + 1e-38, "dgain")
    again = sg.rms_norm_backward(dy, h, rstd, gain, grad_h=gh)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgain)


def test_norm_backward_of_more_columns_than_one_launch_has_threads():
    R, D = 2, (1 << 27) + 100
    h, dy, gain = rand((R, D), BF16, 1), rand((R, D), BF16, 2), torch.ones(D, device="cuda")
    rstd = torch.tensor([0.5, 2.0], device="cuda")
    dx, dgain = sg.rms_norm_backward(dy, h, rstd, gain)
    for at in (slice(0, 300), slice((1 << 25) - 100, (1 << 25) + 100), slice(D - 300, D)):
        terms = dy[:, at].double() * h[:, at].double() * rstd.double()[:, None]
        within(dgain[at], terms.sum(0), 4 * 2.0**-24 * terms.abs().sum(0) + 1e-38)


def test_norm_backward_against_differences():
    R, D = 6, 200
    x, dy, v = (rand((R, D), F32, s) for s in (1, 2, 3))
    gain, w = 1 + rand((D,), F32, 4, 0.3), rand((D,), F32, 5)
    _, h, rstd = sg.rms_norm(x, gain)
    dx, dgain = sg.rms_norm_backward(dy, h, rstd, gain)

    def loss(s, t):
        y, _, _ = ref_norm(x.double() + s * v.double(), None, gain.double() + t * w.double(), 1e-6)
        return float((y * dy.double()).sum())

    e = 1e-5  # central differences in float64: truncation near e^2, cancellation near 1e-16 / e
    along_x, along_g = (loss(e, 0) - loss(-e, 0)) / (2 * e), (loss(0, e) - loss(0, -e)) / (2 * e)
    size = float((dx.double() * v.double()).abs().sum())
    assert abs(float((dx.double() * v.double()).sum()) - along_x) <= 1e-5 * size
    size = float((dgain.double() * w.double()).abs().sum())
    assert abs(float((dgain.double() * w.double()).sum()) - along_g) <= 1e-5 * size


def test_norm_of_no_rows():
    gain = torch.ones(40, device="cuda")
    for out8 in (False, True):
        y, h, rstd = sg.rms_norm(torch.empty((0, 40), device="cuda"), gain, out8=out8)
        assert tuple(y.shape) == (0, 40) and rstd.numel() == 0
    dx, dgain = sg.rms_norm_backward(torch.empty((0, 40), device="cuda"), h, rstd, gain)
    assert tuple(dx.shape) == (0, 40) and bool((dgain == 0).all())


# ------------------------------------------------------------------ 8-bit product

def as64(b):
    return sg.unpack8(b, dtype=F32).double()


def check_product(c, a, b, K):
    ref = a @ b.t()
    size = a.abs() @ b.abs().t()
    within(c, ref, UNIT[c.dtype] * ref.abs() + (K + 64) * 2.0**-24 * size + 1e-38)


MATMULS = [(1, 1, 1), (1, 64, 128), (1, 4096, 512), (2, 17, 130), (5, 300, 1000), (16, 256, 640), (17, 33, 257),
           (31, 1024, 2048), (33, 65, 129), (50, 700, 300), (64, 64, 512), (100, 700, 900), (257, 129, 1030), (777, 1000, 300),
           (1600, 1700, 384), (4100, 3900, 256), (300, 9, 5000), (9, 9, 9000)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,N,K", MATMULS)
def test_matmul8(M, N, K, dtype):
    a = rand((M, K), F32, M + K) * torch.exp2(torch.arange(K, device="cuda") % 23 - 11.0)  # scales that differ
    b = rand((N, K), F32, N + K) * torch.exp2(-(torch.arange(K, device="cuda") // 128 % 5) * 3.0)
    a, b = sg.pack8(a), sg.pack8(b)
    out = torch.full((M, N), NAN, dtype=dtype, device="cuda")
    assert sg.matmul8(a, b, dtype=dtype, out=out) is out
    check_product(out, as64(a), as64(b), K)
    assert torch.equal(sg.matmul8(a, b, dtype=dtype), out)  # the same order of sums in every call


@pytest.mark.parametrize("M,N,K", [(1, 40, 300), (20, 40, 300), (70, 100, 300)])
def test_matmul8_writes_only_its_columns_and_keeps_nan_in_its_row(M, N, K):
    x = rand((M, K), F32, 1)
    x[M - 1, 5] = NAN
    a, b = sg.pack8(x), sg.pack8(rand((N, K), F32, 2))
    big = torch.full((M, N + 9), 7.0, dtype=BF16, device="cuda")
    sg.matmul8(a, b, out=big[:, 4 : 4 + N])
    assert bool((big[:, :4] == 7).all()) and bool((big[:, 4 + N :] == 7).all())
    c = big[:, 4 : 4 + N]
    assert bool(torch.isnan(c[M - 1]).all()) and not bool(torch.isnan(c[: M - 1]).any())
    x[M - 1] = 0
    check_product(sg.matmul8(sg.pack8(x), b), as64(sg.pack8(x)), as64(b), K)


def test_matmul8_result_past_two_to_the_31_elements():
    M, N, K = 66_001, 32_900, 128
    a, b = sg.pack8(rand((M, K), BF16, 1)), sg.pack8(rand((N, K), BF16, 2))
    c = sg.matmul8(a, b)
    rows, cols = slice(M - 70, M), slice(N - 90, N)
    for r, s in ((rows, cols), (rows, slice(0, 50)), (slice(0, 50), cols)):
        check_product(c[r, s], as64(a)[r], as64(b)[s], K)


def test_matmul8_of_few_rows_and_more_columns_than_one_launch():
    M, N, K, cut = 3, (1 << 26) + 1000, 5, 1 << 26
    a, b = sg.pack8(rand((M, K), BF16, 1)), sg.pack8(rand((N, K), BF16, 2))
    c = sg.matmul8(a, b)
    for at in (slice(0, 100), slice(cut - 100, cut + 100), slice(N - 100, N)):
        rows = sg.Block8(b.values[at].contiguous(), b.scales[at].contiguous(), (at.stop - at.start, K))
        check_product(c[:, at], as64(a), as64(rows), K)


@pytest.mark.parametrize("M,N,K", [(3, 50, 70), (200, 130, 300), (1000, 520, 390)])
def test_matmul8_backward(M, N, K):
    x, w, dc = rand((M, K), BF16, 1), rand((N, K), BF16, 2, 0.1), rand((M, N), BF16, 3)
    a_t, b_t = sg.pack8(x, transpose=True), sg.pack8(w, transpose=True)
    da, db = sg.matmul8_backward(dc, a_t, b_t)
    check_product(da, as64(sg.pack8(dc)), as64(b_t), N)
    check_product(db, as64(sg.pack8(dc, transpose=True)), as64(a_t), M)
    # and the gradients of x w^T themselves: each operand of a product is off by 2^-4 of its elements, with signs
    # that do not agree, so the product's norm by less than their sum
    for got, ref in ((da, dc.double() @ w.double()), (db, dc.double().t() @ x.double())):
        assert float((got.double() - ref).norm()) <= 2 * 2.0**-4 * float(ref.norm())


def test_matmul8_of_nothing():
    b = sg.pack8(rand((5, 30), F32, 1))
    none = sg.Block8.empty(0, 30, b.device)
    assert tuple(sg.matmul8(none, b).shape) == (0, 5) and tuple(sg.matmul8(b, none).shape) == (5, 0)


def test_matmul8_backward_of_no_rows():
    x, w = torch.empty((0, 20), dtype=BF16, device="cuda"), rand((30, 20), BF16, 2)
    a_t, b_t = sg.pack8(x, transpose=True), sg.pack8(w, transpose=True)
    assert a_t.shape == (20, 0) and tuple(sg.unpack8(a_t).shape) == (20, 0)
    for dtype in (F32, BF16):
        da, db = sg.matmul8_backward(torch.empty((0, 30), dtype=dtype, device="cuda"), a_t, b_t)
        assert tuple(da.shape) == (0, 20) and da.dtype == dtype
        assert tuple(db.shape) == (30, 20) and db.dtype == dtype and bool((db == 0).all())
    out = torch.full((30, 25), 7.0, device="cuda")
    rows, cols = sg.pack8(torch.empty((0, 30), device="cuda"), transpose="both")
    assert rows.shape == (0, 30) and cols.shape == (30, 0)
    sg.matmul8(cols, a_t, dtype=F32, out=out[:, 2:22])
    assert bool((out[:, 2:22] == 0).all()) and bool((out[:, :2] == 7).all()) and bool((out[:, 22:] == 7).all())
    with pytest.raises(ValueError):
        sg.gated(sg.pack8(x, transpose=True), a_t, a_t)


# ------------------------------------------------------------------ gated block

def act64(g, name):
    if name == "silu":
        t = torch.sigmoid(g)
        return g * t, t * (1 + g * (1 - t))
    p = 0.5 * torch.erfc(-g / math.sqrt(2))
    return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def gated_bound(x, wg, wu, name, K):
    """float64 h, and its bound in fp32: both products' sums, through factors |act'| <= 1.13."""
    g, u = x @ wg.t(), x @ wu.t()
    eg, eu = ((x.abs() @ w.abs().t()) * (K + 64) * 2.0**-24 for w in (wg, wu))
    a, _ = act64(g, name)
    # act itself: exp, a reciprocal and products, 2^-20 of |g|
    bound = 1.13 * (eg * u.abs() + eg * eu) + eu * a.abs() + 2.0**-20 * (g * u).abs()
    return g, u, eg, eu, a * u, bound


GATED = [(1, 1, 1), (1, 64, 128), (1, 2048, 300), (3, 130, 70), (16, 640, 200), (17, 96, 129), (33, 100, 130), (64, 72, 300),
         (65, 257, 64), (300, 72, 500), (999, 200, 273), (513, 1000, 1100), (2050, 64, 3000)]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,K,F", GATED)
def test_gated(M, K, F, act):
    x, wg, wu = rand((M, K), BF16, 1), rand((F, K), BF16, 2, K**-0.5), rand((F, K), BF16, 3, K**-0.5)
    g, u, eg, eu, ref, bound = gated_bound(x.double(), wg.double(), wu.double(), act, K)
    h, saved = sg.gated(x, wg, wu, act=act)
    assert saved is None
    within(h, ref, 2.0**-8 * ref.abs() + bound + 1e-38)
    h1, kept = sg.gated(x, wg, wu, act=act, save="same")
    assert torch.equal(h, h1) and kept.x is x
    within(kept.g, g, 2.0**-8 * g.abs() + eg)
    within(kept.u, u, 2.0**-8 * u.abs() + eu)
    h2, kept = sg.gated(x, wg, wu, act=act, save="8bit")
    assert torch.equal(h, h2)
    same_blocks(kept.x, x)
    for b, r, e in ((kept.g, g, eg), (kept.u, u, eu)):
        scale = torch.exp2(b.scales.view(torch.uint8).double() - 127).repeat_interleave(128, 1)[:, :F]
        within(sg.unpack8(b, dtype=F32), r, (2.0**-4 * r.abs()) + scale * 2.0**-10 + 2 * e)
        assert bool((b.values.float()[:, F:] == 0).all())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,K,F", GATED)
def test_gated_8bit(M, K, F, act):
    x, wg, wu = (sg.pack8(t) for t in (rand((M, K), BF16, 1), rand((F, K), F32, 2, K**-0.5),
                                       rand((F, K), F32, 3, K**-0.5)))
    _, _, _, _, ref, bound = gated_bound(as64(x), as64(wg), as64(wu), act, K)
    h, _ = sg.gated(x, wg, wu, act=act)
    assert h.dtype == BF16
    within(h, ref, 2.0**-8 * ref.abs() + bound + 1e-38)
    b, _ = sg.gated(x, wg, wu, act=act, out8=True)
    scale = torch.exp2(b.scales.view(torch.uint8).double() - 127).repeat_interleave(128, 1)[:, :F]
    within(sg.unpack8(b, dtype=F32), ref, 2.0**-4 * ref.abs() + scale * 2.0**-10 + 2 * bound + 1e-38)
    assert bool((b.values.float()[:, F:] == 0).all())
    top = sg.unpack8(b, dtype=F32).abs()
    top = torch.nn.functional.pad(top, (0, b.values.shape[1] - F)).view(M, -1, 128).amax(-1)
    fits = torch.exp2(b.scales.view(torch.uint8).float() - 127)[:, : top.shape[1]]
    # the smallest power: a block's largest value is above 224 of its scale (or the block is zero)
    assert bool(((top > 223 * fits) | (top == 0)).all()) and bool((top <= 448 * fits).all())


def test_gated_takes_strided_rows():
    big = rand((300, 900), BF16, 1)
    x, wg, wu = big[1:100, 4:204], big[5:255, 12:212], big[40:290, 400:600]
    assert x.data_ptr() % 16 == 0 and wg.data_ptr() % 16 == 0
    h, _ = sg.gated(x, wg, wu)  # rows 1,800 bytes apart: no multiple of 16
    want, saved = sg.gated(x.contiguous(), wg.contiguous(), wu.contiguous(), save="same")
    assert torch.equal(h, want)
    dh = big[100:199, 11:261]
    strided = sg.GatedSaved(x, saved.g, saved.u, "silu", "same")
    for a, b in zip(sg.gated_backward(dh, strided, wg, wu),
                    sg.gated_backward(dh.contiguous(), saved, wg.contiguous(), wu.contiguous())):
        assert torch.equal(a, b)


def test_gated_saturates_and_keeps_nan_in_its_row():
    M, K, F = 40, 64, 100
    x, wg, wu = rand((M, K), BF16, 1, 300.0), rand((F, K), BF16, 2), rand((F, K), BF16, 3)
    for act in ("silu", "gelu"):  # |g| in the thousands: act is 0 or g
        _, _, _, _, ref, bound = gated_bound(x.double(), wg.double(), wu.double(), act, K)
        within(sg.gated(x, wg, wu, act=act)[0], ref, 2.0**-8 * ref.abs() + bound + 1e-30)
    x[3, 5] = NAN
    h, saved = sg.gated(x, wg, wu, save="8bit")
    assert bool(torch.isnan(h[3]).all()) and int(torch.isnan(h).sum()) == F
    g = sg.unpack8(saved.g, dtype=F32)
    assert bool(torch.isnan(g[3]).all()) and int(torch.isnan(g).sum()) == F


def one_column(values, M):
    """x [M, 8] and weights [2, 8] whose g is `values` in turn and whose u is 1."""
    x = torch.zeros((M, 8), dtype=BF16, device="cuda")
    x[:, 0] = torch.tensor(values, device="cuda").repeat(-(-M // len(values)))[:M].to(BF16)
    x[:, 1] = 1
    wg, wu = (torch.zeros((2, 8), dtype=BF16, device="cuda") for _ in range(2))
    wg[:, 0] = 1
    wu[:, 1] = 1
    return x, wg, wu


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M", [30, 90])
def test_gated_at_the_ends_of_the_range(M, act):
    values = [s * v for v in (1e4, 1e15, 2e19, 1e20, 1e30, 2e38, 3.3e38) for s in (1, -1)]
    x, wg, wu = one_column(values, M)
    g = x[:, :1].double()
    # far from zero: act is g or 0, its derivative 1 or 0, and every step of that is exact
    a, da = g.clamp(min=0), (g > 0).double()
    h, saved = sg.gated(x, wg, wu, act=act, save="same")
    assert torch.equal(h.double(), a.expand(M, 2))
    dh = torch.zeros((M, 2), dtype=BF16, device="cuda")
    dh[:, 0] = 1
    dx = sg.gated_backward(dh, saved, wg, wu)[0]
    assert torch.equal(dx[:, 0].double(), da[:, 0]) and torch.equal(dx[:, 1].double(), a[:, 0])


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M", [30, 90])
def test_gated_keeps_an_infinity(M, act):
    x, w, _ = one_column([INF, 2.0, 3e38], M)
    x[:, 1] = 0
    assert bool((sg.gated(2 * x, w, w, act=act)[0][::3] == INF).all())  # act(inf) inf
    assert bool((sg.gated(2 * x, w, w, act=act)[0][2::3] == INF).all())


@pytest.mark.parametrize("M", [30, 90])
def test_gelu_far_below_zero(M):
    values = [-8 + i / 5 for i in range(26)]  # from -8 to -3, where 1 + erf cancels
    x, wg, wu = one_column(values, M)
    g = x[:, 0].double()
    p = 0.5 * torch.special.erfc(-g / math.sqrt(2))
    d = g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    h, saved = sg.gated(x, wg, wu, act="gelu", save="same")
    # the argument z = -g / sqrt 2 is off by 2^-24 z, so erfc by 2 z^2 2^-24 < 2^-18 of itself, and the exponential
    # likewise; 2^-16 with the functions' own few units
    within(h[:, 0], g * p, (2.0**-8 + 2.0**-16) * (g * p).abs())
    dh = torch.zeros((M, 2), dtype=BF16, device="cuda")
    dh[:, 0] = 1
    dx = sg.gated_backward(dh, saved, wg, wu)[0]
    within(dx[:, 0], p + d, 2 * 2.0**-8 * (p + d).abs() + 2.0**-16 * (p + d.abs()))
    within(dx[:, 1], g * p, (2 * 2.0**-8 + 2.0**-16) * (g * p).abs())


def kept64(saved):
    if saved.save == "8bit":
        return as64(saved.x), as64(saved.g), as64(saved.u)
    return saved.x.double(), saved.g.double(), saved.u.double()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("save", ["same", "8bit"])
@pytest.mark.parametrize("M,K,F", GATED)
def test_gated_backward(M, K, F, save, act):
    x, wg, wu = rand((M, K), BF16, 1), rand((F, K), BF16, 2, K**-0.5), rand((F, K), BF16, 3, K**-0.5)
    dh = rand((M, F), BF16, 4)
    _, saved = sg.gated(x, wg, wu, act=act, save=save)
    got = sg.gated_backward(dh, saved, wg, wu)
    xs, g, u = kept64(saved)
    a, da = act64(g, act)
    d = dh.double()
    dg, du = d * u * da, d * a
    # dg and du are rounded to bf16 (2^-9) after an activation off by 2^-20 (1 + |g|)
    eg, eu = dg.abs() * 2.0**-8 + (d * u).abs() * 2.0**-20 * (1 + g.abs()), du.abs() * 2.0**-8 + d.abs() * 2.0**-20 * g.abs()
    wgd, wud = wg.double(), wu.double()
    refs = (dg @ wgd + du @ wud, dg.t() @ xs, du.t() @ xs)
    sums = ((dg.abs() @ wgd.abs() + du.abs() @ wud.abs(), eg @ wgd.abs() + eu @ wud.abs(), 2 * F),
            (dg.abs().t() @ xs.abs(), eg.t() @ xs.abs(), M), (du.abs().t() @ xs.abs(), eu.t() @ xs.abs(), M))
    for y, ref, (size, err, n) in zip(got, refs, sums):
        assert y.dtype == BF16
        within(y, ref, 2.0**-8 * ref.abs() + (n + 128) * 2.0**-24 * size + err + 1e-38)
    # either alone gives the same
    dx, none_g, none_u = sg.gated_backward(dh, saved, wg, wu, need_w=False)
    assert torch.equal(dx, got[0]) and none_g is None and none_u is None
    none_x, dwg, dwu = sg.gated_backward(dh, saved, wg, wu, need_x=False)
    assert none_x is None and torch.equal(dwg, got[1]) and torch.equal(dwu, got[2])


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_backward_against_differences(act):
    M, K, F = 70, 96, 130
    x, wg, wu = rand((M, K), BF16, 1), rand((F, K), BF16, 2, K**-0.5), rand((F, K), BF16, 3, K**-0.5)
    dh = rand((M, F), BF16, 4)
    _, saved = sg.gated(x, wg, wu, act=act, save="same")
    grads = sg.gated_backward(dh, saved, wg, wu)
    at = [t.double() for t in (x, wg, wu)]

    def loss(i, s, v):
        p = [t + s * v if j == i else t for j, t in enumerate(at)]
        return float((act64(p[0] @ p[1].t(), act)[0] * (p[0] @ p[2].t()) * dh.double()).sum())

    for i, grad in enumerate(grads):
        v = rand(at[i].shape, F32, 20 + i).double()
        e = 1e-5
        along = (loss(i, e, v) - loss(i, -e, v)) / (2 * e)
        terms = grad.double() * v
        # four roundings to bf16 on the way (g, u, dg or du, the result), each 2^-9 of a term, signs not aligned:
        # the sum is off by less than 4 2^-9 of the terms' sum of magnitudes
        assert abs(float(terms.sum()) - along) <= 4 * 2.0**-9 * float(terms.abs().sum())


@pytest.mark.parametrize("M, K, F", [(70, 72, 100), (65, 24, 65), (257, 264, 200), (1, 8, 1), (129, 65, 64)])
def test_gated_backward_reads_nothing_beside_its_rows(M, K, F):
    def amid(t):  # the same numbers with NaN behind every row and below the last
        wide = torch.full((t.shape[0] + 70, (t.shape[1] + 23) // 8 * 8), NAN, dtype=BF16, device="cuda")
        wide[: t.shape[0], : t.shape[1]] = t
        return wide[: t.shape[0], : t.shape[1]]

    x, wg, wu = rand((M, K), BF16, 1), rand((F, K), BF16, 2, K**-0.5), rand((F, K), BF16, 3, K**-0.5)
    dh = rand((M, F), BF16, 4)
    want = sg.gated_backward(dh, sg.gated(x, wg, wu, save="same")[1], wg, wu)
    far = [amid(t) for t in (x, wg, wu)]
    got = sg.gated_backward(amid(dh), sg.gated(*far, save="same")[1], far[1], far[2])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_gated_backward_past_two_to_the_31_elements():
    M, K, F, n = 70_001, 64, 16_384, 100  # dg and du together 2.3 10^9 elements; only the last rows have a gradient
    x, wg, wu = rand((M, K), BF16, 1), rand((F, K), BF16, 2, K**-0.5), rand((F, K), BF16, 3, K**-0.5)
    g, u = torch.ones((M, F), dtype=BF16, device="cuda"), torch.ones((M, F), dtype=BF16, device="cuda")
    dh = torch.zeros((M, F), dtype=BF16, device="cuda")
    g[-n:], u[-n:], dh[-n:] = rand((n, F), BF16, 4), rand((n, F), BF16, 5), rand((n, F), BF16, 6)
    dx, dwg, dwu = sg.gated_backward(dh, sg.GatedSaved(x, g, u, "silu", "same"), wg, wu)
    assert bool((dx[:-n] == 0).all())
    a, da = act64(g[-n:].double(), "silu")
    d, u64, xs = dh[-n:].double(), u[-n:].double(), x[-n:].double()
    dg, du = d * u64 * da, d * a
    # as in test_gated_backward: dg and du rounded to bf16, sums in fp32, the result rounded
    eg = dg.abs() * 2.0**-8 + (d * u64).abs() * 2.0**-20 * (1 + g[-n:].double().abs())
    eu = du.abs() * 2.0**-8 + d.abs() * 2.0**-20 * g[-n:].double().abs()
    for y, ref, size, err, terms in (
            (dx[-n:], dg @ wg.double() + du @ wu.double(), dg.abs() @ wg.double().abs() + du.abs() @ wu.double().abs(),
             eg @ wg.double().abs() + eu @ wu.double().abs(), 2 * F),
            (dwg, dg.t() @ xs, dg.abs().t() @ xs.abs(), eg.t() @ xs.abs(), M),
            (dwu, du.t() @ xs, du.abs().t() @ xs.abs(), eu.t() @ xs.abs(), M)):
        within(y, ref, 2.0**-8 * ref.abs() + (terms + 128) * 2.0**-24 * size + err + 1e-38)


def test_gated_of_no_rows():
    wg, wu = rand((30, 20), BF16, 1), rand((30, 20), BF16, 2)
    for save in ("same", "8bit"):
        h, saved = sg.gated(torch.empty((0, 20), dtype=BF16, device="cuda"), wg, wu, save=save)
        dx, dwg, dwu = sg.gated_backward(h, saved, wg, wu)
        assert tuple(h.shape) == (0, 30) and tuple(dx.shape) == (0, 20)
        assert tuple(dwg.shape) == (30, 20) and bool((dwg == 0).all()) and bool((dwu == 0).all())


def test_gated_of_no_rows_and_more_weights_than_one_launch_has_threads():
    F, K = 70_001, 32_768
    w = torch.empty((F, K), dtype=BF16, device="cuda")
    junk = torch.ones((2 * F, K), dtype=BF16, device="cuda")  # the gradients' memory, most likely
    del junk
    g = torch.empty((0, F), dtype=BF16, device="cuda")
    saved = sg.GatedSaved(torch.empty((0, K), dtype=BF16, device="cuda"), g, g, "silu", "same")
    _, dwg, dwu = sg.gated_backward(g, saved, w, w)
    assert not bool(dwg.any()) and not bool(dwu.any())


def test_gated_copies_more_rows_than_one_launch_has_threads():
    M, K, F = (1 << 29) + 1001, 3, 2  # rows of six bytes: copied into rows of 128, 69 GB
    torch.cuda.empty_cache()
    x, wg, wu = torch.zeros((M, K), dtype=BF16, device="cuda"), rand((F, K), BF16, 2), rand((F, K), BF16, 3)
    x[:500], x[-500:] = rand((500, K), BF16, 4), rand((500, K), BF16, 5)
    h = sg.gated(x, wg, wu)[0]
    for at in (slice(0, 600), slice(M - 600, M)):
        _, _, _, _, ref, bound = gated_bound(x[at].double(), wg.double(), wu.double(), "silu", K)
        within(h[at], ref, 2.0**-8 * ref.abs() + bound + 1e-38)
    del x, h
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ every tile, with its whole loop

@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,K,F", list(shapes.GATED))
def test_gated_in_every_tile(M, K, F, act):
    test_gated(M, K, F, act)
    test_gated_8bit(M, K, F, act)


@pytest.mark.parametrize("save", ["same", "8bit"])
@pytest.mark.parametrize("M,K,F", list(shapes.BACKWARD))
def test_gated_backward_in_every_tile(M, K, F, save):
    test_gated_backward(M, K, F, save, "silu")


@pytest.mark.parametrize("M,K,F", list(shapes.BACKWARD_LONG))
def test_gated_backward_past_two_to_the_31_elements_in_the_large_tile(M, K, F):
    n = 200  # the last rows alone have a gradient
    x, wg, wu = rand((M, K), BF16, 1), rand((F, K), BF16, 2, K**-0.5), rand((F, K), BF16, 3, K**-0.5)
    g, u = torch.ones((M, F), dtype=BF16, device="cuda"), torch.ones((M, F), dtype=BF16, device="cuda")
    dh = torch.zeros((M, F), dtype=BF16, device="cuda")
    g[-n:], u[-n:], dh[-n:] = rand((n, F), BF16, 4), rand((n, F), BF16, 5), rand((n, F), BF16, 6)
    dx, dwg, dwu = sg.gated_backward(dh, sg.GatedSaved(x, g, u, "silu", "same"), wg, wu)
    assert not bool(dx[:-n].any())
    a, da = act64(g[-n:].double(), "silu")
    d, u64, xs, wgd, wud = dh[-n:].double(), u[-n:].double(), x[-n:].double(), wg.double(), wu.double()
    dg, du = d * u64 * da, d * a
    # as in test_gated_backward: dg and du rounded to bf16, sums in fp32, the result rounded
    eg = dg.abs() * 2.0**-8 + (d * u64).abs() * 2.0**-20 * (1 + g[-n:].double().abs())
    eu = du.abs() * 2.0**-8 + d.abs() * 2.0**-20 * g[-n:].double().abs()
    for y, ref, size, err, terms in (
            (dx[-n:], dg @ wgd + du @ wud, dg.abs() @ wgd.abs() + du.abs() @ wud.abs(), eg @ wgd.abs() + eu @ wud.abs(), 2 * F),
            (dwg, dg.t() @ xs, dg.abs().t() @ xs.abs(), eg.t() @ xs.abs(), M),
            (dwu, du.t() @ xs, du.abs().t() @ xs.abs(), eu.t() @ xs.abs(), M)):
        within(y, ref, 2.0**-8 * ref.abs() + (terms + 128) * 2.0**-24 * size + err + 1e-38)


@pytest.mark.parametrize("M,K,F", [*shapes.GATED, *shapes.BACKWARD])
def test_every_tile_reads_nothing_beside_its_rows(M, K, F):
    test_gated_backward_reads_nothing_beside_its_rows(M, K, F)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,N,K", list(shapes.PRODUCT8))
def test_matmul8_in_every_tile(M, N, K, dtype):
    test_matmul8(M, N, K, dtype)


# ------------------------------------------------------------------ as programs call them

def serve(x, residual, gain, w):
    y, h, _ = sg.rms_norm(x, gain, residual=residual, out8=True)
    a, _ = sg.gated(y, w[0], w[1], out8=True)
    return sg.matmul8(a, w[2]), h


@pytest.mark.parametrize("M", [1, 50])
def test_a_captured_chain_replays(M):
    D, F = 256, 384
    w = [sg.pack8(rand(s, F32, i, 0.06)) for i, s in enumerate([(F, D), (F, D), (D, F)])]
    gain = 1 + rand((D,), F32, 5, 0.3)
    x, r = rand((M, D), BF16, 6), rand((M, D), BF16, 7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        serve(x, r, gain, w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c, h = serve(x, r, gain, w)
    for seed in range(3):
        x.copy_(rand((M, D), BF16, 30 + seed))
        graph.replay()
        want, wh = serve(x, r, gain, w)
        torch.cuda.synchronize()
        assert torch.equal(c, want) and torch.equal(h, wh)


def test_arguments_by_their_names():
    x, w, gain = rand((8, 64), BF16, 1), rand((16, 64), BF16, 2), torch.ones(64, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def step(**on):
        b = sg.pack8(x=x, transpose=False, **on)
        y, h, rstd = sg.rms_norm(x=x, gain=gain, residual=x, eps=1e-6, out8=False, **on)
        c = sg.matmul8(a=b, b=b, dtype=F32, out=None, **on)
        a, saved = sg.gated(x=x, w_gate=w, w_up=w, act="gelu", save="same", out8=False, **on)
        return (sg.unpack8(b=b, dtype=F32, out=None, **on), y, c, a,
                *sg.rms_norm_backward(grad_y=y, h=h, rstd=rstd, gain=gain, grad_h=y, need_gain=True, **on),
                *sg.matmul8_backward(grad_out=c, a_t=sg.pack8(x=x, transpose=True, **on),
                                     b_t=sg.pack8(x=x, transpose=True, **on), **on),
                *sg.gated_backward(grad_h=a, saved=saved, w_gate=w, w_up=w, need_x=True, need_w=True, **on))

    here, there = step(), step(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(here, there))
    with pytest.raises(TypeError):
        sg.pack8()
    with pytest.raises(TypeError):
        sg.gated(w_gate=w, w_up=w, stream=side)


def test_another_stream():
    x, wg, wu = rand((300, 200), BF16, 1), rand((260, 200), BF16, 2, 0.1), rand((260, 200), BF16, 3, 0.1)
    dh, gain = rand((300, 260), BF16, 4), torch.ones(200, device="cuda")

    def step(**on):
        y, _, _ = sg.rms_norm(x, gain, **on)
        h, saved = sg.gated(y, wg, wu, save="8bit", **on)
        return (h, *sg.gated_backward(dh, saved, wg, wu, **on), sg.matmul8(saved.x, saved.x, **on))

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = step(stream=side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_refusals():
    x, w = rand((8, 64), BF16, 1), rand((16, 64), BF16, 2)
    gain = torch.ones(64, device="cuda")
    b = sg.pack8(x)
    y, h, rstd = sg.rms_norm(x, gain)
    _, saved = sg.gated(x, w, w, save="same")
    bad = [
        lambda: sg.pack8(x.half()), lambda: sg.pack8(x[0]), lambda: sg.pack8(x.cpu()), lambda: sg.pack8(x.t()),
        lambda: sg.pack8(x, transpose="rows"), lambda: sg.pack8(x[:, :0]), lambda: sg.unpack8(x),
        lambda: sg.unpack8(b, dtype=torch.float16), lambda: sg.unpack8(b, out=torch.empty(8, 63, device="cuda")),
        lambda: sg.Block8(b.values, b.scales, (8, 200)), lambda: sg.Block8(b.values.float(), b.scales, (8, 64)),
        lambda: sg.Block8(b.values, b.scales.view(torch.uint8), (8, 64)), lambda: sg.Block8(b.values, b.scales, (7, 64)),
        lambda: sg.rms_norm(x, gain[:63]), lambda: sg.rms_norm(x, gain.bfloat16()), lambda: sg.rms_norm(x, gain, eps=-1),
        lambda: sg.rms_norm(x, gain, residual=x[:7]), lambda: sg.rms_norm(x, gain, residual=x.float()),
        lambda: sg.rms_norm_backward(y, h.float(), rstd, gain), lambda: sg.rms_norm_backward(y, h, rstd[:7], gain),
        lambda: sg.rms_norm_backward(y, h, rstd, gain, grad_h=x[:, :63]),
        lambda: sg.matmul8(b, x), lambda: sg.matmul8(b, sg.pack8(x[:, :63])), lambda: sg.matmul8(b, b, dtype=torch.float16),
        lambda: sg.matmul8(b, b, out=torch.empty(8, 9, dtype=BF16, device="cuda")),
        lambda: sg.matmul8_backward(x, b, b), lambda: sg.gated(x, w, w, act="relu"), lambda: sg.gated(x, w, w, save="fp8"),
        lambda: sg.gated(x, w, w[:15]), lambda: sg.gated(x, w[:, :63], w[:, :63]), lambda: sg.gated(x.float(), w, w),
        lambda: sg.gated(x, w, w, out8=True), lambda: sg.gated(b, b, b, save="8bit"), lambda: sg.gated(b, w, w),
        lambda: sg.gated(x, w, rand((16, 70), BF16, 1)[:, :64]), lambda: sg.gated_backward(x, None, w, w),
        lambda: sg.gated_backward(x, saved, w, w), lambda: sg.gated_backward(saved.g.float(), saved, w, w),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
    with pytest.raises(sg.SpinGTPError):  # rows that start at an odd address
        sg.gated(rand((8, 66), BF16, 1)[:, 1:65], w, w)


def test_saved_blocks_of_another_width_are_refused():
    x, w, dh = rand((70, 100), BF16, 1), rand((40, 100), BF16, 2), rand((70, 40), BF16, 3)
    _, saved = sg.gated(x, w, w, save="8bit")
    wide = rand((40, 120), BF16, 4)  # the same padded width
    with pytest.raises(ValueError):
        sg.gated_backward(dh, saved, wide, wide)
    w50, dh50 = rand((50, 100), BF16, 2), rand((70, 50), BF16, 3)
    with pytest.raises(ValueError):
        sg.gated_backward(dh50, saved, w50, w50)
