"""AdamW's 8-bit states where beta1^2 / beta2 is 1 or more, so that m / sqrt(v) of exact sums has no bound that lasts (GPU)."""

import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2607_01408_amd as sg  # noqa: E402
from tests.test_gpu_training import BF16, F32, blocks_of, held, rand  # noqa: E402

BETAS = [(0.95, 0.9), (0.9, 0.81), (0.9, 0.8), (0.99, 0.5)]


@pytest.mark.parametrize("where", ["host", "device"])
@pytest.mark.parametrize("betas,step", [(b, t) for b in BETAS for t in (1, 2, 10, 300) if (b[0] ** 2 / b[1]) ** t < 1e6])
def test_a_v_of_zero_beside_an_m_makes_no_step_past_the_steps_bound(betas, step, where):
    """|m| <= c sqrt(v) for sums of `step` gradients, c^2 = (1 - b1)^2 / (1 - b2) (1 + r + ... + r^(step - 1))."""
    n, (b1, b2) = 256, betas
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m, v = blocks_of(torch.full((n,), 1e-3, device="cuda")), blocks_of(torch.zeros(n, device="cuda"))
    at = step if where == "host" else torch.tensor([step], device="cuda")
    sg.adamw([p], [g], [m], [v], step=at, lr=1e-3, betas=betas, eps=0.0, weight_decay=0.0)
    r = b1 * b1 / b2
    c = (1 - b1) / math.sqrt(1 - b2) * math.sqrt(math.fsum(r**i for i in range(step)))
    want = 1e-3 * c * math.sqrt(1 - b2**step) / (1 - b1**step)
    # some ten roundings in fp32
    assert bool(((p.abs() / want - 1).abs() <= 2.0**-19).all()), float(p.abs().max() / want)


@pytest.mark.parametrize("betas", BETAS)
def test_small_gradients_beside_a_large_one(betas):
    """Roots below the smallest number of their block's format beside m's that are rounded up to theirs: a step without
    gradients stays as short as the two formats allow."""
    n, (b1, b2) = 1 << 16, betas
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 1e-3, device="cuda")
    first = torch.arange(n, device="cuda") % 128 == 0
    g[first] = 1e3
    m, v = sg.adamw_state(p, bits=8)
    sg.adamw([p], [g], [m], [v], step=1, lr=1e-3, betas=betas, weight_decay=0.0)
    some = (held(m) != 0) & ~first
    assert bool((held(v) > 0).all()) and bool(some.any())
    before = p.clone()
    sg.adamw([p], [torch.zeros_like(g)], [m], [v], step=2, lr=1e-3, betas=betas, weight_decay=0.0)
    # the smallest numbers are 2^-9 of a block's scale, less than two parts in 448 of the largest m and at least one of
    # the largest root, which are 1e3 (1 - b1) and 1e3 sqrt(1 - b2)
    most = 1e-3 * 2 * b1 * (1 - b1) / math.sqrt(b2 * (1 - b2)) * math.sqrt(1 - b2 * b2) / (1 - b1 * b1)
    assert bool(((p - before)[~first].abs() <= most * (1 + 2.0**-10)).all()), float((p - before)[~first].abs().max() / most)


@pytest.mark.parametrize("betas", BETAS)
def test_no_v_is_lost_on_the_way(betas):
    n = 4096
    p, m, v = torch.zeros(n, device="cuda"), *sg.adamw_state(torch.zeros(n, device="cuda"), bits=8)
    spread = torch.exp(6 * rand((n,), F32, 1))
    for step in range(1, 30):
        g = rand((n,), F32, 10 + step) * spread * (step < 20)
        sg.adamw([p], [g.to(BF16)], [m], [v], step=step, lr=1e-3, betas=betas, weight_decay=0.0)
        assert bool((held(v) > 0).all()) and bool(torch.isfinite(p).all())


def test_a_mean_that_is_kept_where_the_bound_lasts():
    """Below that the roots go to zero as before: the mean of v over many small ones is kept."""
    n = 1 << 18
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 1e-3, device="cuda")
    first = torch.arange(n, device="cuda") % 128 == 0
    g[first] = 1e3
    m, v = sg.adamw_state(p, bits=8)
    sg.adamw([p], [g], [m], [v], step=1, lr=1e-3, weight_decay=0.0)
    got, want = held(v)[~first].pow(2), 1e-3 * float(g[1]) ** 2
    assert bool((got == 0).any())
    # n choices between zero and the smallest number's square `span`: five standard deviations, each at most sqrt(span want)
    span = float(got.max())
    assert abs(float(got.mean()) - want) <= 5 * math.sqrt(span * want / n) + 2.0**-15 * span
