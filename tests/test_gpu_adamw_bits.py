"""AdamW's weights and states against their definition in separate fp32 operations of the same device, bit by bit (GPU).

The operations and their order: m = b1 m + c1 x, v = b2 v + c2 (x x), x = g factor; with 8-bit states v is then (m / c)^2
where that is more; p = p decay - rate (m / (sqrt(v) root + eps)).  A state's magnitude t in its block's unit goes to the upper
of its neighbours lo and hi where share (hi - lo) < t - lo, of v's root where share ((hi - lo) (hi + lo)) < v - lo lo."""

import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2607_01408_amd as sg  # noqa: E402
from tests.test_gpu_training import BF16, F32, SIZES, blocks_of, rand, words  # noqa: E402


def f32(x):
    return torch.tensor(x, dtype=F32, device="cuda")


def numbers(step, lr, betas, eps, weight_decay):
    """The options as fp32 numbers."""
    b1, b2 = betas
    r = b1 * b1 / b2
    if 1 - r > 2.0**-20:
        least = math.sqrt((1 - b2) * (1 - r)) / (1 - b1)
    else:
        log_r = 2 * math.log(b1) - math.log(b2)
        total = step if log_r == 0 else math.expm1(step * log_r) / math.expm1(log_r)
        least = math.sqrt(-math.expm1(math.log(b2)) / total) / -math.expm1(math.log(b1))
    log_b1 = math.log(b1) if b1 > 0 else -math.inf
    return dict(b1=f32(b1), c1=f32(1 - b1), b2=f32(b2), c2=f32(1 - b2), eps=f32(eps), least=f32(least), lasting=1 - r > 2.0**-20,
                decay=f32(1 - lr * weight_decay), rate=f32(lr / -math.expm1(step * log_b1)),
                root=f32(1 / math.sqrt(-math.expm1(step * math.log(b2)))))


def step32(p, g, m, v, o, factor, eight):
    x = g.float() if factor is None else g.float() * factor
    m = o["b1"] * m + o["c1"] * x
    v = o["b2"] * v + o["c2"] * (x * x)
    if eight:
        y = m * o["least"]
        v = torch.where(y * y > v, y * y, v)
    p = p.float() * o["decay"] - o["rate"] * (m / (torch.sqrt(v) * o["root"] + o["eps"]))
    return p, m, v


def unpacked(b):
    power = (b.scales.view(torch.uint8).to(torch.int32) << 23).view(F32).repeat_interleave(128, 1)
    return (b.values.float() * power[:, : b.values.shape[1]])[0, : b.shape[1]]


def put(x, root, share, none_to_zero):
    """The bytes of the values and scales of m (or, with `root`, of v by its root)."""
    n = x.numel()
    x = torch.nn.functional.pad(x, (0, -n % 128)).view(-1, 128)
    share = torch.nn.functional.pad(share, (0, -n % 128)).view(-1, 128)
    t = torch.sqrt(x) if root else x.abs()
    mantissa, e = torch.frexp(t.amax(-1))
    e = torch.where(t.amax(-1) > 0, e - 9 + (mantissa > 0.875).int(), torch.zeros_like(e)).clamp(-126, 127)
    inv = ((127 - e).to(torch.int32) << 23).view(F32)[:, None]
    t = t * inv
    base = torch.where(t < 2.0**-6, 2.0**-6, 0.0).float()
    bits = (t + base).view(torch.int32) & ~0xFFFFF
    lo, hi = bits.view(F32) - base, (bits + 0x100000).view(F32) - base
    if root:
        up = share * ((hi - lo) * (hi + lo)) < x * inv * inv - lo * lo
        if none_to_zero:
            up = up | ((lo == 0) & (x > 0))
    else:
        up = share * (hi - lo) < t - lo
    y = torch.where(up, hi, lo).clamp(max=448)
    y = y if root else torch.copysign(y, x)
    return y.to(torch.float8_e4m3fn).view(torch.uint8).view(-1), (e + 127).to(torch.uint8)


@pytest.mark.parametrize("betas", [(0.9, 0.999), (0.95, 0.9), (0.9, 0.81), (0.0, 0.95)])
@pytest.mark.parametrize("gtype", [F32, BF16])
@pytest.mark.parametrize("ptype", [F32, BF16])
@pytest.mark.parametrize("bits", [32, 8])
def test_every_bit(bits, ptype, gtype, betas):
    p, g = ([rand((n,), t, 10 * i + k, s) for i, n in enumerate(SIZES)] for k, t, s in ((1, ptype, 1.0), (2, gtype, 0.1)))
    spread = [torch.exp(2 * rand((n,), F32, 7 + i)) for i, n in enumerate(SIZES)]
    m = [rand((n,), F32, 10 * i + 3, 0.02) * s for (i, n), s in zip(enumerate(SIZES), spread)]
    v = [(rand((n,), F32, 10 * i + 4, 0.05) * s).abs() for (i, n), s in zip(enumerate(SIZES), spread)]
    m, v = ([blocks_of(t) for t in x] if bits == 8 else x for x in (m, v))
    factor = torch.tensor([0.37], device="cuda")
    for step, seed, scale in ((1, 0, None), (7, 5, factor), (1000, 0x123456789ABCDEF, factor)):
        options = dict(step=step, lr=1e-2, betas=betas, eps=1e-8, weight_decay=0.1)
        o = numbers(**options)
        old = [(a.clone(), b, *((unpacked(c), unpacked(d).square()) if bits == 8 else (c.clone(), d.clone())))
               for a, b, c, d in zip(p, g, m, v)]
        sg.adamw(p, g, m, v, seed=seed, grad_scale=scale, **options)
        for k, (a, c, d, before) in enumerate(zip(p, m, v, old)):
            p1, m1, v1 = step32(*before, o, scale, bits == 8)
            assert torch.equal(a, p1.to(ptype)), (k, step)
            if bits == 32:
                assert torch.equal(c, m1) and torch.equal(d, v1), (k, step)
                continue
            w = words(torch.arange(a.numel(), device="cuda"), k, step, seed)
            for got, x, r, root in ((c, m1, w & 0xFFFF, False), (d, v1, w >> 16, True)):
                values, scales = put(x, root, (r.float() + 0.5) * 2.0**-16, not o["lasting"])
                n = a.numel()
                assert torch.equal(got.values.view(torch.uint8)[0, :n], values[:n]), (k, step, root)
                assert torch.equal(got.scales.view(torch.uint8)[0, : len(scales)], scales), (k, step, root)


@pytest.mark.parametrize("copies", [False, True])
def test_more_tensors_than_a_launch_holds(copies):
    """Three launches' worth of fp32 tensors as each of them alone: a launch holds 99 of them, 82 with copies."""
    count = 3 * 99 + 5
    sizes = [1 + 37 * i % 2500 for i in range(count)]
    made = [[rand((n,), F32, 9 * i + k, 0.1) for i, n in enumerate(sizes)] for k in range(4)]
    made[3] = [t.abs() for t in made[3]]
    alone = [[t.clone() for t in x] for x in made]
    out, one = ([torch.zeros(n, dtype=BF16, device="cuda") if copies and i % 3 else None for i, n in enumerate(sizes)]
                for _ in range(2))
    on = dict(step=4, lr=1e-2, weight_decay=0.1)
    sg.adamw(*made, copies=out if copies else None, **on)
    for i in range(count):
        sg.adamw(*([x[i]] for x in alone), copies=[one[i]] if copies else None, **on)
    for x, y in zip(made, alone):
        assert all(torch.equal(s, t) for s, t in zip(x, y))
    assert all((s is None and t is None) or torch.equal(s, t) for s, t in zip(out, one))
