"""The distillation's gradient where 1 / temperature times a logit is large, in rows that hold NaN, and in rows past 2^31
elements (64-bit reference and bounds of tests/_lm_ref.py)."""

import math

import pytest
import torch

from tests import _lm_ref as R
from tests.test_distill_gpu import DEV, TYPES, base, gen, lib, run  # noqa: F401


pytestmark = pytest.mark.gpu

BOTH = [(0.0, True), (0.4, True), (1.0, True), (0.0, False), (1.0, False)]
# a row in one workgroup's registers, in a wave's, read again, in parts
SIZES = [("f32", 9, 700), ("f32", 650, 700), ("f32", 4, 50_001), ("f32", 130, 110_001), ("f32", 2, 200_002)]


def f32(v):
    return torch.tensor(v, dtype=torch.float32).double().item()


def reference(z, ids, tau, w, b, rest, temp, scale):
    """R.distill, with the gradients outside of the list also where their probabilities are below float64: a word's share of
    the rest times what the teacher leaves it."""
    b, temp, scale = f32(b), f32(temp), f32(scale)
    want = R.distill(z, ids, tau, w, b, rest, temp, scale)
    if rest:
        x = z.double() / temp
        real = (ids >= 0) & (tau > -math.inf)
        inside = torch.zeros((z.shape[0], z.shape[1] + 1), dtype=torch.bool).scatter_(1, torch.where(real, ids.long(), z.shape[1]), True)[:, :-1]
        below = torch.where(inside, -math.inf, x)
        below = below - below.amax(dim=1, keepdim=True)
        log_s = below.logsumexp(dim=1, keepdim=True)
        tr = (1 - torch.where(real, tau.double().exp(), 0.0).sum(dim=1, keepdim=True)).clamp(min=2.0 ** -24)
        k = (w.double() * scale / temp)[:, None]
        grad = -(1 - b) * tr * (below - log_s).exp() * k
        # an exponential is off by 4 roundings of its exponent, the sum by one for each of a thread's elements and the joins
        err = R.EPS24 * (z.shape[1] / 256 + 60 + 4 * torch.where(below > -math.inf, below, 0.0).abs() + 4 * log_s.abs())
        lost = ~inside & (x - x.logsumexp(dim=1, keepdim=True) < -650)
        want["dlogits"] = torch.where(lost, grad, want["dlogits"])
        want["grad_bound"] = torch.where(lost, grad.abs() * err, want["grad_bound"])
    return want


def held(lib, z, ids, tau, w, b, rest, temp, scale):
    grad = torch.full(z.shape, 9.0, dtype=z.dtype, device=DEV)
    _, losses = run(lib, z.to(DEV), ids, tau, w, b, rest, temp, scale, grad)
    want = reference(z, ids, tau, w, b, rest, temp, scale)
    R.near(losses, want["losses"], want["loss_bound"], torch.float32, "losses")
    R.near(grad, want["dlogits"], want["grad_bound"], z.dtype, "gradient")
    return want["dlogits"]


# at 2^-19 log2 e, words of 8 and above are past the products that are taken whole, those below it are not
@pytest.mark.parametrize("temp", [1e-6, 1.4426950408889634 * 2.0 ** -19])
@pytest.mark.parametrize("t,T,V", SIZES)
def test_logits_that_differ_by_a_few_steps(lib, t, T, V, temp):
    """Float32 words near 8, a few of their steps apart, so that exponents are finite and of every size."""
    K, n = 12, min(T, 6)
    z = torch.rand((n, V), generator=gen(1)) * 7
    ids, tau = torch.empty((n, K), dtype=torch.int32), torch.empty((n, K))
    for r in range(n):
        near = torch.randperm(V, generator=gen(r))[:40]
        steps = torch.randint(-6, 7, (40,), generator=gen(50 + r))
        if r == 1:
            steps[:K] += 30  # the list far above the rest
        if r == 2:
            steps[K:] += 30  # and far below
        z[r, near] = (8.0 + steps.double() * 2.0 ** -20).float()
        ids[r] = near[:K].int()
        tau[r] = (torch.log_softmax(torch.randn(K, generator=gen(90 + r)), 0) - 0.2).float()
    reps = -(-T // n)
    z, ids, tau = (v.repeat(reps, 1)[:T] for v in (z, ids, tau))
    w = torch.full((T,), 1.0 / T)
    for b, rest in BOTH[:2] if T > 100 else BOTH:
        want = held(lib, z, ids, tau, w, b, rest, temp, temp)
        near = torch.ones_like(z, dtype=torch.bool).scatter_(1, ids.long(), False) & (z > 7.5)
        assert (want[near].abs() * T > 1e-4).float().mean() > 0.25  # the words outside of the list have gradients to compare


@pytest.mark.parametrize("T,V", [(9, 40), (4, 50_000), (2, 150_001), (161, 180_000)])
@pytest.mark.parametrize("temp", [1e-20, 1e-6])
def test_equal_logits_near_temperature_0(lib, T, V, temp):
    """bf16 words that share the largest logit share the probability, in the list and outside of it."""
    K, n = 6, min(T, 5)
    z = torch.randn((n, V), generator=gen(3)).clamp(max=7.0).to(torch.bfloat16)
    ids = torch.stack([torch.randperm(V, generator=gen(r)) for r in range(n)])
    for r in range(n):
        first = (0, K, 0, 3, 5)[r]  # in the list and outside, outside alone, all of the list
        z[r, ids[r, first:first + (9, 4, K, 9, 3)[r]]] = 8.0
    ids = ids[:, :K].int()
    tau = (torch.log_softmax(torch.randn((n, K), generator=gen(4)), 1) - 0.3).float()
    reps = -(-T // n)
    z, ids, tau = (v.repeat(reps, 1)[:T] for v in (z, ids, tau))
    for b, rest in BOTH[:1] if T > 100 else BOTH:
        held(lib, z, ids, tau, torch.full((T,), 1.0 / T), b, rest, temp, temp)


@pytest.mark.parametrize("T,V", [(5, 900), (4, 40_000), (650, 700)])
@pytest.mark.parametrize("temp", [1e-37, 1e-20, 1e-6, 1e-3])
def test_gradient_near_temperature_0(lib, T, V, temp):
    z, ids, tau, w = base(T, V, 9)
    z[0] = -3.3e38
    z[1, : V // 2] = -3.3e38
    scale = max(temp, 1e-30)  # times a row's weight a number with all its digits
    for b, rest in BOTH:
        grad = torch.full((T, V), 9.0, device=DEV)
        run(lib, z.to(DEV), ids, tau, w, b, rest, temp, scale, grad)
        want = reference(z, ids, tau, w, b, rest, temp, scale)
        R.near(grad, want["dlogits"], want["grad_bound"], torch.float32, "gradient")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(9, 700), (9, 40_000), (170, 20_000), (700, 700), (640, 5000), (130, 200_000), (3, 140_000)])
def test_rows_that_hold_nan(lib, T, V, t):
    """NaN or +inf, listed or not, makes every gradient and loss of its own row NaN and of no other row."""
    z, ids, tau, w = base(T, V, 9, dtype=TYPES[t])
    quiet = z.clone()
    out = torch.ones(V, dtype=torch.bool)
    out[ids[0].long()] = False
    z[0, int(out.nonzero()[5])] = math.nan
    z[1, ids[1, 4].long()] = math.nan
    out = torch.ones(V, dtype=torch.bool)
    out[ids[2].long()] = False
    bad, inf = {0, 1, 2}, 2
    z[2, int(out.nonzero()[-1])] = math.inf
    if T > 5:
        z[4, ids[4, 0].long()] = math.inf
        tau[5, 3] = math.nan
        bad |= {4, 5}
    good = torch.tensor([r not in bad for r in range(T)])
    for b, rest in BOTH:
        grad, same = (torch.full((T, V), 9.0, dtype=TYPES[t], device=DEV) for _ in "12")
        stats, losses = run(lib, z.to(DEV), ids, tau, w, b, rest, 1.0, 1.0, grad)
        _, others = run(lib, quiet.to(DEV), ids, tau, w, b, rest, 1.0, 1.0, same)
        for r in bad:
            assert losses[r].isnan() and grad[r].isnan().all(), (r, b, rest, int((~grad[r].isnan()).sum()))
        assert stats[0].isnan()
        assert torch.equal(losses.cpu()[good], others.cpu()[good]) and torch.equal(grad.cpu()[good], same.cpu()[good])


@pytest.mark.parametrize("T,V,stride", [(700, 2000, 3_100_008), (70, 20_000, 31_200_008), (5, 40_000, (1 << 29) + 8), (5, 140_000, (1 << 29) + 8)])
def test_rows_past_2_to_the_31_elements(lib, T, V, stride):
    """Offsets of rows that 32 bits do not hold: the bits of the same rows side by side."""
    assert (T - 1) * stride > 1 << 31
    z, ids, tau, w = base(T, V, 20, dtype=torch.bfloat16)

    def far(x):
        rows = torch.empty((T - 1) * stride + V, dtype=x.dtype, device=DEV).as_strided((T, V), (stride, 1))
        return rows.copy_(x)

    results = []
    for place in (far, lambda v: v.to(DEV)):
        grad = place(torch.full((T, V), 9.0, dtype=torch.bfloat16))
        stats, losses = run(lib, place(z), ids, tau, w, 0.3, True, 1.0, 1.0, grad)
        results.append((stats, losses, grad.contiguous()))
    for a, b in zip(*results):
        assert torch.equal(a, b)
