"""GPU parity of the distillation loss and its gradient (include/pda_lm.h) against a 64-bit reference with bounds from
the arithmetic (tests/_lm_ref.py)."""

import math

import pytest
import torch

from tests import _lm_ref as R
from tests.test_policy_gpu import VOCABS, lib, padded  # noqa: F401

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def lists(T, V, K, seed, ragged=True, close=0.5, dtype=torch.float32, masked=0.0):
    """Logits, lists of all different words in any order, weights."""
    z = torch.randn((T, V), generator=gen(seed)) * 2
    if masked:
        z[torch.rand((T, V), generator=gen(seed + 1)) < masked] = -math.inf
    ids, tau = torch.full((T, K), -1, dtype=torch.int32), torch.full((T, K), -math.inf)
    n = min(K, V)
    for t in range(T):
        word = torch.randperm(V, generator=gen(seed + 10 + t))[:n]
        mass = 1 - 10 ** (-0.3 - 4 * float(torch.rand(1, generator=gen(seed + t))))
        lt = torch.log_softmax(torch.randn(n, generator=gen(seed + 500 + t)) * 2, 0) + math.log(mass)
        z[t, word] = math.log(V) + 4 + lt + close * torch.randn(n, generator=gen(seed + 900 + t))
        m = int(torch.randint(0, n + 1, (1,), generator=gen(seed + 77 + t))) if ragged and t % 5 == 3 else n
        ids[t, :m], tau[t, :m] = word[:m].int(), lt[:m].float()
    if K > 2:  # empty places need not be the last
        ids[0, K // 2], tau[0, K // 2] = -7, -1.0
        tau[-1, 0] = -math.inf
    w = torch.rand(T, generator=gen(seed + 4)) / T
    if T > 2:
        w[T // 2] = 0
    return z.to(dtype), ids, tau, w


def run(lib, x, ids, tau, w, b, rest, temp, scale=1.0, grad=None, losses=True):
    T, V = x.shape
    stats = torch.full((6,), 9.0, device=DEV)
    loss = torch.full((T,), 9.0, device=DEV) if losses else None
    lib.distill_loss(x, ids.to(DEV), tau.to(DEV), w.to(DEV), stats, grad, loss, reverse=b, rest=rest, temperature=temp,
                     grad_scale=scale)
    return stats, loss


def check(lib, z, ids, tau, w, b, rest, temp, scale, pad=0):
    T, V = z.shape
    x = padded(z, pad)
    grad = torch.full((T, V + 3), 9.0, dtype=z.dtype, device=DEV)
    stats, losses = run(lib, x, ids, tau, w, b, rest, temp, scale, grad[:, :V])
    f32 = lambda v: torch.tensor(v, dtype=torch.float32).double().item()  # noqa: E731
    want = R.distill(z, ids, tau, w, f32(b), rest, f32(temp), scale)
    R.near(losses, want["losses"], want["loss_bound"], torch.float32, "losses")
    R.near(grad[:, :V], want["dlogits"], want["grad_bound"], z.dtype, f"gradient V={V} T={T}")
    assert (grad[:, V:] == 9.0).all()
    wd = w.double()[:, None]
    terms = torch.where(wd != 0, want["terms"] * wd, 0.0)
    slack = torch.where(wd != 0, (want["term_bounds"] + 2 * R.EPS24 * want["terms"].abs()).nan_to_num(0.0, 0.0, 0.0) * wd, 0.0)
    R.near(stats, terms.sum(dim=0), slack.sum(dim=0), torch.float32, "sums")
    # the loss alone, and in place of the logits: the same
    again, _ = run(lib, x, ids, tau, w, b, rest, temp, scale, losses=False)
    assert torch.equal(again, stats)
    again, _ = run(lib, x, ids, tau, w, b, rest, temp, scale, x)
    assert torch.equal(x, grad[:, :V]) and torch.equal(again, stats)
    return stats, losses, grad[:, :V]


CASES = [  # rows, places, padding, temperature, reverse, rest, scale, masked
    (1, 1, 0, 1.0, 0.0, True, 1.0, 0.0),
    (6, 20, 5, 0.8, 0.0, True, 128.0, 0.1),
    (5, 256, 0, 1.3, 0.5, True, 1.0, 0.0),
    (4, 33, 1, 1.0, 1.0, True, 0.25, 0.05),
    (7, 64, 2, 1.0, 0.0, False, 1.0, 0.0),
    (3, 100, 0, 0.9, 0.7, False, 1.0, 0.1),
]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("V", VOCABS)
def test_distill(lib, t, V):
    for n, (T, K, pad, temp, b, rest, scale, masked) in enumerate(CASES):
        print(f"[distill] {t} V={V} T={T} K={K} reverse={b} rest={rest}", flush=True)
        z, ids, tau, w = lists(T, V, K, 1000 * n + V, dtype=TYPES[t], masked=masked)
        check(lib, z, ids, tau, w, b, rest, temp, scale, pad)
    assert lib.read_device_status() == 0


@pytest.mark.parametrize("t,V,T", [("bf16", 1003, 700), ("f32", 4001, 300), ("bf16", 16_391, 170), ("f32", 8193, 170),
                                   ("bf16", 65_537, 165), ("f32", 40_000, 165), ("bf16", 131_073, 161), ("f32", 70_001, 161),
                                   ("bf16", 2047, 600), ("bf16", 2056, 601),
                                   ("f32", 1023, 777), ("f32", 2050, 650), ("bf16", 4096, 640), ("bf16", 8191, 610), ("bf16", 8200, 602),
                                   ("f32", 4100, 603), ("bf16", 40, 1000), ("f32", 3, 5000),
                                   ("bf16", 170_001, 161), ("bf16", 204_801, 161), ("f32", 102_401, 161), ("bf16", 300_001, 5),
                                   # both sides of the rule between a workgroup a row and parts
                                   ("bf16", 32_774, 1), ("bf16", 32_784, 1), ("bf16", 50_000, 28), ("bf16", 50_000, 29), ("f32", 50_001, 56),
                                   ("f32", 50_001, 57), ("bf16", 131_072, 74), ("bf16", 131_072, 75), ("f32", 110_000, 124), ("f32", 110_000, 125),
                                   ("bf16", 524_296, 3), ("bf16", 530_001, 128), ("f32", 262_150, 129)])
def test_many_rows(lib, t, V, T):
    n = 4_000_000 // V + 1
    z, ids, tau, w = lists(min(T, n), V, 70, V, dtype=TYPES[t])
    reps = -(-T // z.shape[0])
    z, ids, tau, w = (v.repeat(reps, *[1] * (v.dim() - 1))[:T] for v in (z, ids, tau, w))
    # a repetition's own place in memory changes how its ends are cut, so each is held against the reference
    x, k = padded(z, 1), min(T, n)
    grad = torch.empty((T, V), dtype=z.dtype, device=DEV)
    _, losses = run(lib, x, ids, tau, w, 0.3, True, 1.1, 1.0, grad)
    f32 = lambda v: torch.tensor(v, dtype=torch.float32).double().item()  # noqa: E731
    want = R.distill(z[:k], ids[:k], tau[:k], w[:k], f32(0.3), True, f32(1.1), 1.0)
    for i in range(0, T, k):
        m = min(k, T - i)
        R.near(losses[i:i + m], want["losses"][:m], want["loss_bound"][:m], torch.float32, "losses")
        R.near(grad[i:i + m], want["dlogits"][:m], want["grad_bound"][:m], z.dtype, "gradient")


def base(T, V, K, seed=3, dtype=torch.float32):
    z, ids, tau, w = lists(T, V, K, seed, ragged=False, dtype=dtype)
    return z, ids, tau, torch.full((T,), 1.0 / T)


@pytest.mark.parametrize("T,V", [(6, 500), (6, 40_000), (200, 20_000), (700, 300), (700, 3000), (610, 8000)])
def test_lists_out_of_the_ordinary(lib, T, V):
    """No entry, every word listed, the same word twice, words past the vocabulary, masked words."""
    K = 12
    z, ids, tau, w = base(T, V, K)
    ids[0], tau[1] = -1, -math.inf          # empty lists
    ids[2, 5], ids[2, 9] = V, 2 ** 31 - 1   # past the vocabulary
    ids[3, 7] = ids[3, 1]                   # twice
    ids[3, 8] = ids[3, 1]
    ids[4, 2] = -1
    ids[5, 3] = ids[5, 10]                  # the first place counts
    tau[5, 10] = -1.5
    for b, rest in ((0.0, True), (1.0, True), (0.4, True), (0.0, False), (1.0, False)):
        stats, losses, grad = check(lib, z, ids, tau, w, b, rest, 1.0, 1.0)
        assert lib.read_device_status() == lib.STATUS_BAD_TARGET | lib.STATUS_TWICE
        assert losses[0] == 0 and losses[1] == 0 and (grad[:2] == 0).all()


@pytest.mark.parametrize("V", [1, 2, 40, 256])
@pytest.mark.parametrize("b,rest", [(0.0, True), (0.6, True), (1.0, False), (0.0, False)])
def test_every_word_listed(lib, V, b, rest):
    """No rest, though the teacher's probabilities do not quite sum to 1."""
    z, ids, tau, w = lists(5, V, V, 3, ragged=False)
    ids = torch.stack([torch.randperm(V, generator=gen(t)) for t in range(5)]).int()
    tau = torch.log_softmax(torch.randn((5, V), generator=gen(9)), 1)
    check(lib, z, ids, tau, w, b, rest, 1.0, 1.0)


@pytest.mark.parametrize("T,V", [(9, 700), (9, 40_000), (170, 20_000), (700, 700), (640, 5000)])
@pytest.mark.parametrize("b,rest", [(0.0, True), (0.5, True), (1.0, True), (0.0, False), (1.0, False)])
def test_masks_and_special_values(lib, T, V, b, rest):
    """Masked words in and out of the list, rows of -inf, NaN and infinities in their own rows, rows of weight 0."""
    K = 9
    z, ids, tau, w = base(T, V, K)
    z[0] = -math.inf
    z[1, ids[1, 2]] = -math.inf                         # a listed word: forward is +inf, its gradient finite
    keep = z[2, ids[2].clamp(min=0).long()].clone()
    z[2] = -math.inf                                     # all others: no rest
    z[2, ids[2].clamp(min=0).long()] = keep
    z[3] = -3.3e38                                       # the type's lowest: an even distribution
    z[4, V // 2:] = -3.3e38
    stats, losses, grad = check(lib, z, ids, tau, w, b, rest, 1.0, 1.0)
    assert (grad[0] == 0).all() and grad[1].isfinite().all()
    if b < 1:
        assert losses[1] == math.inf and losses[0] == math.inf
    z[5, 3], z[6, ids[6, 1]], z[7, 8], tau[8, 2] = math.nan, math.nan, math.inf, math.nan
    w[8] = 0
    x, grad = z.to(DEV), torch.empty((T, V), device=DEV)
    stats, again = run(lib, x, ids, tau, w, b, rest, 1.0, 1.0, grad)
    for r in (5, 6, 7, 8):
        assert again[r].isnan()
    assert stats[0].isnan() and (grad[8] == 0).all()
    assert torch.equal(again[:5], losses[:5]) and torch.equal(again[9:], losses[9:])
    grad.fill_(9.0)
    w[5:9] = 0  # rows that take no part, whatever is in them
    z[5] = math.nan
    z[6] = 300.0
    stats, again = run(lib, z.to(DEV), ids, tau, w, b, rest, 1.0, 1.0, grad)
    quiet, none = run(lib, z.to(DEV), ids, tau, w, b, rest, 1.0, 1.0, grad, losses=False)
    assert (grad[5:9] == 0).all() and not stats[1].isnan() and none is None
    assert torch.equal(quiet, stats)
    grad.fill_(9.0)
    run(lib, x, ids, tau, torch.ones(T) / T, b, rest, 1.0, 1.0, grad)
    for r in (5, 6, 7):
        assert grad[r].isnan().all() or (~grad[r].isnan()).sum() <= K


@pytest.mark.parametrize("t,V", [("bf16", 70_001), ("bf16", 140_000), ("bf16", 200_003), ("f32", 110_001)])
def test_lowest_words_of_long_rows(lib, t, V):
    """Rows in registers, LDS and read again, whose words are the type's lowest in whole or in part."""
    T = 130
    z, ids, tau, w = base(T, V, 40)
    z = z.to(TYPES[t])
    z[0] = -3.3e38
    z[1, : V // 2] = -3.3e38
    z[2, V // 2:] = -3.3e38
    z[3, V - 20_000: V - 9] = -math.inf
    z[4, 5:30] = -3.3e38
    check(lib, z, ids, tau, w, 0.5, True, 1.0, 64.0)


@pytest.mark.parametrize("T,V", [(5, 900), (4, 40_000), (650, 700)])
@pytest.mark.parametrize("temp", [1e-37, 1e-20, 1e24, 1e38])
def test_temperatures(lib, T, V, temp):
    """Near 0 one word takes all, far up all take the same: the parts that are finite are as the reference has them."""
    z, ids, tau, w = base(T, V, 9)
    z[0] = -3.3e38
    z[1, : V // 2] = -3.3e38
    exact = torch.tensor(temp, dtype=torch.float32).double().item()
    for b, rest in ((0.0, True), (1.0, True), (1.0, False)):
        grad = torch.empty((T, V), device=DEV)
        _, losses = run(lib, z.to(DEV), ids, tau, w, b, rest, temp, min(temp, 1.0), grad)
        want = R.distill(z, ids, tau, w, b, rest, exact, min(exact, 1.0))
        finite = want["losses"] < 3e38
        assert (losses.cpu()[~finite] > 2.9e38).all()
        R.near(losses[finite.to(DEV)], want["losses"][finite], want["loss_bound"][finite] + 4 * R.EPS24 * want["losses"][finite].abs(),
               torch.float32, "losses")
        if temp > 1:
            R.near(grad, want["dlogits"], want["grad_bound"] * (1 + 1e-6), torch.float32, "gradient")
        else:
            assert grad.isfinite().all()


@pytest.mark.parametrize("rest", [True, False])
def test_close_distributions_keep_their_digits(lib, rest):
    """A student that has learnt nearly everything: the divergences are far below their terms."""
    T, V, K = 5, 5000, 40
    z = (torch.randn((T, V), generator=gen(1)) * 3).float()
    lp = torch.log_softmax(z.double(), 1)
    top = lp.topk(K, dim=1)
    tau = (top.values + 1e-3 * torch.randn((T, K), generator=gen(2)).double()).float()
    if rest:
        check(lib, z, top.indices.int(), tau, torch.ones(T) / T, 0.0, rest, 1.0, 1.0)
        _, losses = run(lib, z.to(DEV), top.indices.int(), tau, torch.ones(T) / T, 0.0, rest, 1.0)
        want = R.distill(z, top.indices.int(), tau, torch.ones(T) / T, 0.0, rest, 1.0, 1.0)["losses"]
        assert want.max() < 1e-5
        # terms are t a^2 / 2 with a off by 2^-21 at most, of a size of 1e-3
        assert ((losses.cpu().double() - want).abs() <= 4e-3 * want + 1e-12).all()
    else:
        check(lib, z, top.indices.int(), tau, torch.ones(T) / T, 0.0, rest, 1.0, 1.0)


@pytest.mark.parametrize("rows", [3, 300])
@pytest.mark.parametrize("b,rest", [(0.0, True), (0.3, True), (1.0, False)])
def test_gradient_against_differences(lib, rows, b, rest):
    V, K = 2000, 30
    z, ids, tau, w = lists(min(rows, 3), V, K, 5)
    reps = rows // z.shape[0]
    grad = torch.empty((rows, V), device=DEV)
    args = [v.repeat(reps, *[1] * (v.dim() - 1)) for v in (z, ids, tau, w)]
    run(lib, args[0].to(DEV), *args[1:], b, rest, 1.2, 1.0, grad)
    f32 = torch.tensor(1.2, dtype=torch.float32).double().item()
    bb = torch.tensor(b, dtype=torch.float32).double().item()

    def value(z):
        return float((R.distill(z, ids, tau, w, bb, rest, f32, 1.0)["losses"] * w.double()).sum())

    g, e = grad[:z.shape[0]].cpu().double(), 1e-4
    for seed in range(3):
        v = torch.randn(z.shape, generator=gen(30 + seed)).double()
        slope = (value(z.double() + e * v) - value(z.double() - e * v)) / (2 * e)
        # float32 gradients, and differences of second order of a function of size 1
        assert abs(slope - float((g * v).sum())) <= 1e-5 * float((g * v).abs().sum()) + 1e-7


def test_what_a_teacher_writes(lib):
    """Lists from top_logprobs go in as they are: a student equal to its teacher has loss 0 and no gradient to speak of."""
    T, V, K = 50, 30_000, 64
    z = (torch.randn((T, V), generator=gen(1)) * 2).to(DEV)
    ids, tau = torch.empty((T, K), dtype=torch.int32, device=DEV), torch.empty((T, K), device=DEV)
    y = torch.zeros(T, dtype=torch.int64, device=DEV)
    y[3] = -1
    lib.top_logprobs(z, ids, tau, y, temperature=0.7)
    for b in (0.0, 0.5, 1.0):
        stats, losses, grad = torch.empty(6, device=DEV), torch.empty(T, device=DEV), torch.empty_like(z)
        lib.distill_loss(z, ids, tau, torch.ones(T, device=DEV), stats, grad, losses, reverse=b, temperature=0.7)
        assert losses.abs().max() < 1e-6 and grad.abs().max() < 2e-6 and losses[3] == 0
        assert abs(float(stats[5]) - T) < 1e-4


def test_no_rows(lib):
    e, s = torch.empty((0, 10), device=DEV), torch.full((6,), 9.0, device=DEV)
    lib.distill_loss(e, torch.empty((0, 3), dtype=torch.int32, device=DEV), torch.empty((0, 3), device=DEV),
                     torch.empty(0, device=DEV), s, e)
    assert (s == 0).all()
