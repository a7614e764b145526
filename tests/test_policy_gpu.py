"""GPU parity of the log-probabilities of tokens and of the policy loss with its
gradient (include/pda_ops.h) against 64-bit references with bounds from the
arithmetic (tests/_ops_ref.py)."""

import math

import pytest
import torch

from tests import _ops_ref as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    from paper_2605_20863_amd import _lib
    _lib.read_device_status()
    return _lib


def gen(seed):
    return torch.Generator().manual_seed(seed)


def batch(T, V, dtype, seed, amp=2.0, masked=0.0, ignored=0.2):
    """Logits with likely targets, some words masked with -inf, some rows without a target."""
    z = torch.randn((T, V), generator=gen(seed)) * amp
    if masked:
        z[torch.rand((T, V), generator=gen(seed + 1)) < masked] = -math.inf
    y = torch.randint(0, V, (T,), generator=gen(seed + 2))
    z[torch.arange(T), y] = 5 * torch.rand(T, generator=gen(seed + 3)) + 2 * amp
    if ignored:
        y = torch.where(torch.rand(T, generator=gen(seed + 4)) < ignored, torch.full_like(y, -100), y)
    return z.to(dtype), y


def padded(z, pad):
    """z on the device as a view with `pad` more elements a row."""
    T, V = z.shape
    full = torch.full((T, V + pad), float("nan"), dtype=z.dtype, device=DEV)
    full[:, :V] = z.to(DEV)
    return full[:, :V]


def close(got, want, bound, what):
    got = got.cpu().double()
    finite = want.isfinite()
    assert torch.equal(got[~finite], want[~finite]), what
    over = (got - want).abs() - bound - R.EPS24 * want.abs()
    assert (over[finite] <= 0).all(), f"{what}: over by {float(over[finite].max()):.3g}"


# one element, below and at vectors, odd, one part, many parts, beside every register variant's limit
VOCABS = [1, 2, 7, 8, 63, 1000, 4093, 8192, 8193, 16384, 32000, 50001, 65537, 131072, 163841]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("V", VOCABS)
def test_logprobs(lib, t, V):
    for T, pad, temp, idt in ((1, 0, 1.0, torch.int64), (5, 3, 0.7, torch.int32), (67, 1, 1.5, torch.int64)):
        if T * V > 5_000_000:
            T = 9
        print(f"[logprobs] {t} V={V} T={T}", flush=True)
        z, y = batch(T, V, TYPES[t], V + T, masked=0.1 if T > 1 else 0.0)
        x = padded(z, pad)
        lp, H = torch.full((T,), 9.0, device=DEV), torch.full((T,), 9.0, device=DEV)
        lib.token_logprobs(x, y.to(idt).to(DEV), lp, H, temperature=temp)
        _, _, want, ent, bl, bh = R.row_quantities(z, y, torch.tensor(temp, dtype=torch.float32).double().item())
        live = y >= 0
        close(lp, torch.where(live, want, 0.0), bl, "log-probabilities")
        close(H, torch.where(live, ent, 0.0), bh, "entropies")
        alone = torch.empty_like(lp)
        lib.token_logprobs(x, y.to(idt).to(DEV), alone, temperature=temp)
        assert torch.equal(alone, lp)
    assert lib.read_device_status() == 0


def test_many_rows_one_part(lib):
    """More rows than are cut into parts; rows past 2^31 elements."""
    V, T = 40_000, 3000
    x = torch.randn((T, V), generator=torch.Generator(DEV).manual_seed(1), device=DEV, dtype=torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=gen(2))
    lp, H = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    lib.token_logprobs(x, y.to(DEV), lp, H)
    at = torch.arange(0, T, 97)
    _, _, want, ent, bl, bh = R.row_quantities(x[at.to(DEV)].cpu(), y[at], 1.0)
    close(lp[at.to(DEV)], want, bl, "log-probabilities")
    close(H[at.to(DEV)], ent, bh, "entropies")
    V, T = 130_001, 17_000
    x = torch.empty((T, V), device=DEV, dtype=torch.bfloat16).normal_(generator=torch.Generator(DEV).manual_seed(3))
    y = torch.randint(0, V, (T,), generator=gen(4))
    lp, H = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    lib.token_logprobs(x, y.to(DEV), lp, H)
    at = torch.tensor([0, 1, 16_518, 16_519, 16_999])
    _, _, want, ent, bl, bh = R.row_quantities(x[at.to(DEV)].cpu(), y[at], 1.0)
    close(lp[at.to(DEV)], want, bl, "log-probabilities")
    w = torch.full((T,), 1.0 / T, device=DEV)
    stats = torch.empty(8, device=DEV)
    lib.policy_loss(x, y.to(DEV), lp, torch.ones(T, device=DEV), w, stats, dlogits=x)  # in place
    for i, r in enumerate(at.tolist()):
        g = x[r].float().cpu()
        # ratio 1: the gradient at the target is -(1 - p) / T, and sums to 0 over the row
        assert abs(float(g[y[r]]) * T + 1 - math.exp(float(want[i]))) < 4e-3
        assert abs(float(g.double().sum())) * T < 8e-3  # 130,001 roundings of 2^-9 of values that sum to 1
    close(stats[7:].cpu(), torch.ones(1, dtype=torch.float64), 1e-5, "weights")


def losses(T, y, lp, seed, ref=True, wide=1.0):
    """Rollout's and reference log-probabilities, advantages, weights; a log ratio away from the clip's corners."""
    d = torch.randn(T, generator=gen(seed)) * 0.4 * wide
    for c in (math.log(0.8), math.log(1.3), math.log(3.0), 20.0, -20.0):
        d = torch.where((d - c).abs() < 0.02, torch.full_like(d, c + 0.05), d)
    lp = lp.float()
    old = lp - d
    r = lp + torch.randn(T, generator=gen(seed + 1)) * 0.5 if ref else None
    adv = torch.randn(T, generator=gen(seed + 2))
    w = torch.rand(T, generator=gen(seed + 3)) / T
    w[torch.rand(T, generator=gen(seed + 4)) < 0.15] = 0
    return old, r, adv, w


CASES = [  # rows, padding, temperature, reference, dual clip, KL, entropy, scale, masked, log ratios' width
    (1, 0, 1.0, True, 0.0, 0.1, 0.01, 1.0, 0.0, 1.0),
    (6, 5, 0.8, True, 3.0, 0.05, 0.02, 128.0, 0.1, 3.0),
    (23, 0, 1.3, False, 3.0, 0.0, 0.0, 0.25, 0.05, 1.0),
    (230, 1, 1.0, True, 0.0, 0.2, 0.0, 1.0, 0.0, 1.0),
]


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("V", VOCABS)
def test_policy_loss(lib, t, V):
    dt = TYPES[t]
    for n, (T, pad, temp, ref, dual, kl, ent, scale, masked, wide) in enumerate(CASES):
        if T * V > 4_000_000:
            T = max(1, 4_000_000 // V)
        check_policy(lib, dt, T, V, pad, temp, ref, dual, kl, ent, scale, masked, wide, 1000 * n + V)


@pytest.mark.parametrize("t,V,T", [("bf16", 1003, 5000), ("f32", 8191, 700), ("bf16", 16385, 300), ("bf16", 65536, 200),
                                   ("bf16", 131073, 197), ("f32", 81920, 193), ("bf16", 163840, 193), ("f32", 81921, 193)])
def test_policy_loss_of_many_rows(lib, t, V, T):
    check_policy(lib, TYPES[t], T, V, 1, 0.9, True, 3.0, 0.05, 0.01, 1.0, 0.02, 1.0, V)


@pytest.mark.parametrize("t,V,T", [("bf16", 163_857, 130), ("f32", 81_930, 131), ("f32", 114_691, 128),
                                   ("f32", 114_692, 129), ("bf16", 229_383, 130), ("f32", 150_001, 140), ("bf16", 32_000, 127),
                                   ("bf16", 32_000, 128), ("bf16", 16_391, 5), ("bf16", 16_392, 5),
                                   ("bf16", 163_857, 170), ("bf16", 229_383, 161), ("bf16", 229_384, 161),
                                   ("bf16", 32_000, 159), ("bf16", 32_000, 160), ("f32", 20_001, 111), ("f32", 20_001, 112)])
def test_policy_loss_beside_the_rule(lib, t, V, T):
    """Rows too long for registers, read twice; the sizes on both sides of the rule that chooses."""
    check_policy(lib, TYPES[t], T, V, 0, 1.0, True, 0.0, 0.1, 0.01, 1.0, 0.01, 1.0, V + T)


def check_policy(lib, dt, T, V, pad, temp, ref, dual, kl, ent, scale, masked, wide, seed):
    print(f"[policy] {dt} V={V} T={T}", flush=True)
    z, y = batch(T, V, dt, seed, masked=masked)
    temp = torch.tensor(temp, dtype=torch.float32).double().item()
    low, high = (torch.tensor(c, dtype=torch.float32).double().item() for c in (0.2, 0.3))
    _, _, lp, _, _, _ = R.row_quantities(z, y, temp)
    old, r, adv, w = losses(T, y, torch.where(y >= 0, lp, 0.0), seed + 7, ref, wide)
    want = R.policy(z, y, old, r, adv, w, temp, low, high, dual, kl, ent, scale)
    x = padded(z, pad)
    o = [torch.full((T,), 9.0, device=DEV) for _ in range(2)]
    stats, grad = torch.full((8,), 9.0, device=DEV), torch.full((T, V + 3), 9.0, dtype=dt, device=DEV)
    more = dict(ref_logprobs=None if r is None else r.to(DEV), clip_low=0.2, clip_high=high, dual_clip=dual, kl_coef=kl,
                entropy_coef=ent, temperature=temp, grad_scale=scale)
    given = [v.to(DEV) for v in (y, old, adv, w)]
    lib.policy_loss(x, *given, stats, grad[:, :V], *o, **more)
    close(o[0], want["logprobs"], want["lp_bound"], "log-probabilities")
    close(o[1], want["entropy"], want["h_bound"], "entropies")
    R.assert_within(grad[:, :V], want["dlogits"], want["grad_bound"], dt, f"gradient V={V} T={T}")
    assert (grad[:, V:] == 9.0).all()
    # a term's error: its steepness in lp, and roundings of its size
    live = want["weights"] != 0
    slack = want["steep"] + 1 + want["terms"].abs().sum(dim=0)
    err = (want["weights"] * slack * (want["lp_bound"] + want["h_bound"] + 16 * R.EPS24))[live].sum()
    assert ((stats.cpu().double() - want["stats"]).abs() <= err + R.EPS24 * want["stats"].abs() + 1e-30).all(), (stats, want["stats"])
    # the loss alone, and in place of the logits: the same
    again = torch.empty_like(stats)
    lib.policy_loss(x, *given, again, **more)
    assert torch.equal(again, stats)
    lib.policy_loss(x, *given, again, x, **more)
    assert torch.equal(x, grad[:, :V]) and torch.equal(again, stats)
    assert lib.read_device_status() == 0


@pytest.mark.parametrize("rows", [3, 300])  # in parts, and in registers
@pytest.mark.parametrize("V", [500, 20_000])
def test_gradient_against_differences(lib, rows, V):
    """The loss's own differences (in float64, from the reference's loss) agree with dlogits along random directions."""
    z, y = batch(rows, V, torch.float32, 3, ignored=0.1)
    _, _, lp, _, _, _ = R.row_quantities(z, y, 1.0)
    old, r, adv, w = losses(rows, y, torch.where(y >= 0, lp, 0.0), 5)
    low = torch.tensor(0.2, dtype=torch.float32).double().item()
    stats, grad = torch.empty(8, device=DEV), torch.empty((rows, V), device=DEV)
    given = [v.to(DEV) for v in (y, old, adv, w)]
    lib.policy_loss(z.to(DEV), *given, stats, grad, ref_logprobs=r.to(DEV), kl_coef=0.1, entropy_coef=0.05)
    for seed in range(3):
        u = torch.randn((rows, V), generator=gen(40 + seed)).double()
        h = 1e-4
        f = [R.policy(z.double() + s * h * u, y, old, r, adv, w, 1.0, low, low, 0.0, 0.1, 0.05, 1.0)["stats"][0] for s in (1, -1)]
        slope, want = float(f[0] - f[1]) / (2 * h), float((grad.cpu().double() * u).sum())
        size = float((grad.cpu().double() * u).square().sum().sqrt())
        # h^2 of the third derivative (about 1), the reference's 1e-16 over h, float32 elements
        assert abs(slope - want) <= 1e-5 * size + 1e-7, (slope, want)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(7, 3000), (7, 40_000), (200, 3000), (200, 40_000)])
def test_rows_that_masks_leave_nothing_of(lib, t, T, V):
    dt = TYPES[t]
    lowest = torch.finfo(dt).min
    z, y = batch(T, V, dt, 1, ignored=0.0)
    z[0] = -math.inf                                # nothing left
    z[1] = lowest                                   # the type's lowest everywhere: an even distribution
    z[2] = -math.inf
    z[2, y[2]] = 3.0                                # the target alone
    z[3, y[3]] = -math.inf                          # all but the target
    z[4, (y[4] + 1) % V] = float("nan")
    z[5, (y[5] + 1) % V] = math.inf
    z[6] = lowest
    z[6, y[6]] = 1.0
    lp, H, stats = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty(8, device=DEV)
    grad = torch.full((T, V), 9.0, dtype=dt, device=DEV)
    w = torch.full((T,), 1.0 / T)
    w[4] = w[5] = 0
    args = [v.to(DEV) for v in (z, y, torch.full((T,), -1.0), torch.ones(T), w)]
    lib.policy_loss(*args, stats, grad, lp, H, ref_logprobs=torch.full((T,), -1.0, device=DEV), kl_coef=0.1, entropy_coef=0.1)
    a, b = torch.empty_like(lp), torch.empty_like(H)
    lib.token_logprobs(args[0], args[1], a, b)
    for x, e in ((lp, H), (a, b)):
        assert x[0] == -math.inf and e[0] == 0
        assert abs(float(x[1]) + math.log(V)) < 1e-5 and abs(float(e[1]) - math.log(V)) < 1e-5
        assert x[2] == 0 and e[2] == 0 and x[6] == 0 and e[6] == 0
        assert x[3] == -math.inf and math.isfinite(float(e[3]))
        assert all(math.isnan(float(v)) for v in (x[4], x[5], e[4], e[5]))
        assert x[7:].isfinite().all() and e[7:].isfinite().all()
    assert (grad[0] == 0).all() and (grad[4] == 0).all() and (grad[5] == 0).all()
    assert grad.isfinite().all() and stats.isfinite().all()
    assert (grad[2] == 0).all() and (grad[6] == 0).all()
    # with weight, the NaN stays in its row
    w[4] = 1.0 / T
    lib.policy_loss(*args[:4], w.to(DEV), stats, grad)
    assert grad[4].isnan().any() and grad[[0, 1, 2, 3, 5, 6]].isfinite().all() and stats[0].isnan()


def test_targets_outside_the_vocabulary(lib):
    z, _ = batch(4, 100, torch.float32, 1, ignored=0.0)
    lp, H = torch.empty(4, device=DEV), torch.empty(4, device=DEV)
    stats, grad, one = torch.empty(8, device=DEV), torch.empty((4, 100), device=DEV), torch.ones(4, device=DEV)
    for bad in (100, 2 ** 31 - 1, 2 ** 40):
        y = torch.tensor([3, bad, -1, 99], device=DEV)
        lib.token_logprobs(z.to(DEV), y, lp, H)
        assert lib.read_device_status() == lib.STATUS_BAD_TARGET
        assert lp[1] == lp[2] == H[1] == H[2] == 0 and (lp[[0, 3]] < 0).all()
        lib.policy_loss(z.to(DEV), y, lp, one, one, stats, grad)
        assert lib.read_device_status() == lib.STATUS_BAD_TARGET
        assert (grad[[1, 2]] == 0).all() and (grad[[0, 3]] != 0).all() and stats[7] == 2


def test_no_rows(lib):
    z, e = torch.empty((0, 50), device=DEV), torch.empty(0, device=DEV)
    y = torch.empty(0, dtype=torch.int64, device=DEV)
    stats = torch.full((8,), 3.0, device=DEV)
    lib.token_logprobs(z, y, e, e)
    lib.policy_loss(z, y, e, e, e, stats, z)
    assert (stats == 0).all()


@pytest.mark.parametrize("T,V", [(4, 40_000), (256, 9000)])
def test_graph_and_streams(lib, T, V):
    """Captured on a side stream, replayed with logits changed in place; every replay equals the eager call."""
    z, y = batch(T, V, torch.bfloat16, 1)
    x, y = z.to(DEV), y.to(DEV)
    old, adv, w = (torch.randn(T, device=DEV) - 2 for _ in range(3))
    a = [torch.empty(8, device=DEV), torch.empty_like(x), torch.empty(T, device=DEV), torch.empty(T, device=DEV)]
    b = [torch.empty_like(v) for v in a]
    s = torch.cuda.Stream(DEV)
    s.wait_stream(torch.cuda.current_stream())

    def call(o):
        lib.policy_loss(x, y, old, adv, w, o[0], o[1], o[2])
        lib.token_logprobs(x, y, o[3])

    with torch.cuda.stream(s):
        call(a)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call(a)
    for r in range(4):
        x.normal_()
        for v in a:
            v.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        call(b)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a, b)), r
