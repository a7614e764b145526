"""GPU parity of the most likely words of rows of logits (include/pda_lm.h): the words exactly, their
log-probabilities against a 64-bit reference with bounds from the arithmetic (tests/_lm_ref.py)."""

import math

import pytest
import torch

from tests import _lm_ref as R
from tests.test_policy_gpu import VOCABS, batch, lib, padded  # noqa: F401

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def run(lib, x, K, temp, y=None, ent=True):
    T = x.shape[0]
    ids, tops = torch.full((T, K), 9, dtype=torch.int32, device=DEV), torch.full((T, K), 9.0, device=DEV)
    lp = None if y is None else torch.full((T,), 9.0, device=DEV)
    H = torch.full((T,), 9.0, device=DEV) if ent else None
    lib.top_logprobs(x, ids, tops, None if y is None else y.to(DEV), lp, H, temperature=temp)
    return ids, tops, lp, H


def check(lib, z, K, temp, y=None, pad=0, idt=torch.int64):
    x = padded(z, pad)
    exact = torch.tensor(temp, dtype=torch.float32).double().item()
    ids, tops, lp, H = run(lib, x, K, temp, None if y is None else y.to(idt))
    want, (wt, bt), (wl, bl), (wh, bh) = R.top(z, K, exact, y)
    assert torch.equal(ids.cpu().long(), want), (ids.cpu().long() != want).nonzero()[:4]
    R.near(tops, wt, bt, torch.float32, "log-probabilities")
    R.near(H, wh, bh, torch.float32, "entropies")
    if y is not None:
        R.near(lp, wl, bl, torch.float32, "targets' log-probabilities")
    return ids, tops, lp, H


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("V", VOCABS + [1029, 2047, 2056, 4100])
def test_top(lib, t, V):
    for T, pad, temp, K, masked, targets in ((1, 0, 1.0, 1, 0.0, False), (5, 3, 0.7, 20, 0.1, True), (3, 1, 1.0, 256, 0.0, False),
                                             (67, 2, 1.5, 64, 0.02, True), (2, 0, 1.0, 255, 0.5, False)):
        if T * V > 3_000_000:
            T = 9
        print(f"[top] {t} V={V} T={T} K={K}", flush=True)
        z, y = batch(T, V, TYPES[t], V + T + K, masked=masked)
        check(lib, z, K, temp, y if targets else None, pad, torch.int32 if K == 20 else torch.int64)
    assert lib.read_device_status() == 0


@pytest.mark.parametrize("t,V,T", [("bf16", 1003, 1500), ("bf16", 3001, 700), ("bf16", 4103, 650), ("f32", 2051, 605), ("f32", 8191, 1030), ("bf16", 40_001, 1100), ("f32", 50_001, 300),
                                   ("bf16", 131_072, 140)])
def test_many_rows(lib, t, V, T):
    g = torch.Generator(DEV).manual_seed(V)
    x = torch.empty((T, V + 1), device=DEV, dtype=TYPES[t]).normal_(0, 2, generator=g)[:, :V]
    at = torch.arange(0, T, 61)
    for K in (1, 50, 256):
        ids, tops, _, H = run(lib, x, K, 1.0)
        want, (wt, bt), _, (wh, bh) = R.top(x[at.to(DEV)].cpu(), K, 1.0)
        assert torch.equal(ids[at.to(DEV)].cpu().long(), want)
        R.near(tops[at.to(DEV)], wt, bt, torch.float32, "log-probabilities")
        R.near(H[at.to(DEV)], wh, bh, torch.float32, "entropies")
        # each word is its row's, once; each row's values go down
        assert torch.equal(x.gather(1, ids.long()).float().argsort(dim=1, descending=True, stable=True),
                           torch.arange(K, device=DEV).expand(T, K))
        assert (ids.sort(dim=1).values.diff(dim=1) > 0).all()


def orders(V):
    """Rows in which the words that pass what came before are many."""
    i = torch.arange(V, dtype=torch.float32)
    saw = (i % 300) / 7
    return {"rising": i / V * 30, "falling": -i / V * 30, "equal": torch.zeros(V), "rising steps": (i // 37) / V * 300, "saw": saw,
            "blocks": (i // 2048) % 3, "late": torch.where(i > V - 700, 5.0 + i / V, torch.zeros(V)),
            "one thread's": torch.where(i % 2048 < 16, 9.0 + i / V, i / V), "zeros": torch.where(i % 2 == 0, 0.0, -0.0),
            "zero bar": torch.where(i % 3 == 0, 0.0, -1.0 - i / V), "lowest": torch.full((V,), -3.3e38), "two": torch.where((i == 5) | (i == V - 1), 1.0, -math.inf)}


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("V", [260, 700, 2040, 4003, 20_003, 131_072])
def test_orders(lib, t, V):
    rows = orders(V)
    z = torch.stack(list(rows.values())).to(TYPES[t])
    for K in (1, 17, 256):
        for T in (1, 60):  # few rows and many
            print(f"[orders] {t} V={V} K={K} T={T}", flush=True)
            if T == 1:
                for r in range(len(rows)):
                    check(lib, z[r:r + 1], K, 1.0)
            else:
                check(lib, z.repeat(T if V < 30_000 else 3, 1), K, 1.0, None, 1)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("V", [50, 1500, 9000, 70_001])
@pytest.mark.parametrize("T", [7, 300])
def test_masks_and_special_values(lib, t, V, T):
    """Rows of -inf, of NaN, with NaN and infinities; rows that take no part."""
    K = 30
    g = torch.Generator().manual_seed(V)
    z = torch.randn((T, V), generator=g).to(TYPES[t])
    z[0] = -math.inf
    z[1] = math.nan
    z[2, V // 2] = math.nan
    z[3, 3] = math.inf
    z[4, 10:] = -math.inf
    y = torch.arange(T) % V
    y[5], y[6] = -1, V
    x = padded(z, 1)
    ids, tops, lp, H = (v.cpu() for v in run(lib, x, K, 1.0, y))
    assert lib.read_device_status() == lib.STATUS_BAD_TARGET
    assert (ids[0] == -1).all() and (tops[0] == -math.inf).all() and lp[0] == -math.inf and H[0] == 0
    assert torch.equal(ids[1], torch.arange(K, dtype=torch.int32)) and tops[1].isnan().all()
    assert ids[2, 0] == V // 2 and ids[3, 0] == 3
    for r in (1, 2, 3):
        assert tops[r].isnan().all() and lp[r].isnan() and H[r].isnan()
    assert (ids[4, :10] >= 0).all() and (ids[4, 10:] == -1).all() and (tops[4, 10:] == -math.inf).all()
    for r in (5, 6):
        assert (ids[r] == -1).all() and (tops[r] == -math.inf).all() and lp[r] == 0 and H[r] == 0
    want, (wt, bt), (wl, bl), (wh, bh) = R.top(z, K, 1.0, torch.where(y == V, -1, y))
    rest = [4] + list(range(7, T))
    assert torch.equal(ids[rest].long(), want[rest])
    R.near(tops[rest], wt[rest], bt[rest], torch.float32, "log-probabilities")
    R.near(lp[rest], wl[rest], bl[rest], torch.float32, "targets'")
    if T > 7:
        R.near(H[rest], wh[rest], bh[rest], torch.float32, "entropies")


@pytest.mark.parametrize("V", [3000, 9000, 70_001])
def test_infinities_and_nan_among_each_other(lib, V):
    """More of +inf than places, and NaN before, among and after them; more NaN than places."""
    z = torch.randn((4, V), generator=torch.Generator().manual_seed(V))
    z[0, 5:500] = math.inf
    z[0, V - 3] = math.nan
    z[1, 100:2900:7] = math.nan
    z[1, 0] = math.inf
    z[2, V // 2] = math.inf
    z[3, 40], z[3, 41], z[3, V - 1] = math.inf, -math.nan, math.nan
    for K in (1, 2, 20, 256):
        for x in (z, z.to(torch.bfloat16)):
            rank = torch.where(x.isnan(), 3e38, torch.where(x == math.inf, 2e38, x.double()))
            want = rank.sort(dim=1, descending=True, stable=True).indices[:, :K]
            for r in (x, x.repeat(300, 1)):
                ids, tops, _, _ = run(lib, r.to(DEV), K, 1.0)
                assert torch.equal(ids.cpu().long(), want.repeat(r.shape[0] // 4, 1)) and tops.isnan().all()


def test_options_change_nothing_else(lib):
    """Without targets, log-probabilities or entropies the words and their values are the same; K cuts the list."""
    for T, V in ((3, 131_072), (2000, 5000)):
        z, y = batch(T, V, torch.bfloat16, 1, ignored=0.0)
        x = z.to(DEV)
        ids, tops, lp, H = run(lib, x, 64, 0.9, y)
        a, b, _, h = run(lib, x, 64, 0.9)
        assert torch.equal(a, ids) and torch.equal(b, tops) and torch.equal(h, H)
        a, b, _, _ = run(lib, x, 64, 0.9, None, False)
        assert torch.equal(a, ids) and torch.equal(b, tops)
        a, b, l2, _ = run(lib, x, 5, 0.9, y, False)
        assert torch.equal(a, ids[:, :5]) and torch.equal(b, tops[:, :5]) and torch.equal(l2, lp)
        # as the call for given words alone has them, up to the order of float32 sums
        one, e = torch.empty_like(lp), torch.empty_like(lp)
        lib.token_logprobs(x, y.to(DEV), one, e, temperature=0.9)
        assert (one - lp).abs().max() < 2e-5 and (e - H).abs().max() < 2e-5


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("temp", [1e-37, 1e-30, 1e-6, 1e6, 1e24, 1e38])
@pytest.mark.parametrize("T,V", [(5, 900), (4, 9000), (3, 70_001), (700, 3000)])
def test_temperatures(lib, t, temp, T, V):
    """From one word that takes all (or shares it with its equals) to an even distribution, with masked and lowest logits."""
    z, y = batch(T, V, TYPES[t], 7, masked=0.01)
    z[0] = -3.3e38
    z[1, : V // 2] = -3.3e38
    if temp < 1:
        z[2, 5], z[2, V - 2] = 40.0, 40.0
    x = padded(z, 1)
    exact = torch.tensor(temp, dtype=torch.float32).double().item()
    ids, tops, lp, H = run(lib, x, 20, temp, y)
    want, (wt, bt), (wl, bl), (wh, bh) = R.top(z, 20, exact, y)
    assert torch.equal(ids.cpu().long(), want)
    # a log-probability past float32's range is -inf; 1 / temperature is rounded once more
    over = lambda v: torch.where(v < -torch.finfo(torch.float32).max, -math.inf, v)  # noqa: E731
    more = 2 * R.EPS24
    R.near(tops, over(wt), bt + more * wt.abs().nan_to_num(0, 0, 0), torch.float32, "log-probabilities")
    R.near(lp, over(wl), bl + more * wl.abs().nan_to_num(0, 0, 0), torch.float32, "targets'")
    R.near(H, wh, bh + more, torch.float32, "entropies")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(300, 70_001), (3, 131_072)])
def test_masks_that_begin_late(lib, t, T, V):
    """Masked and lowest words in the first, a later or the last of a row's batches alone, and in one thread's vector."""
    z, y = batch(T, V, TYPES[t], 11)
    third = V // 3
    for r in range(T):
        low = -math.inf if r % 2 else -3.3e38
        part = (slice(0, third), slice(third, 2 * third), slice(2 * third, V), slice(V - 5, V - 4), slice(V // 2, V // 2 + 8))[r % 5]
        z[r, part] = low
    exact = torch.tensor(0.9, dtype=torch.float32).double().item()
    ids, tops, lp, H = run(lib, padded(z, 0), 20, 0.9, y)
    want, (wt, bt), (wl, bl), (wh, bh) = R.top(z, 20, exact, y)
    assert torch.equal(ids.cpu().long(), want)
    # -3.3e38 / 0.9 = -3.67e38 rounds to -inf: it is more than half a step past -3.4028e38
    wl = torch.where(wl < -torch.finfo(torch.float32).max, -math.inf, wl)
    R.near(tops, wt, bt, torch.float32, "log-probabilities")
    R.near(lp, wl, bl, torch.float32, "targets'")
    R.near(H, wh, bh, torch.float32, "entropies")


def test_rows_past_32_bits(lib):
    """Rows that start past 2^31 elements."""
    T, V = 17_000, 130_001
    x = torch.empty((T, V), device=DEV, dtype=torch.bfloat16).normal_(generator=torch.Generator(DEV).manual_seed(3))
    at = torch.tensor([0, 1, 16_518, 16_519, 16_999])
    ids, tops, _, _ = run(lib, x, 8, 1.0)
    want, (wt, bt), _, _ = R.top(x[at.to(DEV)].cpu(), 8, 1.0)
    assert torch.equal(ids[at.to(DEV)].cpu().long(), want)
    R.near(tops[at.to(DEV)], wt, bt, torch.float32, "log-probabilities")


def test_no_rows(lib):
    e = torch.empty((0, 10), device=DEV)
    lib.top_logprobs(e, torch.empty((0, 3), dtype=torch.int32, device=DEV), torch.empty((0, 3), device=DEV))
