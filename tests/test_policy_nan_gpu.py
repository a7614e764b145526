"""A logit that is NaN shows in every sum over its row's terms, unless the row's weight is 0."""

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("T,V", [(3, 1000), (40, 1000), (3, 40_000), (200, 40_000)])
def test_nan_shows_in_the_sums(T, V):
    from paper_2605_20863_amd import _lib

    g = torch.Generator().manual_seed(T)
    z = torch.randn((T, V), generator=g).to(DEV)
    y = (torch.arange(T) % V).to(DEV)
    z[1, (T + 5) % V] = float("nan")
    old, ref, w = torch.full((T,), -7.0, device=DEV), torch.full((T,), -7.0, device=DEV), torch.full((T,), 1 / T, device=DEV)
    adv, stats = torch.ones(T, device=DEV), torch.zeros(8, device=DEV)
    named = lambda: dict(zip(_lib.POLICY_STATS, stats.tolist()))  # noqa: E731
    _lib.policy_loss(z, y, old, adv, w, stats, ref_logprobs=ref, kl_coef=0.1)
    assert all(v != v for k, v in named().items() if k in ("loss", "policy", "kl", "entropy", "ratio", "old_kl"))
    assert abs(named()["weight"] - 1) < 1e-5
    w[1] = 0
    _lib.policy_loss(z, y, old, adv, w, stats, ref_logprobs=ref, kl_coef=0.1)
    assert all(v == v for v in named().values())
