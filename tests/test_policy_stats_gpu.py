"""What the policy loss's seventh sum, e^-d - 1 + d, is the mean of: over every word of a small vocabulary, weighted with
the probability that either policy draws it."""

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("V", [7, 900])
def test_distance_from_the_rollouts_policy(V):
    from paper_2605_20863_amd import _lib

    g = torch.Generator().manual_seed(V)
    z = torch.randn(V, generator=g)
    logp, logq = torch.log_softmax(z.double(), 0), torch.log_softmax(z.double() + 0.5 * torch.randn(V, generator=g), 0)
    p, q = logp.exp(), logq.exp()
    kl = (p * (logp - logq)).sum()
    chi2, back = (q * q / p).sum() - 1, (q * (logq - logp)).sum()
    stats, y, zero = torch.empty(8, device=DEV), torch.arange(V, device=DEV), torch.zeros(V, device=DEV)
    for w, want in ((p, kl), (q, chi2 - back)):
        _lib.policy_loss(z.expand(V, V).contiguous().to(DEV), y, logq.float().to(DEV), zero, w.float().to(DEV), stats)
        # a term of size 1 to a few, off by some roundings of the log-probabilities' 2 to 10
        assert abs(float(stats[_lib.POLICY_STATS.index("old_kl")]) - float(want)) < 1e-5 * (1 + float(want))
        assert abs(float(stats[7]) - 1) < 1e-5
