"""Masks of the type's lowest value at very high temperatures: a masked word's probability is 0 there too."""

import pytest
import torch

from tests import _ops_ref as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("temp", [1.0, 1e20, 1e24, 1e30])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(3, 50), (3, 5000), (3, 50_000), (200, 5000), (200, 30_000)])
def test_masked_words(t, T, V, temp):
    from paper_2605_20863_amd import _lib

    g = torch.Generator().manual_seed(V)
    z = torch.randn((T, V), generator=g) * min(temp, 1e6)
    y = torch.randint(0, V, (T,), generator=g)
    masked = torch.rand((T, V), generator=g) < 0.3
    masked[:, : V // 2] = True  # whole parts and threads of nothing else
    masked[torch.arange(T), y] = False
    z[masked] = torch.finfo(t).min
    z = z.to(t)
    lp, H, out, stats = (torch.empty(n, device=DEV) for n in (T, T, T, 8))
    grad = torch.empty((T, V), dtype=t, device=DEV)
    _lib.token_logprobs(z.to(DEV), y.to(DEV), lp, H, temperature=temp)
    _, _, want, ent, bl, bh = R.row_quantities(z, y, torch.tensor(temp, dtype=torch.float32).double().item())
    for got, w, b in ((lp, want, bl), (H, ent, bh)):
        assert ((got.cpu().double() - w).abs() <= b + R.EPS24 * w.abs()).all(), (got, w)
    one = torch.ones(T, device=DEV)
    _lib.policy_loss(z.to(DEV), y.to(DEV), lp, one, one, stats, grad, out, temperature=temp, grad_scale=temp)
    assert ((out.cpu().double() - want).abs() <= bl + R.EPS24 * want.abs()).all()
    assert (grad.cpu()[masked] == 0).all() and grad.isfinite().all()
