"""64-bit references of the operators of include/pda_lm.h, on the CPU, from their
definitions, with the error bounds that float32 arithmetic and one rounding of
each result give them."""

import math

import torch

from tests._ops_ref import E4M3_MAX, EPS24, HALF, MIN_SCALE

# Half a step of an e4m3 code, relative (3 fraction bits) and among the smallest codes (a step is 2^-9).
E4M3_HALF, E4M3_LEAST = 2.0 ** -4, 2.0 ** -10
# A row's sum of squares: 8 in a vector, up to 4 vectors of a thread, 6 joins of lanes and 16 of waves, halved by the
# root; the mean, its root, the reciprocal and two products: 17 + 6.
NORM = 24 * EPS24


def norm(h, w, eps):
    """y in float64, and its bound before rounding."""
    h = h.double()
    y = h * w.double() / torch.sqrt((h * h).mean(dim=1, keepdim=True) + eps)
    return y, NORM * y.abs()


def fp8(y, bound, group):
    """(scales, their bound, y / scale, its bound) by groups of a row's neighbours."""
    T, H = y.shape
    parts = y.view(T, -1, group or H)
    s = (parts.abs().amax(dim=2) / E4M3_MAX).clamp(min=MIN_SCALE)
    z = (parts / s[:, :, None]).view(T, H)
    ds = (NORM + 2 * EPS24) * s
    # the quotient's: y's, the scale's, its own rounding; then to a code
    arith = (2 * NORM + 4 * EPS24) * z.abs()
    return s, ds, z, arith + torch.maximum(E4M3_HALF * (z.abs() + arith), torch.full_like(z, E4M3_LEAST))


def norm_grad(h, w, g, q, eps):
    """(dh, bound, dw, bound)."""
    h, g, w = h.double(), g.double(), w.double()
    r = 1 / torch.sqrt((h * h).mean(dim=1, keepdim=True) + eps)
    y, gw = h * r, g * w
    dh = r * (gw - y * (gw * y).mean(dim=1, keepdim=True))
    size = r * (gw.abs() + y.abs() * (gw * y).abs().mean(dim=1, keepdim=True))
    if q is not None:
        dh, size = dh + q.double(), size + q.double().abs()
    terms = g * y
    # a term: as y; its sums: in a thread and over a workgroup's rows, below 24 here
    return dh, 3 * NORM * size, terms.sum(dim=0), (NORM + 32 * EPS24) * terms.abs().sum(dim=0)


def rows(logits, temperature):
    """Per row: x = l - max scaled, log p, log of the sum, the bound on that of float32 sums without its word's own."""
    z = logits.double() / temperature
    x = z - z.amax(dim=1, keepdim=True)
    e = x.exp()
    s = e.sum(dim=1, keepdim=True)
    lse = s.log()
    p = e / s
    mean = (p * torch.where(e > 0, x, 0.0).abs()).sum(dim=1, keepdim=True)
    # an exponential is off by 3 roundings of x, the sum by one for each of a thread's elements (of 256) and the joins
    depth = logits.shape[1] / 256 + 40
    return x, x - lse, lse, p, EPS24 * (depth + 6 * (2 + mean) + 4 * lse.abs()), mean


def top(logits, K, temperature, targets=None):
    """ids, (log-probabilities, bound), (the targets', bound), (entropies, bound)."""
    T, V = logits.shape
    x, logp, lse, p, base, mean = rows(logits, temperature)
    order = torch.sort(logits.float() + 0.0, dim=1, descending=True, stable=True).indices[:, :K]
    best, far = logp.gather(1, order), x.gather(1, order).abs()
    ids, tops, bounds = torch.full((T, K), -1), torch.full((T, K), -math.inf, dtype=torch.float64), torch.zeros((T, K)).double()
    n = order.shape[1]
    live = torch.ones((T, 1), dtype=torch.bool) if targets is None else (targets >= 0)[:, None]
    here = live & (logits.gather(1, order) > -math.inf)
    ids[:, :n] = torch.where(here, order, -1)
    tops[:, :n] = torch.where(here, best, -math.inf)
    bounds[:, :n] = torch.where(here, base + 4 * EPS24 * far, 0.0)
    H = -(p * torch.where(p > 0, logp, 0.0)).sum(dim=1)
    H, hb = torch.where(live[:, 0], H, 0.0), (2 * base * (1 + mean) + EPS24 * 8 * mean)[:, 0]
    lp = lb = None
    if targets is not None:
        y = targets.long().clamp(min=0)[:, None]
        lp = torch.where(live, logp.gather(1, y), 0.0)[:, 0]
        lb = (base + 4 * EPS24 * torch.where(lp.isfinite()[:, None], x.gather(1, y).abs(), 0.0))[:, 0]
    return ids, (tops, bounds), (lp, lb), (H, hb)


def distill(logits, ids, tau, w, b, rest, temperature, scale):
    """dict of losses, terms [T, 6], dlogits and their bounds. Divergences and gradients from their definitions, word by
    word (a word of a second place counts once)."""
    T, V = logits.shape
    x, logp, lse, p, base, _ = rows(logits, temperature)
    teacher = torch.full((T, V), math.nan, dtype=torch.float64)
    for t in range(T):
        for i, v in reversed(list(zip(ids[t].tolist(), tau[t].tolist()))):
            if 0 <= i < V and v != -math.inf:
                teacher[t, i] = v
    inside = ~teacher.isnan()
    err = base + 4 * EPS24 * torch.where(p > 0, x, 0.0).abs()  # of log p
    a = torch.where(inside, logp - teacher, 0.0)
    t = torch.where(inside, teacher.exp(), 0.0)
    zero = lambda m, v: torch.where(m, v, 0.0)  # noqa: E731
    S, P = t.sum(dim=1, keepdim=True), zero(inside, p).sum(dim=1, keepdim=True)
    ta, pa = zero(t > 0, t * a), zero(inside & (p > 0), p * a)
    F, R = -ta.sum(dim=1, keepdim=True), pa.sum(dim=1, keepdim=True)
    each = 16 * EPS24
    # a term's error: its slope in log p times that one's, and roundings of its size
    dF = (t * err + each * (ta.abs() + t + p * inside)).nan_to_num(0.0, 0.0, 0.0).sum(dim=1, keepdim=True)
    dR = zero(inside, p * (err * (1 + a.abs()) + each * (1 + a.abs()))).nan_to_num(0.0).sum(dim=1, keepdim=True) + each * S
    if rest:
        others = torch.where(inside, -math.inf, x).logsumexp(dim=1, keepdim=True) - lse
        some = others > -math.inf
        tr = zero(some, (1 - S).clamp(min=2.0 ** -24))
        ar = zero(some, others - tr.log())
        pr = others.exp()
        F, R = F - tr * ar, R + pr * ar
        top_of = zero(some, torch.where(inside, -math.inf, x).amax(dim=1, keepdim=True)).abs()
        er = 2 * base + 4 * EPS24 * top_of
        dF = dF + (tr + pr) * er + each * (tr + pr + (tr * ar).abs() + 1)
        dR = dR + pr * (1 + ar.abs()) * er + each * (pr * (1 + ar.abs()) + tr + 1)
        share = torch.where(inside | (p == 0), 0.0, p / pr)
        gF = p * (S + tr) - t - share * tr
        gR = p * (torch.where(inside, a, ar) - R)
        sizeF = p * (S + tr) + t + share * tr
        sizeR = p * (torch.where(inside, a, ar).abs().nan_to_num(0.0, 0.0, 0.0) + R.abs() + 2)
        err = err + torch.where(inside, 0.0, er)
    else:
        gF = p * S - t
        gR = zero(inside, p * (a + 1)) - p * (R + P)
        sizeF = p * S + t
        sizeR = p * (a.abs().nan_to_num(0.0, 0.0, 0.0) + R.abs() + P + 3)
    gR = torch.where(p > 0, gR, 0.0)
    far = torch.where(p > 0, logp, 0.0).abs()
    grad = (1 - b) * gF + b * gR
    bound = ((1 - b) * sizeF + b * sizeR) * (2 * err + EPS24 * 8 * (far + 4)) + b * p * dR
    none = ~(p.sum(dim=1, keepdim=True) > 0)  # -inf alone
    F, R, P = torch.where(none, torch.where(S > 0, math.inf, 0.0), F), torch.where(none, 0.0, R), torch.where(none, 0.0, P)
    dF, dR, base = (torch.where(none, 0.0, v) for v in (dF, dR, base))  # these are exact
    loss = (0.0 if b == 1 else (1 - b) * F) + (0.0 if b == 0 else b * R)
    k = (w.double() * scale / temperature)[:, None]
    flat = (k != 0) & ~none
    dloss = ((0.0 if b == 1 else (1 - b) * dF) + (0.0 if b == 0 else b * dR) + each * torch.where(loss.isfinite(), loss, 0.0).abs())
    return dict(losses=loss[:, 0], loss_bound=dloss[:, 0] + 0 * loss[:, 0].nan_to_num(0.0, 0.0, 0.0),
                terms=torch.cat([loss, F, R, S, P, torch.ones_like(F)], dim=1),
                term_bounds=torch.cat([dloss, dF, dR, each * S, base + each * P, torch.zeros_like(F)], dim=1),
                dlogits=torch.where(flat, grad * k, 0.0), grad_bound=torch.where(flat, bound * k.abs(), 0.0))


def near(got, want, bound, dtype, what):
    """|got - want| within the arithmetic's bound and one rounding to dtype, and the same where want is not finite."""
    got = got.detach().cpu().double()
    finite = want.isfinite()
    same = (got == want) | (got.isnan() & want.isnan())
    assert same[~finite].all(), f"{what}: {got[~finite & ~same][:4]} for {want[~finite & ~same][:4]}"
    limit = bound + HALF[dtype] * 1.01 * (want.abs() + bound) + 1e-37
    over = torch.where(finite, (got - want).abs() - limit, -1.0)
    over = torch.where(finite & got.isnan(), math.inf, over)
    worst = int(over.argmax()) if over.numel() else 0
    assert (over <= 0).all(), f"{what}: {got.reshape(-1)[worst]} for {want.reshape(-1)[worst]}, over by {float(over.max()):.3g}"
