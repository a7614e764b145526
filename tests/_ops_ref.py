"""64-bit references of the operators around attention (include/pda_ops.h), on
the CPU, from their definitions, with the error bounds that float32 arithmetic
and one rounding of each result give them."""

import numpy as np
import torch

E4M3_MAX, MIN_SCALE = 448.0, 2.0 ** -126
EPS24 = 2.0 ** -24  # float32: half the distance from 1 to the next number
HALF = {torch.float32: EPS24, torch.bfloat16: 2.0 ** -8}  # relative error of one rounding (24 and 8 significant bits)


def angles(positions, rot, base=1e4):
    """cos_sin table [positions, rot] float32."""
    inv = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * inv
    return torch.cat([a.cos(), a.sin()], dim=1).float()


def pairs(rot, interleaved):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def turn(x, table, positions, interleaved, back=False):
    """x [T, H, D] float64 with its first dims turned by the table's rows."""
    rot = table.shape[1]
    i, j = pairs(rot, interleaved)
    c, s = table.double()[positions.long()][:, None].chunk(2, dim=-1)
    s = -s if back else s
    y = x.clone()
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y


def rms(x, eps):
    return 1.0 / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + eps)


def norm_turn(x, w, table, positions, eps, interleaved):
    """(result, bound on the error of float32 arithmetic) of norm and rotation."""
    n = x.double()
    if w is not None:
        n = n * rms(n, eps) * w.double()
    # the norm: 12 roundings of the sum of squares (8 in a lane, 4 joins), halved by
    # the root, its own, two products; the rotation: 3 on |n_i c| + |n_j s|
    bound = 16 * EPS24 * 2 * n.abs().amax(dim=-1, keepdim=True)
    return turn(n, table, positions, interleaved), bound


def norm_turn_grad(x, w, table, positions, grad, eps, interleaved):
    """(dx, bound, dw, bound) of norm and rotation."""
    g = turn(grad.double(), table, positions, interleaved, back=True)
    top = g.abs().amax(dim=-1, keepdim=True)
    if w is None:
        return g, 8 * EPS24 * 2 * top, None, None
    x = x.double()
    r = rms(x, eps)
    y = x * r
    terms = g * y
    dw = terms.sum(dim=(0, 1))
    # a term: 16 roundings; its sum in a lane, over lanes, waves and workgroups: under 48 here
    dw_bound = 64 * EPS24 * (top * y.abs()).sum(dim=(0, 1))
    gw = g * w.double()
    dx = r * (gw - y * (gw * y).mean(dim=-1, keepdim=True))
    most = (gw.abs().amax(dim=-1, keepdim=True) + top * w.double().abs().max())
    return dx, 32 * EPS24 * r * most * (1 + y.abs()), dw, dw_bound


def assert_within(got, want, bound, dtype, what):
    """|got - want| within the arithmetic's bound and one rounding to dtype."""
    got = got.detach().cpu().double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    limit = bound + HALF[dtype] * 1.01 * (want.abs() + bound) + 1e-37
    over = (got - want).abs() - limit
    worst = int(over.argmax())
    assert (over <= 0).all(), (f"{what}: {got.reshape(-1)[worst]} for {want.reshape(-1)[worst]}, "
                               f"over by {float(over.max()):.3g}")


# ------------------------------------------------------------- cache


def encode(x, scale):
    """E4M3 codes of float32 x / scale, rounded once, clamped, to nearest even."""
    z = np.clip((x.astype(np.float32) / np.float32(scale)).astype(np.float32), -448.0, 448.0)
    return torch.from_numpy(np.ascontiguousarray(z)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def decode(codes):
    return torch.from_numpy(np.ascontiguousarray(codes)).view(torch.float8_e4m3fn).float().numpy()


def places(offsets, lens, num_tokens, table_width):
    """(sequence, position) of every packed token, in order; offsets None: equal counts."""
    B = len(lens)
    if offsets is None:
        offsets = np.arange(B + 1) * (num_tokens // max(B, 1))
    out = []
    for b in range(B):
        n = offsets[b + 1] - offsets[b]
        length = min(max(lens[b], 0), 16 * table_width)
        out += [(offsets[b] + i, b, length - n + i) for i in range(n)]
    return out


def write_fp8_tile(tile, scale, new, slots, is_v):
    """One fp8 tile [16, D] (rows of slots) and its scale after the new float32 rows
    went to `slots` (ascending): tile, scale."""
    first = slots[0]
    amax = np.float32(max(np.abs(new).max(), 0))
    s = np.float32(scale)
    if first == 0 or not s > 0 or amax > np.float32(E4M3_MAX) * s:
        old, s = s, np.float32(max(amax / np.float32(E4M3_MAX), np.float32(MIN_SCALE)))
        if first > 0:
            back = (decode(tile[:first]) * old).astype(np.float32)
            tile[:first] = encode(back, s)
    tile[slots] = encode(new, s)
    return tile, s


# ------------------------------------------------------------- logits


def row_quantities(logits, targets, temperature):
    """Per live row: log p [V], lp, H, bounds on lp and H, in float64."""
    z = logits.double() / temperature
    m = z.amax(dim=1, keepdim=True)
    x = z - m
    e = x.exp()
    s = e.sum(dim=1)
    lse = s.log()
    p = e / s[:, None]
    xs = torch.where(e > 0, x, 0.0)
    mean = (p * xs.abs()).sum(dim=1)
    logp = x - lse[:, None]
    lp = logp.gather(1, targets.long().clamp(min=0)[:, None])[:, 0]
    H = -(p * torch.where(e > 0, logp, 0.0)).sum(dim=1)
    # an exponent is off by 3 roundings of x, the sum by one for each of a thread's
    # elements (of 256 threads) and the joins
    depth = logits.shape[1] / 256 + 40
    bound = EPS24 * (depth + 6 * (2 + mean) + 4 * lse.abs() + 4 * torch.where(lp.isfinite(), (lp + lse).abs(), 0.0))
    return logp, p, lp, H, bound, 2 * bound * (1 + mean) + EPS24 * 8 * mean


def policy(logits, targets, old, ref, adv, w, temperature, low, high, dual, kl_coef, ent_coef, grad_scale):
    """dict of stats, dlogits, logprobs, entropy and bounds, in float64."""
    T, V = logits.shape
    live = targets >= 0
    logp, p, lp, H, bl, bh = row_quantities(logits, targets, temperature)
    lp, H = torch.where(live, lp, 0.0), torch.where(live, H, 0.0)
    old, adv, w = old.double(), adv.double(), w.double()
    w = torch.where(live, w, 0.0)
    x = lp - old
    d = x.clamp(-20, 20)
    r = d.exp()
    plain, cut = -adv * r, -adv * r.clamp(1 - low, 1 + high)
    held = cut > plain
    pg = torch.maximum(plain, cut)
    if dual:
        top = (adv < 0) & (pg > -adv * dual)
        pg, held = torch.where(top, -adv * dual, pg), held | top
    g = torch.where(held | (x.abs() > 20), 0.0, plain)
    kl = torch.zeros_like(lp)
    if ref is not None:
        y = ref.double() - lp
        u = y.clamp(-20, 20)
        kl = u.exp() - 1 - u
        g = g + kl_coef * torch.where(y.abs() > 20, 0.0, 1 - u.exp())
    loss = pg + kl_coef * kl - ent_coef * H
    terms = torch.stack([loss, pg, kl, H, held.double(), r, (-d).exp() - 1 + d, torch.ones_like(lp)])
    stats = torch.where(w != 0, terms * w, 0.0).sum(dim=1)
    slope = p * (ent_coef * (logp + H[:, None])).nan_to_num(0.0, 0.0, 0.0)
    grad = slope - p * g[:, None]
    grad[torch.arange(T), targets.long().clamp(min=0)] += g
    k = (w * grad_scale / temperature)[:, None]
    size = p * (g.abs()[:, None] + ent_coef * ((logp + H[:, None]).abs().nan_to_num(0.0, 0.0, 0.0) + 1))
    size[torch.arange(T), targets.long().clamp(min=0)] += g.abs()
    # an element's exponent, twice the row's own bounds; g follows lp with slope |plain| + kl_coef e^u
    steep = plain.abs() + (kl_coef * torch.exp((ref.double() - lp).clamp(-20, 20)) if ref is not None else 0.0)
    x = torch.where(p > 0, logp, 0.0).abs()
    bound = size * (EPS24 * 8 * (x + 4) + 2 * (bl + bh)[:, None]) + (p + 1e-30) * (steep * (bl + 16 * EPS24))[:, None]
    bound[torch.arange(T), targets.long().clamp(min=0)] += steep * (bl + 16 * EPS24)
    return dict(stats=stats, dlogits=torch.where(k != 0, grad * k, 0.0), logprobs=lp, entropy=H, lp_bound=bl, h_bound=bh,
                grad_bound=torch.where(k != 0, bound * k.abs(), 0.0), terms=terms, weights=w, steep=steep)
