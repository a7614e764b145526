"""Timed cases of the operators around attention in a rollout, log-prob and update program.

A case is one pass through one of the operators:

    append    head norms and rotation of new queries and keys, keys and values written into the paged cache:
              a decode step (chunk 1), speculative verification (a few tokens a sequence), chunked prefill, or
              every token of every sequence (chunk 0, the log-prob forward)
    rope      the same norms and rotation without a cache, as a training forward makes them
    rope_bwd  its gradient: of the queries, the keys and both weights
    logp      log-probabilities of given tokens, and entropies, from logits
    policy    the clipped policy loss with its KL and entropy terms, and its gradient at the logits

With ``own`` false the operators run in their plain form, elementary torch operations in 32 bits; with ``own`` true
through ``paper_2605_20863_amd._lib``. Lengths depend on the case alone (its ``lseed``), so that every seed is
the same work; tensors and block tables come from the seed.
"""

import math

import numpy as np
import torch

own = False

BS = 16  # tokens per cache block
DEV = "cuda"
EPS = 1e-6
FP8_MAX, MIN_SCALE = 448.0, 2.0 ** -126
CLAMP = 20.0  # bound on log ratios
IGNORED = -100  # target of a token that takes no part
CLIP_LOW, CLIP_HIGH, DUAL = 0.2, 0.28, 3.0
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


def _append(name, B, hq, hkv, d, kv, median, sigma, lo, hi, chunk, **more):
    return dict(name=name, op="append", B=B, hq=hq, hkv=hkv, d=d, kv=kv, median=median, sigma=sigma, lo=lo, hi=hi,
                chunk=chunk, **_rope(d, more))


def _rope(d, more):
    return dict(dict(rot=d, inter=False, norm=True, lseed=1), **more)


def _train(name, op, T, hq, hkv, d, t, **more):
    return dict(name=name, op=op, T=T, hq=hq, hkv=hkv, d=d, t=t, **_rope(d, more))


def _head(name, op, T, V, t, **more):
    return dict(dict(name=name, op=op, T=T, V=V, t=t, pad=0, temp=1.0, lseed=1), **more)


def listed():
    return [
        # a few interactive chats, one new token each: launches and latency count
        _append("append_chat_bf16", 3, 32, 4, 128, "bf16", 700, 0.6, 64, 2048, 1),
        # one decode step of a large batch over an fp8 cache
        _append("append_decode_fp8", 512, 64, 8, 128, "fp8", 8192, 0.9, 128, 65536, 1),
        # chunked prefill of a 7B-class batch: 512 tokens a sequence, rotation without norms
        _append("append_chunk_bf16", 64, 28, 4, 128, "bf16", 2048, 0.8, 64, 16384, 512, norm=False),
        # the log-prob forward: every token of 64 rollouts
        _append("append_logprob_bf16", 64, 32, 4, 128, "bf16", 2048, 0.8, 64, 16384, 0),
        # a training micro-batch of 16k packed tokens
        _train("rope_train_bf16", "rope", 16384, 64, 4, 128, "bf16"),
        # a small float32 model, odd token count, half of each head rotated in interleaved pairs
        _train("rope_small_f32", "rope", 777, 4, 4, 64, "f32", rot=32, inter=True),
        _train("rope_bwd_train_bf16", "rope_bwd", 16384, 32, 4, 128, "bf16"),
        _train("rope_bwd_small_f32", "rope_bwd", 777, 4, 4, 64, "f32", rot=32, inter=True),
        # the sampled tokens of one decode step
        _head("logp_decode_bf16", "logp", 64, 131072, "bf16", temp=0.7),
        # the log-prob forward of a micro-batch
        _head("logp_forward_bf16", "logp", 8192, 131072, "bf16"),
        # one update micro-batch: loss and gradient over a large vocabulary
        _head("policy_bf16", "policy", 4096, 131072, "bf16", kl=0.04, ent=0.001),
        # a short odd batch in float32, odd vocabulary in padded rows
        _head("policy_small_f32", "policy", 37, 50001, "f32", pad=7, kl=0.1, ent=0.01, temp=0.9),
    ]


HEADS = [(28, 4, 128), (32, 4, 128), (64, 4, 128), (32, 8, 128), (64, 8, 128), (8, 1, 128), (16, 4, 64)]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "append", "rope", "rope_bwd", "logp", "policy", "policy"])
    lseed = rng.randrange(2, 1 << 30)
    if op in ("logp", "policy"):
        t = rng.choice(["bf16", "bf16", "f32"])
        V = _logint(rng, 1000, 200000)
        T = _logint(rng, 1, max(2, min(8192, 1.0e9 / (V * (4 if t == "f32" else 2)))))
        c = _head("", op, T, V, t, pad=rng.choice([0, 0, rng.randint(1, 64)]), temp=rng.choice([1.0, 1.0, 0.7, 1.3]),
                  lseed=lseed)
        if op == "policy":
            c.update(kl=rng.choice([0.0, 0.01, 0.1]), ent=rng.choice([0.0, 0.001, 0.01]))
        return _pure(c)
    hq, hkv, d = rng.choice(HEADS)
    more = dict(lseed=lseed, norm=rng.random() < 0.7, inter=rng.random() < 0.25, rot=rng.choice([d, d, d // 2]))
    if op != "append":
        t = rng.choice(["bf16", "bf16", "f32"])
        T = _logint(rng, 1, 12000)
        return _pure(_train("", op, T, hq, hkv, d, t, **more))
    kv = rng.choice(["bf16", "bf16", "fp8", "f32"])
    sigma = round(rng.uniform(0.2, 0.9), 2)
    chunk = rng.choice([1, 1, 1, rng.randint(2, 4), 0, _logint(rng, 8, 2048), _logint(rng, 8, 2048)])
    B = _logint(rng, 1, 512 if 0 < chunk <= 4 else 64)
    most = 16384 if chunk else max(64, min(8192, 50000 // B))
    median = _logint(rng, 48, most)
    if chunk:
        chunk = min(chunk, max(1, 50000 // B))
    return _pure(_append("", B, hq, hkv, d, kv, median, sigma, 4, min(65536, 4 * median), chunk, **more))


def _pure(c):
    del c["name"]
    return c


# ------------------------------------------------------------------ sizes


def _lengths(c):
    """(sequence lengths after the append, new tokens of each)."""
    rng = np.random.default_rng(c["lseed"])
    x = np.exp(rng.normal(math.log(c["median"]), c["sigma"], size=c["B"]))
    L = np.clip(np.rint(x), c["lo"], c["hi"]).astype(np.int64)
    return L, L if c["chunk"] == 0 else np.minimum(L, c["chunk"])


def _esz(t):
    return {"f32": 4, "bf16": 2, "fp8": 1}[t]


def _in_type(c):
    return "f32" if c["kv"] == "f32" else "bf16"


def work(c):
    """Every input read once, every output written once; of a table the rows in use, each once."""
    if c["op"] in ("logp", "policy"):
        T, V, e = c["T"], c["V"], _esz(c["t"])
        if c["op"] == "logp":
            return {"bytes": T * (V * e + 8 + 8), "flops": 6.0 * T * V}
        return {"bytes": T * (2 * V * e + 8 + 4 * 4 + 8) + 32, "flops": 12.0 * T * V}
    hq, hkv, d, rot = c["hq"], c["hkv"], c["d"], c["rot"]
    if c["op"] == "append":
        L, n = _lengths(c)
        T, e = int(n.sum()), _esz(_in_type(c))
        rows = len(np.unique(np.concatenate([np.arange(a - b, a) for a, b in zip(L, n)])))
        tiles = int(((L + BS - 1) // BS - (L - n) // BS).sum())
        byt = T * ((2 * hq + 2 * hkv) * d * e + 2 * hkv * d * _esz(c["kv"])) + rows * rot * 4 + tiles * 4 + 8 * c["B"]
        if c["kv"] == "fp8":
            byt += 2 * tiles * hkv * 4
        return {"bytes": byt, "flops": T * (hq + hkv) * (3.0 * rot + (4 * d if c["norm"] else 0))}
    T, e = c["T"], _esz(c["t"])
    rows = T * (hq + hkv)
    byt = (2 if c["op"] == "rope" else 3) * rows * d * e + T * (4 + rot * 4)
    return {"bytes": byt, "flops": rows * (3.0 * rot + (12 * d if c["norm"] else 0))}


# ------------------------------------------------------------------ inputs


def _gen(seed, *key):
    s = np.random.SeedSequence(entropy=int(seed), spawn_key=key).generate_state(1, dtype=np.uint64)[0]
    return torch.Generator(device=DEV).manual_seed(int(s & np.uint64((1 << 62) - 1)))


def _randn(shape, dtype, gen, amp=1.0):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).mul_(amp).to(dtype)


def _rand(shape, gen):
    return torch.rand(shape, generator=gen, device=DEV, dtype=torch.float32)


def _table(positions, rot):
    """Cosines and sines of every position's angles: [positions, rot] float32, cosines first."""
    inv = 1e6 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    a = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * inv
    return torch.cat([a.cos(), a.sin()], dim=1).to(torch.float32)


def _weights(c, dt, seed):
    if not c["norm"]:
        return None, None
    return tuple((1.0 + 0.2 * _randn((c["d"],), torch.float32, _gen(seed, k))).to(dt) for k in (10, 11))


def prepare(c, seed):
    if c["op"] in ("logp", "policy"):
        return _prepare_head(c, seed)
    if c["op"] == "append":
        return _prepare_append(c, seed)
    T, hq, hkv, d, dt = c["T"], c["hq"], c["hkv"], c["d"], TYPES[c["t"]]
    # one projection's output, and the gradient's place in its own packed rows
    qkv = _randn((T, (hq + 2 * hkv) * d), dt, _gen(seed, 1))
    s = dict(case=c, **_views(qkv, hq, hkv, d))
    s["wq"], s["wk"] = _weights(c, dt, seed)
    # several packed sequences, positions counted from each one's start
    n = max(1, T // 5)
    s["positions"] = (torch.arange(T, device=DEV) % n).to(torch.int32)
    s["table"] = _table(n, c["rot"])
    if c["op"] == "rope":
        s["q_out"], s["k_out"] = (torch.empty((T, h, d), dtype=dt, device=DEV) for h in (hq, hkv))
        return s
    s["gq"], s["gk"] = (_randn((T, h, d), dt, _gen(seed, k), 1e-2) for k, h in ((2, hq), (3, hkv)))
    g = _views(torch.empty_like(qkv), hq, hkv, d)
    s["dq"], s["dk"] = g["q"], g["k"]
    s["dwq"], s["dwk"] = (torch.empty(d, dtype=torch.float32, device=DEV) if c["norm"] else None for _ in "qk")
    return s


def _views(qkv, hq, hkv, d):
    T = qkv.shape[0]
    x = qkv.view(T, hq + 2 * hkv, d)
    return dict(q=x[:, :hq], k=x[:, hq:hq + hkv], v=x[:, hq + hkv:])


def _prepare_append(c, seed):
    B, hq, hkv, d, kv = c["B"], c["hq"], c["hkv"], c["d"], c["kv"]
    L, n = _lengths(c)
    dt, T = TYPES[_in_type(c)], int(n.sum())
    # only the blocks that the new tokens touch exist; the tables are as wide as the longest sequence
    first, last = (L - n) // BS, (L + BS - 1) // BS
    count = last - first
    nb = int(count.sum()) + 3
    perm = np.random.default_rng(seed).permutation(nb)
    table = np.full((B, int(last.max())), -1, dtype=np.int32)
    rows = np.repeat(np.arange(B), count)
    cols = np.arange(count.sum()) - np.repeat(np.cumsum(count) - count, count) + np.repeat(first, count)
    table[rows, cols] = perm[: len(rows)]
    s = dict(case=c, T=T, lens=torch.from_numpy(L.astype(np.int32)).to(DEV), block_table=torch.from_numpy(table).to(DEV))
    even = bool((n == n[0]).all())
    s["offsets"] = None if even else torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).to(DEV)
    new = _views(_randn((T, (hq + 2 * hkv) * d), dt, _gen(seed, 1)), hq, hkv, d)
    s["q"], s["new_k"], s["new_v"] = new["q"], new["k"], new["v"]
    s["wq"], s["wk"] = _weights(c, dt, seed)
    s["table"] = _table(int(L.max()), c["rot"])
    s["q_out"] = torch.empty((T, hq, d), dtype=dt, device=DEV)
    s["scales"] = None
    shape = (nb, hkv, BS, d), (nb, hkv, d, BS)
    if kv == "fp8":
        # earlier tokens' codes with their tiles' scales; half of the new tokens' tiles need larger ones
        s["k"], s["v"] = ((_rand(x, _gen(seed, i)) * 896 - 448).to(TYPES["fp8"]) for i, x in zip((2, 3), shape))
        s["scales"] = (0.004 + 0.004 * _rand((2, nb, hkv), _gen(seed, 4)))
    else:
        s["k"], s["v"] = (_randn(x, TYPES[kv], _gen(seed, i)) for i, x in zip((2, 3), shape))
    return s


def _prepare_head(c, seed):
    T, V, dt = c["T"], c["V"], TYPES[c["t"]]
    logits = torch.randn((T, V + c["pad"]), generator=_gen(seed, 1), device=DEV, dtype=dt)[:, :V]
    logits.mul_(2.0)
    target = torch.randint(0, V, (T,), generator=_gen(seed, 2), device=DEV)
    rows = torch.arange(T, device=DEV)
    logits[rows, target] += (6 + 12 * _rand((T,), _gen(seed, 3))).to(dt)  # a sampled token is a likely one
    s = dict(case=c, logits=logits, target=target, logp=torch.empty(T, device=DEV), ent=torch.empty(T, device=DEV))
    if c["op"] == "logp":
        return s
    lp = torch.empty(T, device=DEV)
    for i in range(0, T, 512):
        z = logits[i:i + 512].float() / c["temp"]
        lp[i:i + 512] = z.gather(1, target[i:i + 512, None])[:, 0] - z.logsumexp(dim=1)
    # old and reference policies a few updates away; a log ratio within 1e-3 of a corner of the clip is moved off
    # it, where the gradient jumps and one rounding decides
    move = 0.2 * torch.randn(T, generator=_gen(seed, 4), device=DEV)
    for corner in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH), math.log(DUAL)):
        move = torch.where((move - corner).abs() < 1e-3, corner + 2e-3, move)
    s["old"] = lp - move
    s["ref"] = lp + 0.3 * torch.randn(T, generator=_gen(seed, 5), device=DEV) if c["kl"] > 0 else None
    # one advantage for each response of up to 256 tokens; prompt and padding rows take no part
    n = min(T, 256)
    s["adv"] = torch.randn(T // n + 1, generator=_gen(seed, 6), device=DEV)[rows // n]
    live = _rand((T,), _gen(seed, 7)) < 0.9
    live[0] = True
    s["target"] = torch.where(live, target, IGNORED)
    s["w"] = live.float() / live.sum()
    s["stats"] = torch.empty(8, device=DEV)
    s["dlogits"] = torch.empty((T, V), dtype=dt, device=DEV)
    return s


# ------------------------------------------------------------------ the plain forms


def _pairs(x, inter):
    """The two members of every rotated pair."""
    r = x.shape[-1]
    return (x[..., 0::2], x[..., 1::2]) if inter else (x[..., : r // 2], x[..., r // 2:])


def _unpair(a, b, inter):
    return torch.stack([a, b], dim=-1).flatten(-2) if inter else torch.cat([a, b], dim=-1)


def _turn(x, angles, c, back=False):
    """x [T, H, d] with its first rot dims turned by the angles' rows [T, rot], or turned back."""
    cos, sin = angles[:, None].chunk(2, dim=-1)
    if back:
        sin = -sin
    a, b = _pairs(x[..., : c["rot"]], c["inter"])
    y = _unpair(a * cos - b * sin, b * cos + a * sin, c["inter"])
    return torch.cat([y, x[..., c["rot"]:]], dim=-1) if c["rot"] < c["d"] else y


def _normed(x, w):
    x = x.float()
    return x if w is None else x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w.float()


def _norm_back(x, w, g):
    """Gradients of x and w of _normed, from that of its result."""
    if w is None:
        return g, None
    x = x.float()
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    y = x * r
    dw = (g * y).sum(dim=(0, 1))
    g = g * w.float()
    return r * (g - y * (g * y).mean(dim=-1, keepdim=True)), dw


def _places(s):
    """Position, block and slot of every new token."""
    c, T = s["case"], s["T"]
    t = torch.arange(T, device=DEV)
    o = s["offsets"]
    if o is None:
        o = torch.arange(c["B"] + 1, device=DEV) * (T // c["B"])
    o = o.long()
    b = torch.searchsorted(o, t, right=True) - 1
    pos = s["lens"].long()[b] - o[b + 1] + t
    return pos, s["block_table"][b, pos // BS].long(), pos % BS


def _write_fp8(cache, scales, x, block, slot, first, is_v):
    """x [T, hkv, d] into an fp8 cache's tiles; a tile whose new tokens pass its range gets their amax's scale."""
    amax = torch.zeros_like(scales).index_reduce_(0, block, x.abs().amax(dim=-1), "amax")
    fresh = (first[:, None] == 0) | (scales <= 0) | (amax > FP8_MAX * scales)
    touched = (first < BS)[:, None]
    new = torch.where(fresh & touched, torch.clamp(amax / FP8_MAX, min=MIN_SCALE), scales)
    tiles = cache.transpose(2, 3) if is_v else cache  # [nb, hkv, slot, d]
    old = (tiles.float() * scales[:, :, None, None] / new[:, :, None, None]).clamp(-FP8_MAX, FP8_MAX)
    earlier = torch.arange(BS, device=DEV)[None, :] < first[:, None]
    again = (fresh & touched)[:, :, None, None] & earlier[:, None, :, None]
    y = torch.where(again, old, tiles.float())
    y[block, :, slot] = (x / new[block][:, :, None]).clamp(-FP8_MAX, FP8_MAX)
    cache.copy_((y.transpose(2, 3) if is_v else y).to(cache.dtype))
    scales.copy_(new)


def _run_append(s):
    c = s["case"]
    pos, block, slot = _places(s)
    angles = s["table"][pos]
    s["q_out"].copy_(_turn(_normed(s["q"], s["wq"]), angles, c))
    k, v = _turn(_normed(s["new_k"], s["wk"]), angles, c), s["new_v"].float()
    if c["kv"] != "fp8":
        s["k"][block, :, slot] = k.to(s["k"].dtype)
        s["v"][block, :, :, slot] = v.to(s["v"].dtype)
        return
    first = torch.full((s["k"].shape[0],), BS, device=DEV).index_reduce_(0, block, slot, "amin")
    _write_fp8(s["k"], s["scales"][0], k, block, slot, first, False)
    _write_fp8(s["v"], s["scales"][1], v, block, slot, first, True)


def _run_rope(s):
    c, angles = s["case"], s["table"][s["positions"].long()]
    s["q_out"].copy_(_turn(_normed(s["q"], s["wq"]), angles, c))
    s["k_out"].copy_(_turn(_normed(s["k"], s["wk"]), angles, c))


def _run_rope_bwd(s):
    c, angles = s["case"], s["table"][s["positions"].long()]
    for x, w, g, dx, dw in (("q", "wq", "gq", "dq", "dwq"), ("k", "wk", "gk", "dk", "dwk")):
        a, b = _norm_back(s[x], s[w], _turn(s[g].float(), angles, c, back=True))
        s[dx].copy_(a)
        if b is not None:
            s[dw].copy_(b)


def _logp(s):
    """z less its largest, probabilities, log of the sum, and the target's log-probability and the entropy."""
    c = s["case"]
    z = s["logits"].float() / c["temp"]
    z = z - z.amax(dim=1, keepdim=True)
    e = z.exp()
    total = e.sum(dim=1)
    lse = total.log()
    rows, y = torch.arange(c["T"], device=DEV), s["target"].clamp(min=0)
    lp = torch.where(s["target"] >= 0, z[rows, y] - lse, 0.0)
    ent = torch.where(s["target"] >= 0, lse - (e * z).sum(dim=1) / total, 0.0)
    return z, e / total[:, None], lse, lp, ent


def _run_logp(s):
    _, _, _, lp, ent = _logp(s)
    s["logp"].copy_(lp)
    s["ent"].copy_(ent)


def _run_policy(s):
    c, w, A = s["case"], s["w"], s["adv"]
    z, p, lse, lp, ent = _logp(s)
    d = lp - s["old"]
    inside = d.abs() <= CLAMP
    r = d.clamp(-CLAMP, CLAMP).exp()
    plain, cut = -A * r, -A * r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH)
    clipped = cut > plain
    pg = torch.maximum(plain, cut)
    floor = -A * DUAL
    dual = (A < 0) & (pg > floor)
    pg = torch.where(dual, floor, pg)
    # where the cut form is the larger one, it is a constant
    g = torch.where(clipped | dual | ~inside, 0.0, plain)
    kl = torch.zeros_like(lp)
    if s["ref"] is not None:
        u = s["ref"] - lp
        near = u.abs() <= CLAMP
        u = u.clamp(-CLAMP, CLAMP)
        kl = torch.expm1(u) - u
        g = g - torch.where(near, c["kl"] * torch.expm1(u), 0.0)
    loss = pg + c["kl"] * kl - c["ent"] * ent
    old_kl = torch.expm1(-d.clamp(-CLAMP, CLAMP)) + d.clamp(-CLAMP, CLAMP)
    terms = torch.stack([loss, pg, kl, ent, (clipped | dual).float(), r, old_kl, torch.ones_like(lp)])
    s["stats"].copy_((terms * w).sum(dim=1))
    s["logp"].copy_(lp)
    s["ent"].copy_(ent)
    k = (w / c["temp"])[:, None]
    out = p * ((c["ent"] * (z - lse[:, None] + ent[:, None])) - g[:, None])
    rows, y = torch.arange(c["T"], device=DEV), s["target"].clamp(min=0)
    out[rows, y] += g
    s["dlogits"].copy_(torch.where(k != 0, out * k, 0.0))


PLAIN = {"append": _run_append, "rope": _run_rope, "rope_bwd": _run_rope_bwd, "logp": _run_logp, "policy": _run_policy}


# ------------------------------------------------------------------ the framework's calls


def _own(s):
    from paper_2605_20863_amd import _lib

    c = s["case"]
    op = c["op"]
    if op == "append":
        _lib.paged_qk_norm_rope_append(s["q"], s["new_k"], s["new_v"], s["wq"], s["wk"], s["table"], s["offsets"],
                                       s["k"], s["v"], s["scales"], s["block_table"], s["lens"], s["q_out"], eps=EPS,
                                       interleaved=c["inter"])
    elif op == "rope":
        _lib.qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], s["table"], s["positions"], s["q_out"], s["k_out"], eps=EPS,
                          interleaved=c["inter"])
    elif op == "rope_bwd":
        _lib.qk_norm_rope_backward(s["q"], s["k"], s["wq"], s["wk"], s["table"], s["positions"], s["gq"], s["gk"],
                                   s["dq"], s["dk"], s["dwq"], s["dwk"], eps=EPS, interleaved=c["inter"])
    elif op == "logp":
        _lib.token_logprobs(s["logits"], s["target"], s["logp"], s["ent"], temperature=c["temp"])
    else:
        _lib.policy_loss(s["logits"], s["target"], s["old"], s["adv"], s["w"], s["stats"], s["dlogits"], s["logp"],
                         s["ent"], ref_logprobs=s["ref"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH, dual_clip=DUAL,
                         kl_coef=c["kl"], entropy_coef=c["ent"], temperature=c["temp"])


OUTPUTS = {"append": ("q_out", "k", "v", "scales"), "rope": ("q_out", "k_out"), "rope_bwd": ("dq", "dk", "dwq", "dwk"),
           "logp": ("logp", "ent"), "policy": ("stats", "dlogits", "logp", "ent")}


def run(s):
    op = s["case"]["op"]
    if own:
        _own(s)
    else:
        PLAIN[op](s)
    return {name: s[name] for name in OUTPUTS[op] if s[name] is not None}


# ------------------------------------------------------------------ 64-bit results


def _rotated(x, w, angles, c):
    """Norm and rotation of x [T, H, d] in 64 bits, pairs turned as complex numbers."""
    x = x.to(torch.float64)
    if w is not None:
        x = x / torch.sqrt((x ** 2).sum(dim=-1, keepdim=True) / c["d"] + EPS) * w.to(torch.float64)
    return _spun(x, angles, c, 1)


def _spun(x, angles, c, sign):
    h, x = c["rot"] // 2, x.clone()
    at = torch.arange(h, device=x.device)
    i, j = (2 * at, 2 * at + 1) if c["inter"] else (at, at + h)
    a = angles.to(torch.float64)[:, None]
    y = torch.complex(x[..., i], x[..., j]) * torch.complex(a[..., :h], sign * a[..., h:])
    x[..., i], x[..., j] = y.real, y.imag
    return x


def _grads(x, w, g, angles, c):
    """Gradients in 64 bits: through the rotation's transpose, then the norm's Jacobian (I - x x^T / (d m)) / sqrt(m)."""
    g, x = _spun(g.to(torch.float64), angles, c, -1), x.to(torch.float64)
    if w is None:
        return g, None
    m = (x ** 2).sum(dim=-1, keepdim=True) / c["d"] + EPS
    dw = (g * x / torch.sqrt(m)).sum(dim=0).sum(dim=0)
    g = g * w.to(torch.float64)
    return g / torch.sqrt(m) - x * (g * x).sum(dim=-1, keepdim=True) / (c["d"] * m ** 1.5), dw


def exact(c, seed):
    """run()'s outputs in float64; an fp8 cache's codes are choices between neighbours and have no such value."""
    s = prepare(c, seed)
    if c["op"] == "append":
        return _exact_append(s, c)
    if c["op"] in ("logp", "policy"):
        return _exact_head(s, c)
    angles = s["table"][s["positions"].long()]
    if c["op"] == "rope":
        return {"q_out": _rotated(s["q"], s["wq"], angles, c), "k_out": _rotated(s["k"], s["wk"], angles, c)}
    (dq, dwq), (dk, dwk) = _grads(s["q"], s["wq"], s["gq"], angles, c), _grads(s["k"], s["wk"], s["gk"], angles, c)
    out = {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    return {k: v for k, v in out.items() if v is not None}


def _exact_append(s, c):
    L, n = _lengths(c)
    at = np.concatenate([np.arange(a - b, a) for a, b in zip(L, n)])
    seq = np.repeat(np.arange(c["B"]), n)
    tab = s["block_table"].cpu().numpy()
    block, slot = (torch.from_numpy(x.astype(np.int64)).to(DEV) for x in (tab[seq, at // BS], at % BS))
    angles = s["table"][torch.from_numpy(at).to(DEV)]
    out = {"q_out": _rotated(s["q"], s["wq"], angles, c)}
    k, v = _rotated(s["new_k"], s["wk"], angles, c), s["new_v"].to(torch.float64)
    if c["kv"] != "fp8":
        out["k"], out["v"] = s["k"].to(torch.float64), s["v"].to(torch.float64)
        out["k"][block, :, slot] = k
        out["v"][block, :, :, slot] = v
        return out
    scales = s["scales"].to(torch.float64)
    lowest = torch.full((s["k"].shape[0],), BS, device=DEV).scatter_reduce_(0, block, slot, "amin")
    for i, x in enumerate((k, v)):
        top = torch.zeros_like(scales[i])
        top.scatter_reduce_(0, block[:, None].expand(-1, c["hkv"]), x.abs().amax(dim=-1), "amax")
        raised = (lowest < BS)[:, None] & ((lowest == 0)[:, None] | (top > FP8_MAX * scales[i]))
        scales[i] = torch.where(raised, (top / FP8_MAX).clamp(min=MIN_SCALE), scales[i])
    return dict(out, k=None, v=None, scales=scales)


def _exact_head(s, c):
    T, V = c["T"], c["V"]
    policy = c["op"] == "policy"
    lp, ent = (torch.zeros(T, dtype=torch.float64, device=DEV) for _ in range(2))
    d = torch.empty((T, V), dtype=torch.float64, device=DEV) if policy else None
    terms = torch.zeros((8, T), dtype=torch.float64, device=DEV)
    step = max(1, (1 << 27) // V)
    for i in range(0, T, step):
        at = slice(i, min(T, i + step))
        y = s["target"][at]
        live = y >= 0
        logp = torch.log_softmax(s["logits"][at].to(torch.float64) / c["temp"], dim=1)
        p = logp.exp()
        h = -(p * logp).sum(dim=1)
        x = logp.gather(1, y.clamp(min=0)[:, None])[:, 0]
        lp[at], ent[at] = torch.where(live, x, 0.0), torch.where(live, h, 0.0)
        if not policy:
            continue
        A, w = (s[k][at].to(torch.float64) for k in ("adv", "w"))
        t, slope = _exact_terms(s, c, at, lp[at], A)
        t[0] -= c["ent"] * h
        t[3] = h
        terms[:, at] = torch.where(w != 0, t * w, 0.0)
        g = -p * slope[:, None] + c["ent"] * p * (logp + h[:, None])
        g[torch.arange(len(y), device=DEV), y.clamp(min=0)] += slope
        d[at] = torch.where((w != 0)[:, None], g * (w / c["temp"])[:, None], 0.0)
    if not policy:
        return {"logp": lp, "ent": ent}
    return {"stats": terms.sum(dim=1), "dlogits": d, "logp": lp, "ent": ent}


def _exact_terms(s, c, at, lp, A):
    """A token's loss terms without the entropy, and the loss's derivative by its log-probability."""
    x = lp - s["old"][at].to(torch.float64)
    r = torch.exp(x.clamp(-CLAMP, CLAMP))
    pg, cut = -A * r, -A * r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH)
    held = cut > pg
    pg = torch.where(held, cut, pg)
    low = (A < 0) & (pg > -A * DUAL)
    pg = torch.where(low, -A * DUAL, pg)
    slope = torch.where(held | low | (x.abs() > CLAMP), 0.0, -A * r)
    kl = torch.zeros_like(lp)
    if s["ref"] is not None:
        u = s["ref"][at].to(torch.float64) - lp
        v = u.clamp(-CLAMP, CLAMP)
        kl = torch.exp(v) - 1 - v
        slope = slope + c["kl"] * torch.where(u.abs() > CLAMP, 0.0, 1 - torch.exp(v))
    v = x.clamp(-CLAMP, CLAMP)
    one = torch.ones_like(lp)
    t = torch.stack([pg + c["kl"] * kl, pg, kl, one, (held | low).to(torch.float64), r, torch.exp(-v) - 1 + v, one])
    return t, slope
