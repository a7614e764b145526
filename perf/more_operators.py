"""Timed cases of the operators around a transformer's blocks and behind its head, in rollout and distillation programs.

A case is one pass through one of the operators:

    norm      a block's output added to the residual stream, the stream's root-mean-square norm, and its rounding to
              the type of the product that reads it (bf16, f32, or fp8 with a scale for each row or group of a row)
    norm_bwd  its gradient: of the stream (and so of both summands) and of the weights
    top       the most likely alternatives of every row of logits and their log-probabilities, with that of a given
              token and the entropy: what a server answers with, and what a teacher hands on
    distill   distillation from a teacher's list of likely tokens: the loss and its gradient at the student's logits

With ``own`` false the operators run in their plain form, elementary torch operations in 32 bits; with ``own`` true
through ``paper_2605_20863_amd._lib``. What decides on the amount of work depends on the case alone (its ``lseed``);
tensors come from the seed.
"""

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
FP8_MAX, MIN_SCALE = 448.0, 2.0 ** -126
LEAST_REST = 2.0 ** -24  # a teacher's probability outside of its list is taken as at least this
IGNORED = -100  # target of a token that takes no part
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
SIZE = {"f32": 4, "bf16": 2, "fp8": 1}


def _norm(name, op, T, H, t, **more):
    return dict(dict(name=name, op=op, T=T, H=H, t=t, out=t, group=0, add=True, pad=0, wt="bf16"), **more)


def _head(name, op, T, V, K, t, **more):
    return dict(dict(name=name, op=op, T=T, V=V, K=K, t=t, pad=0, temp=1.0, lseed=1, targets=True, rev=0.0, rest=True), **more)


def listed():
    return [
        # a few interactive chats, one token each, in front of an fp8 projection: launches and latency count
        _norm("norm_chat_fp8", "norm", 3, 4096, "bf16", out="fp8", group=128),
        # chunked prefill or a training micro-batch of 16k tokens
        _norm("norm_prefill_bf16", "norm", 16384, 4096, "bf16"),
        # one decode step of a large batch into fp8, one scale a token
        _norm("norm_decode_fp8", "norm", 512, 8192, "bf16", out="fp8"),
        _norm("norm_bwd_train_bf16", "norm_bwd", 16384, 4096, "bf16"),
        # a small float32 model, odd token count, rows of a wider buffer
        _norm("norm_bwd_small_f32", "norm_bwd", 777, 1000, "f32", pad=24, wt="f32"),
        # the answers of one decode step with 20 alternatives each
        _head("top_decode_bf16", "top", 64, 131072, 20, "bf16", temp=0.7),
        # a chat's next token in float32, odd vocabulary in padded rows
        _head("top_chat_f32", "top", 2, 150001, 5, "f32", pad=15),
        # a teacher's forward over a micro-batch: 64 tokens of each row for its student, no targets
        _head("top_teacher_bf16", "top", 4096, 131072, 64, "bf16", targets=False),
        # one update micro-batch of a student: forward divergence with a bucket for the rest
        _head("distill_bf16", "distill", 4096, 131072, 64, "bf16"),
        # few long rows, long lists, forward and reverse mixed
        _head("distill_mixed_bf16", "distill", 96, 131072, 256, "bf16", rev=0.5),
        # a short odd batch in float32, reverse divergence over the list alone, odd vocabulary in padded rows
        _head("distill_small_f32", "distill", 37, 50001, 100, "f32", pad=7, rev=1.0, rest=False, temp=0.9),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_bwd", "top", "top", "distill", "distill"])
    t = rng.choice(["bf16", "bf16", "f32"])
    if op in ("norm", "norm_bwd"):
        H = 8 * _logint(rng, 8, 2048)
        T = _logint(rng, 1, min(32768, 5e8 / (H * SIZE[t] * 4)))
        c = _norm("", op, T, H, t, add=rng.random() < 0.8, pad=8 * rng.choice([0, 0, rng.randint(1, 16)]), wt=rng.choice([t, "f32"]))
        if op == "norm":
            c["out"] = rng.choice([t, t, "fp8", "fp8", "f32"])
            c["group"] = rng.choice([g for g in (0, 0, 64, 128) if g == 0 or H % g == 0]) if c["out"] == "fp8" else 0
        return _pure(c)
    V = _logint(rng, 1000, 200000)
    T = _logint(rng, 1, max(2, min(8192, 1.0e9 / (V * SIZE[t]))))
    c = _head("", op, T, V, _logint(rng, 1, 256), t, pad=rng.choice([0, 0, rng.randint(1, 64)]),
              temp=rng.choice([1.0, 1.0, 0.7, 1.3]), lseed=rng.randrange(2, 1 << 30))
    if op == "top":
        c["targets"] = rng.random() < 0.7
    else:
        c.update(rev=rng.choice([0.0, 0.0, 1.0, round(rng.random(), 2)]), rest=rng.random() < 0.7)
    return _pure(c)


def _pure(c):
    del c["name"]
    return c


def work(c):
    """Every input read once, every output written once."""
    T = c["T"]
    if c["op"] in ("norm", "norm_bwd"):
        H, e, w = c["H"], SIZE[c["t"]], SIZE[c["wt"]]
        if c["op"] == "norm_bwd":
            return {"bytes": T * H * e * (4 if c["add"] else 3) + H * (w + 4), "flops": 12.0 * T * H}
        scales = 0 if c["out"] != "fp8" else 4 * T * (H // c["group"] if c["group"] else 1)
        return {"bytes": T * H * (e * (3 if c["add"] else 1) + SIZE[c["out"]]) + H * w + scales, "flops": 6.0 * T * H}
    V, K, e = c["V"], c["K"], SIZE[c["t"]]
    if c["op"] == "top":
        return {"bytes": T * (V * e + 8 * K + 4 + (12 if c["targets"] else 0)), "flops": 7.0 * T * V}
    return {"bytes": T * (2 * V * e + 8 * K + 8) + 24, "flops": 10.0 * T * V}


# ------------------------------------------------------------------ inputs


def _gen(seed, key):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + key) & ((1 << 62) - 1))


def _randn(shape, gen, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device=DEV, dtype=dtype)


def _rand(shape, gen):
    return torch.rand(shape, generator=gen, device=DEV, dtype=torch.float32)


def prepare(c, seed):
    return (_prepare_norm if c["op"] in ("norm", "norm_bwd") else _prepare_head)(c, seed)


def _prepare_norm(c, seed):
    T, H, dt = c["T"], c["H"], TYPES[c["t"]]
    s = dict(case=c)
    s["weight"] = (1.0 + 0.2 * _randn((H,), _gen(seed, 1))).to(TYPES[c["wt"]])
    # a residual stream: a few channels are much larger than the rest
    loud = 1.0 + 30.0 * (_rand((H,), _gen(seed, 2)) < 0.004).float()
    stream = (_randn((T, H + c["pad"]), _gen(seed, 3), dt)[:, :H]).mul_(loud.to(dt))
    new = _randn((T, H), _gen(seed, 4), dt).mul_(0.5)
    if c["op"] == "norm_bwd":
        s["h"], s["grad_out"] = stream, new.mul_(0.02)
        s["grad_sum"] = _randn((T, H), _gen(seed, 5), dt).mul_(0.01) if c["add"] else None
        s["grad_h"], s["grad_weight"] = torch.empty((T, H), dtype=dt, device=DEV), torch.empty(H, device=DEV)
        return s
    s["x"], s["residual"] = (new, stream) if c["add"] else (stream, None)
    s["sum"] = torch.empty((T, H), dtype=dt, device=DEV) if c["add"] else None
    s["out"] = torch.empty((T, H), dtype=TYPES[c["out"]], device=DEV)
    s["scales"] = None
    if c["out"] == "fp8":
        s["scales"] = torch.empty((T, H // c["group"] if c["group"] else 1), device=DEV)
    return s


def _lists(c, seed):
    """K tokens of every row, all different, and a teacher's log-probabilities of them, largest first."""
    T, V, K = c["T"], c["V"], min(c["K"], c["V"])
    edge = torch.arange(K + 1, device=DEV) * V // K
    ids = edge[:-1] + (_rand((T, K), _gen(seed, 10)) * (edge[1:] - edge[:-1])).long().clamp(max=V - 1)
    ids = torch.minimum(ids, edge[1:] - 1).gather(1, _rand((T, K), _gen(seed, 11)).argsort(dim=1))
    score = -1.2 * torch.log1p(torch.arange(K, device=DEV).float()) * (0.5 + 1.5 * _rand((T, 1), _gen(seed, 12)))
    score = (score - 0.1 * _rand((T, K), _gen(seed, 13))).sort(dim=1, descending=True).values.double()
    mass = 1 - 10 ** (-0.5 - 2.5 * _rand((T, 1), _gen(seed, 14)).double())
    return ids, (score - score.logsumexp(dim=1, keepdim=True) + mass.log()).float()


def _prepare_head(c, seed):
    T, V, K, dt = c["T"], c["V"], c["K"], TYPES[c["t"]]
    logits = _randn((T, V + c["pad"]), _gen(seed, 1), dt)[:, :V]
    logits.mul_(2.0 * c["temp"])
    rows = torch.arange(T, device=DEV)
    # the head of a row's distribution stands out of it, near to what a teacher gives
    ids, tau = _lists(c, seed)
    logits.scatter_(1, ids, (c["temp"] * (math.log(V) + 5 + tau + 0.5 * _randn(tau.shape, _gen(seed, 15)))).to(dt))
    live = torch.rand((T,), generator=_gen(c["lseed"], 16), device=DEV) < 0.9
    live[0] = True
    s = dict(case=c, logits=logits)
    if c["op"] == "top":
        s["ids"] = torch.empty((T, K), dtype=torch.int32, device=DEV)
        s["tops"] = torch.empty((T, K), device=DEV)
        s["target"], s["logp"] = None, None
        if c["targets"]:
            s["target"] = torch.where(live, ids[rows, (_rand((T,), _gen(seed, 17)) ** 3 * ids.shape[1]).long().clamp(max=ids.shape[1] - 1)], IGNORED)
            s["logp"] = torch.empty(T, device=DEV)
        s["ent"] = torch.empty(T, device=DEV)
        return s
    # some teachers' lists are shorter; prompt and padding rows have weight 0
    n = torch.where(_rand((T, 1), _gen(seed, 18)) < 0.12, (_rand((T, 1), _gen(seed, 19)) * (ids.shape[1] + 1)).long(), ids.shape[1])
    gone = torch.arange(ids.shape[1], device=DEV) >= n
    s["ids"] = torch.full((T, K), -1, dtype=torch.int32, device=DEV)
    s["tau"] = torch.full((T, K), -math.inf, device=DEV)
    s["ids"][:, :ids.shape[1]] = torch.where(gone, -1, ids).to(torch.int32)
    s["tau"][:, :ids.shape[1]] = torch.where(gone, -math.inf, tau)
    s["w"] = live.float() / live.sum()
    s["stats"], s["losses"] = torch.empty(6, device=DEV), torch.empty(T, device=DEV)
    s["dlogits"] = torch.empty((T, V), dtype=dt, device=DEV)
    return s


# ------------------------------------------------------------------ the plain forms


def _run_norm(s):
    c, x = s["case"], s["x"].float()
    if s["residual"] is not None:
        # the norm sees the stream as it is kept, in its own type
        s["sum"].copy_(x + s["residual"].float())
        x = s["sum"].float()
    y = x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS) * s["weight"].float()
    if c["out"] == "fp8":
        y = y.view(c["T"], s["scales"].shape[1], -1)
        s["scales"].copy_((y.abs().amax(dim=2) / FP8_MAX).clamp(min=MIN_SCALE))
        y = (y / s["scales"][:, :, None]).clamp(-FP8_MAX, FP8_MAX).view(c["T"], -1)
    s["out"].copy_(y)


def _run_norm_bwd(s):
    x, g = s["h"].float(), s["grad_out"].float()
    r = torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS)
    y = x * r
    s["grad_weight"].copy_((g * y).sum(dim=0))
    g = g * s["weight"].float()
    d = r * (g - y * (g * y).mean(dim=1, keepdim=True))
    s["grad_h"].copy_(d if s["grad_sum"] is None else d + s["grad_sum"].float())


def _run_top(s):
    c = s["case"]
    V, step = c["V"], max(1, (1 << 26) // c["V"])
    k = min(c["K"], V)
    s["ids"].fill_(-1)
    s["tops"].fill_(-math.inf)
    for i in range(0, c["T"], step):
        at = slice(i, min(c["T"], i + step))
        l = s["logits"][at].float() + 0.0
        z = l / c["temp"]
        z = z - z.amax(dim=1, keepdim=True)
        e = z.exp()
        total = e.sum(dim=1, keepdim=True)
        lse = total.log()
        # a word's place in its row's order as one whole number: its logit's, then the lower index
        u = l.view(torch.int32)
        key = (u ^ ((u >> 31) & 0x7FFFFFFF)).long() * (1 << 31) + (V - 1 - torch.arange(V, device=DEV))
        word = V - 1 - (key.topk(k, dim=1).values & 0x7FFFFFFF)
        lp = z.gather(1, word) - lse
        word = torch.where(lp == -math.inf, -1, word)
        live = torch.ones_like(lse, dtype=torch.bool)
        if s["target"] is not None:
            y = s["target"][at, None]
            live = y >= 0
            s["logp"][at] = torch.where(live, z.gather(1, y.clamp(min=0)) - lse, 0.0)[:, 0]
        s["ids"][at, :k] = torch.where(live, word, -1).to(torch.int32)
        s["tops"][at, :k] = torch.where(live, lp, -math.inf)
        s["ent"][at] = torch.where(live, lse - (e * z).sum(dim=1, keepdim=True) / total, 0.0)[:, 0]


def _run_distill(s):
    c, w = s["case"], s["w"][:, None]
    z = s["logits"].float() / c["temp"]
    z = z - z.amax(dim=1, keepdim=True)
    real = (s["ids"] >= 0) & (s["tau"] > -math.inf)
    at = torch.where(real, s["ids"].long(), c["V"])
    listed_ = torch.zeros((c["T"], c["V"] + 1), dtype=torch.bool, device=DEV).scatter_(1, at, True)[:, :-1]
    at = at.clamp(max=c["V"] - 1)
    lse = z.exp().sum(dim=1, keepdim=True).log()
    lp = torch.where(real, z.gather(1, at) - lse, 0.0)
    tau = torch.where(real, s["tau"], 0.0)
    t, p, a = (torch.where(real, x, 0.0) for x in (tau.exp(), lp.exp(), lp - tau))
    S, P = t.double().sum(dim=1, keepdim=True).float(), p.sum(dim=1, keepdim=True)
    fwd, rev = (-t * a).sum(dim=1, keepdim=True), (p * a).sum(dim=1, keepdim=True)
    others = z.masked_fill(listed_, -math.inf)
    top = others.amax(dim=1, keepdim=True)
    lpr = (others - top).exp().sum(dim=1, keepdim=True).log() + top - lse
    pr = lpr.exp()
    total = S
    if c["rest"]:
        some = ~listed_.all(dim=1, keepdim=True)
        tr = (1 - torch.where(real, s["tau"], -math.inf).double().exp().sum(dim=1, keepdim=True)).clamp(min=LEAST_REST).float()
        tr = torch.where(some, tr, 0.0)
        ar = torch.where(some, lpr - tr.log(), 0.0)
        fwd, rev, total = fwd - tr * ar, rev + pr * ar, S + tr
        by_word = (1 - c["rev"]) * (total - torch.where(some, tr / pr, 0.0)) + c["rev"] * (ar - rev)
        by_list = (1 - c["rev"]) * (p * total - t) + c["rev"] * p * (a - rev)
    else:
        by_word = (1 - c["rev"]) * total - c["rev"] * (rev + P)
        by_list = (1 - c["rev"]) * (p * total - t) + c["rev"] * p * (a + 1 - rev - P)
    loss = (1 - c["rev"]) * fwd + c["rev"] * rev
    terms = torch.cat([loss, fwd, rev, S, P, torch.ones_like(loss)], dim=1)
    s["stats"].copy_((terms * w).sum(dim=0))
    s["losses"].copy_(loss[:, 0])
    d = (others - lse).exp() * by_word  # 0 for the listed words
    d.scatter_add_(1, at, torch.where(real, by_list, 0.0))
    s["dlogits"].copy_(torch.where(w != 0, d * (w / c["temp"]), 0.0))


PLAIN = {"norm": _run_norm, "norm_bwd": _run_norm_bwd, "top": _run_top, "distill": _run_distill}


# ------------------------------------------------------------------ the framework's calls


def _own(s):
    from paper_2605_20863_amd import _lib

    c = s["case"]
    op = c["op"]
    if op == "norm":
        _lib.add_rms_norm(s["x"], s["weight"], s["out"], s["residual"], s["sum"], s["scales"], eps=EPS)
    elif op == "norm_bwd":
        _lib.add_rms_norm_backward(s["h"], s["weight"], s["grad_out"], s["grad_h"], s["grad_weight"], s["grad_sum"], eps=EPS)
    elif op == "top":
        _lib.top_logprobs(s["logits"], s["ids"], s["tops"], s["target"], s["logp"], s["ent"], temperature=c["temp"])
    else:
        _lib.distill_loss(s["logits"], s["ids"], s["tau"], s["w"], s["stats"], s["dlogits"], s["losses"], reverse=c["rev"],
                          rest=c["rest"], temperature=c["temp"])


OUTPUTS = {"norm": ("out", "scales", "sum"), "norm_bwd": ("grad_h", "grad_weight"), "top": ("ids", "tops", "logp", "ent"),
           "distill": ("stats", "losses", "dlogits")}


def run(s):
    op = s["case"]["op"]
    if own:
        _own(s)
    else:
        PLAIN[op](s)
    return {name: s[name] for name in OUTPUTS[op] if s[name] is not None}


# ------------------------------------------------------------------ 64-bit results


def exact(c, seed):
    """run()'s outputs in float64. Where the stream's sum is rounded before the norm, that rounding is part of the
    definition; fp8 outputs are given as what is rounded to a code."""
    s = prepare(c, seed)
    return {"norm": _exact_norm, "norm_bwd": _exact_norm_bwd, "top": _exact_top, "distill": _exact_distill}[c["op"]](s, c)


def _exact_norm(s, c):
    h = s["x"].to(torch.float64)
    out = {}
    if c["add"]:
        total = h + s["residual"].to(torch.float64)
        h = total.to(TYPES[c["t"]]).to(torch.float64)
    h = h / torch.sqrt((h ** 2).sum(dim=1, keepdim=True) / c["H"] + EPS) * s["weight"].to(torch.float64)
    if c["out"] == "fp8":
        g = c["group"] or c["H"]
        parts = h.unflatten(1, (-1, g))
        top = torch.maximum(parts.max(dim=2).values, -parts.min(dim=2).values) / FP8_MAX
        out["scales"] = torch.where(top < MIN_SCALE, MIN_SCALE, top)
        h = (parts / out["scales"].unsqueeze(2)).flatten(1)
    out["out"] = h
    if c["add"]:
        out["sum"] = total
    return {k: out[k] for k in OUTPUTS["norm"] if k in out}


def _exact_norm_bwd(s, c):
    h, w, g = (s[k].to(torch.float64) for k in ("h", "weight", "grad_out"))
    m = (h ** 2).sum(dim=1, keepdim=True) / c["H"] + EPS
    dw = (g * h / m.sqrt()).sum(dim=0)
    # the Jacobian (I - h h^T / (H m)) / sqrt(m)
    g = g * w
    d = g / m.sqrt() - h * (g * h).sum(dim=1, keepdim=True) / (c["H"] * m ** 1.5)
    if c["add"]:
        d = d + s["grad_sum"].to(torch.float64)
    return {"grad_h": d, "grad_weight": dw}


def _exact_top(s, c):
    T, V, K = c["T"], c["V"], c["K"]
    ids = torch.full((T, K), -1, dtype=torch.int32, device=DEV)
    tops = torch.full((T, K), -math.inf, dtype=torch.float64, device=DEV)
    logp, ent = (torch.zeros(T, dtype=torch.float64, device=DEV) for _ in range(2))
    k, step = min(K, V), max(1, (1 << 25) // V)
    for i in range(0, T, step):
        at = slice(i, min(T, i + step))
        lp = torch.log_softmax(s["logits"][at].to(torch.float64) / c["temp"], dim=1)
        order = torch.sort(s["logits"][at], dim=1, descending=True, stable=True).indices[:, :k]
        best = lp.gather(1, order)
        h = -(lp.exp() * lp).sum(dim=1)
        live = torch.ones_like(h, dtype=torch.bool)
        if c["targets"]:
            y = s["target"][at]
            live = y >= 0
            logp[at] = torch.where(live, lp.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
        ids[at, :k] = torch.where(live[:, None] & (best > -math.inf), order, -1).to(torch.int32)
        tops[at, :k] = torch.where(live[:, None], best, -math.inf)
        ent[at] = torch.where(live, h, 0.0)
    out = {"ids": ids, "tops": tops, "logp": logp if c["targets"] else None, "ent": ent}
    return {n: x for n, x in out.items() if x is not None}


def _exact_distill(s, c):
    """Rows' divergences from their definition; gradients are those of -sum_b t_b log p_b and sum_b p_b log(p_b / t_b) by the
    words' logits, through log p = z - lse."""
    T, V, b = c["T"], c["V"], c["rev"]
    d = torch.empty((T, V), dtype=torch.float64, device=DEV)
    terms = torch.zeros((T, 6), dtype=torch.float64, device=DEV)
    step = max(1, (1 << 26) // V)
    for i in range(0, T, step):
        at = slice(i, min(T, i + step))
        logp = torch.log_softmax(s["logits"][at].to(torch.float64) / c["temp"], dim=1)
        n = logp.shape[0]
        # the teacher's log-probability of every word, NaN outside of its list
        teacher = torch.full((n, V + 1), math.nan, dtype=torch.float64, device=DEV)
        ids, tau = s["ids"][at].long(), s["tau"][at].to(torch.float64)
        ok = (ids >= 0) & torch.isfinite(tau)
        teacher.scatter_(1, torch.where(ok, ids, V), tau)
        teacher = teacher[:, :V]
        inside = ~torch.isnan(teacher)
        p = logp.exp()
        gap = torch.where(inside, logp - teacher, 0.0)
        t = torch.where(inside, teacher.exp(), 0.0)
        S, P = t.sum(dim=1), torch.where(inside, p, 0.0).sum(dim=1)
        f, r = -(t * gap).sum(dim=1), (p * gap).sum(dim=1)
        if c["rest"]:
            others = torch.logsumexp(torch.where(inside, -math.inf, logp), dim=1)
            some = ~inside.all(dim=1)
            tr = torch.where(some, (1 - S).clamp(min=LEAST_REST), 0.0)
            ar = torch.where(some, others - tr.log(), 0.0)
            pr = others.exp()
            f, r = f - tr * ar, r + pr * ar
            share = torch.where(inside, 0.0, torch.exp(logp - others[:, None]))  # of the rest, given the rest
            df = p * (S + tr)[:, None] - t - share * tr[:, None]
            dr = p * (torch.where(inside, gap, ar[:, None]) - r[:, None])
        else:
            df = p * S[:, None] - t
            dr = torch.where(inside, p * (gap + 1), 0.0) - p * (r + P)[:, None]
        loss = (1 - b) * f + b * r
        w = s["w"][at].to(torch.float64)
        terms[at] = torch.stack([loss, f, r, S, P, torch.ones_like(f)], dim=1)
        d[at] = torch.where(w[:, None] != 0, ((1 - b) * df + b * dr) * (w / c["temp"])[:, None], 0.0)
    return {"stats": (terms * s["w"].to(torch.float64)[:, None]).sum(dim=0), "losses": terms[:, 0].clone(), "dlogits": d}
