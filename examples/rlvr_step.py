"""One RLVR step of a one-layer policy on random weights, through the library's operators:

    rollout   prompts in chunks and responses token by token: norm, rotation and cache append of the new tokens, attention
              over the paged cache, log-probabilities of the sampled tokens
    log-prob  every token of the rollouts at once under a reference policy, over its own paged cache
    update    norm and rotation with their gradient (qk_norm_rope as an autograd function; attention in plain torch),
              the clipped policy loss with its KL term, and its gradient at the logits

    python3 examples/rlvr_step.py [--kv fp8]
"""

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_20863_amd import _lib  # noqa: E402

DEV, BS = "cuda", 16


class QKNormRope(torch.autograd.Function):
    """Norms and rotation of a training forward, gradients by the library."""

    @staticmethod
    def forward(ctx, q, k, wq, wk, table, positions):
        ctx.save_for_backward(q, k, wq, wk, table, positions)
        return _lib.qk_norm_rope(q, k, wq, wk, table, positions, torch.empty_like(q), torch.empty_like(k))

    @staticmethod
    def backward(ctx, gq, gk):
        q, k, wq, wk, table, positions = ctx.saved_tensors
        dq, dk = torch.empty_like(q), torch.empty_like(k)
        dwq, dwk = (torch.empty(w.shape, dtype=torch.float32, device=w.device) for w in (wq, wk))
        _lib.qk_norm_rope_backward(q, k, wq, wk, table, positions, gq.contiguous(), gk.contiguous(), dq, dk, dwq, dwk)
        return dq, dk, dwq.to(wq.dtype), dwk.to(wk.dtype), None, None


class Policy:
    """Embedding, one attention layer with head norms, residual, output head; float32 weights."""

    def __init__(self, vocab=1009, width=256, hq=8, hkv=2, d=64, positions=512, seed=0):
        g = torch.Generator(DEV).manual_seed(seed)
        self.hq, self.hkv, self.d, self.scale = hq, hkv, d, 1 / math.sqrt(d)
        shapes = dict(emb=(vocab, width), qkv=(width, (hq + 2 * hkv) * d), out=(hq * d, width), head=(width, vocab))
        self.w = {n: torch.randn(s, generator=g, device=DEV) * (1.0 if n == "emb" else s[0] ** -0.5) for n, s in shapes.items()}
        self.w["wq"], self.w["wk"] = (torch.ones(d, device=DEV) for _ in "qk")
        inv = 1e4 ** (-torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d)
        a = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * inv
        self.table = torch.cat([a.cos(), a.sin()], 1).float()

    def heads(self, tokens, dtype):
        """(embeddings, views of q, k, v in the packed projection)."""
        x = self.w["emb"][tokens]
        y = (x @ self.w["qkv"]).to(dtype).view(len(tokens), -1, self.d)
        return x, y[:, :self.hq], y[:, self.hq:self.hq + self.hkv], y[:, self.hq + self.hkv:]

    def logits(self, x, attended):
        return (x + attended.float().reshape(len(x), -1) @ self.w["out"]) @ self.w["head"]

    def paged(self, cache, tokens, lens, offsets=None):
        """Logits of new tokens (bf16 attention over the paged cache, which gets them first)."""
        x, q, k, v = self.heads(tokens, torch.bfloat16)
        qr = torch.empty(q.shape, dtype=q.dtype, device=DEV)
        wq, wk = (self.w[n].to(torch.bfloat16) for n in ("wq", "wk"))
        _lib.paged_qk_norm_rope_append(q, k, v, wq, wk, self.table, offsets, cache["k"], cache["v"], cache["scales"],
                                       cache["table"], lens, qr)
        out = torch.empty_like(qr)
        if offsets is None:
            _lib.paged_decode_attention(qr, cache["k"], cache["v"], cache["table"], lens, cache["scales"], out, self.scale)
        else:
            _lib.paged_prefill_attention(qr, offsets, cache["k"], cache["v"], cache["table"], lens, cache["scales"], out,
                                         self.scale)
        return self.logits(x, out)

    def train_logits(self, tokens, positions, lens):
        """Logits of packed sequences with a graph for autograd (float32)."""
        x, q, k, v = self.heads(tokens, torch.float32)
        q, k = QKNormRope.apply(q, k, self.w["wq"], self.w["wk"], self.table, positions)
        outs, group = [], self.hq // self.hkv
        for qs, ks, vs in zip(q.split(lens), k.split(lens), v.split(lens)):
            ks, vs = (t.repeat_interleave(group, dim=1).transpose(0, 1) for t in (ks, vs))
            s = qs.transpose(0, 1) @ ks.transpose(1, 2) * self.scale
            s = s.masked_fill(torch.ones(s.shape[-2:], dtype=torch.bool, device=DEV).triu(1), -math.inf)
            outs.append((s.softmax(-1) @ vs).transpose(0, 1))
        return self.logits(x, torch.cat(outs))


def new_cache(policy, seqs, blocks, kv):
    nb, dt = seqs * blocks, torch.float8_e4m3fn if kv == "fp8" else torch.bfloat16
    g = torch.Generator(DEV).manual_seed(1)
    return dict(k=torch.zeros((nb, policy.hkv, BS, policy.d), device=DEV).to(dt),
                v=torch.zeros((nb, policy.hkv, policy.d, BS), device=DEV).to(dt),
                scales=torch.zeros((2, nb, policy.hkv), device=DEV) if kv == "fp8" else None,
                table=torch.randperm(nb, generator=g, device=DEV).to(torch.int32).view(seqs, blocks))


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def rollout(policy, prompts, steps, kv, gen):
    """Sampled responses [B, steps] and their log-probabilities."""
    B, lens = len(prompts), [len(p) for p in prompts]
    cache = new_cache(policy, B, (max(lens) + steps) // BS + 1, kv)
    offsets = int32([0] + torch.tensor(lens).cumsum(0).tolist())
    z = policy.paged(cache, torch.cat(prompts), int32(lens), offsets)[(offsets[1:] - 1).long()]
    length, tokens, logps = int32(lens), [], []
    for _ in range(steps):
        t = torch.multinomial(z.softmax(-1), 1, generator=gen)[:, 0]
        lp = torch.empty(B, device=DEV)
        _lib.token_logprobs(z, t, lp)
        tokens.append(t)
        logps.append(lp)
        length = length + 1
        z = policy.paged(cache, t, length)
    return torch.stack(tokens, 1), torch.stack(logps, 1)


def main(kv="bf16", prompts=4, samples=8, steps=24, updates=5, seed=0):
    gen = torch.Generator(DEV).manual_seed(seed)
    policy, ref = Policy(), Policy()
    vocab = policy.w["emb"].shape[0]
    asked = [torch.randint(0, vocab, (5 + 9 * i,), generator=gen, device=DEV) for i in range(prompts)]
    asked = [p for p in asked for _ in range(samples)]
    answers, old = rollout(policy, asked, steps, kv, gen)

    # GRPO: a response's advantage is its reward among its prompt's samples; here even tokens are rewarded
    reward = (answers % 2 == 0).float().mean(1).view(prompts, samples)
    adv = ((reward - reward.mean(1, True)) / (reward.std(1, keepdim=True) + 1e-4)).view(-1, 1).expand(-1, steps)

    # packed sequences: position i predicts token i + 1; prompt positions and the last one have no target
    seqs = [torch.cat([p, a]) for p, a in zip(asked, answers)]
    lens = [len(s) for s in seqs]
    tokens, positions = torch.cat(seqs), torch.cat([torch.arange(n, device=DEV) for n in lens]).to(torch.int32)
    target = torch.full((len(tokens),), -1, device=DEV)
    first = torch.tensor([len(p) - 1 for p in asked]) + torch.tensor([0] + lens[:-1]).cumsum(0)
    at = (first[:, None] + torch.arange(steps)).to(DEV)
    target[at] = answers
    per_token = {}
    for name, x in (("old", old), ("adv", adv), ("w", torch.full_like(old, 1 / old.numel()))):
        per_token[name] = torch.zeros(len(tokens), device=DEV)
        per_token[name][at] = x

    # reference log-probabilities: one pass over every token, keys and values into a paged cache of its own
    offsets = int32([0] + torch.tensor(lens).cumsum(0).tolist())
    z = ref.paged(new_cache(ref, len(seqs), max(lens) // BS + 1, kv), tokens, int32(lens), offsets)
    ref_logp, entropy = (torch.empty(len(tokens), device=DEV) for _ in range(2))
    _lib.token_logprobs(z, target, ref_logp, entropy)

    history, stats = [], torch.empty(8, device=DEV)
    for t in policy.w.values():
        t.requires_grad_()
    logp = torch.empty(len(tokens), device=DEV)
    for i in range(updates):
        z = policy.train_logits(tokens, positions, lens)
        grad = torch.empty_like(z)
        _lib.policy_loss(z.detach(), target, per_token["old"], per_token["adv"], per_token["w"], stats, grad, logp,
                         ref_logprobs=ref_logp, clip_high=0.28, kl_coef=0.01)
        z.backward(grad)
        if i == 0:
            first_gap = float((logp - per_token["old"])[at].abs().max())
        with torch.no_grad():
            for t in policy.w.values():
                t -= 0.5 * t.grad
                t.grad = None
        history.append(dict(zip(_lib.POLICY_STATS, stats.tolist())))
        print(f"update {i}: " + "  ".join(f"{k} {v:.4f}" for k, v in history[-1].items()), flush=True)
    print(f"rollout's log-probabilities ({kv} cache) against the trainer's: at most {first_gap:.3f} apart; "
          f"mean entropy {float(entropy[at].mean()):.3f}; device status {_lib.read_device_status()}")
    return history, first_gap


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--kv", choices=("bf16", "fp8"), default="bf16")
    main(ap.parse_args().kv)
