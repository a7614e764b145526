"""On-policy distillation of a one-layer student on random weights, through the library's operators:

    rollout   the student answers prompts: chunks and tokens through norm, rotation, cache append and paged attention
    teacher   every token of the answers at once over its own paged cache; the most likely words of each position and
              their log-probabilities (top_logprobs) are all that is kept of its logits
    update    the student's forward with the residual stream's norms and their gradient (add_rms_norm as an autograd
              function), the loss against the teacher's lists and its gradient at the logits (distill_loss)

    python3 examples/distill_step.py [--reverse 0.5]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from paper_2605_20863_amd import _lib  # noqa: E402
import rlvr_step  # noqa: E402

DEV = "cuda"


class AddRMSNorm(torch.autograd.Function):
    """(norm of x + residual, x + residual); gradients by the library."""

    @staticmethod
    def forward(ctx, x, residual, weight):
        out, stream = torch.empty_like(x), torch.empty_like(x)
        _lib.add_rms_norm(x, weight, out, residual, stream)
        ctx.save_for_backward(stream, weight)
        return out, stream

    @staticmethod
    def backward(ctx, g_out, g_stream):
        stream, weight = ctx.saved_tensors
        g, dw = torch.empty_like(stream), torch.empty(weight.shape, device=weight.device)
        _lib.add_rms_norm_backward(stream, weight, g_out.contiguous(), g, dw, g_stream.contiguous())
        return g, g, dw.to(weight.dtype)


class Model(rlvr_step.Policy):
    """rlvr_step's model with norms of the residual stream before attention and before the head."""

    def __init__(self, seed=0, **kw):
        super().__init__(seed=seed, **kw)
        width = self.w["emb"].shape[1]
        self.w["n1"], self.w["n2"] = (torch.ones(width, device=DEV) for _ in "12")

    def heads(self, tokens, dtype):
        x = self.w["emb"][tokens]
        n, x = AddRMSNorm.apply(torch.zeros_like(x), x, self.w["n1"])
        y = (n @ self.w["qkv"]).to(dtype).view(len(tokens), -1, self.d)
        return x, y[:, :self.hq], y[:, self.hq:self.hq + self.hkv], y[:, self.hq + self.hkv:]

    def logits(self, x, attended):
        n, _ = AddRMSNorm.apply(attended.float().reshape(len(x), -1) @ self.w["out"], x, self.w["n2"])
        return n @ self.w["head"]


def teacher_lists(teacher, tokens, lens, target, places, temperature):
    """The teacher's most likely words of every position that has a target, [tokens, places] each; other rows are empty."""
    offsets = rlvr_step.int32([0] + torch.tensor(lens).cumsum(0).tolist())
    cache = rlvr_step.new_cache(teacher, len(lens), max(lens) // rlvr_step.BS + 1, "bf16")
    z = teacher.paged(cache, tokens, rlvr_step.int32(lens), offsets)
    ids = torch.empty((len(tokens), places), dtype=torch.int32, device=DEV)
    logp = torch.empty(ids.shape, device=DEV)
    _lib.top_logprobs(z, ids, logp, target, temperature=temperature)
    return ids, logp


def batch(student, prompts, samples, steps, gen):
    """(packed tokens, positions, lengths, targets): answers of the student; prompt positions and the last have no target."""
    vocab = student.w["emb"].shape[0]
    asked = [torch.randint(0, vocab, (5 + 9 * i,), generator=gen, device=DEV) for i in range(prompts)]
    asked = [p for p in asked for _ in range(samples)]
    answers, _ = rlvr_step.rollout(student, asked, steps, "bf16", gen)
    seqs = [torch.cat([p, a]) for p, a in zip(asked, answers)]
    lens = [len(s) for s in seqs]
    target = torch.cat([torch.cat([torch.full((len(p) - 1,), -1, device=DEV), a, torch.full((1,), -1, device=DEV)])
                        for p, a in zip(asked, answers)])
    return torch.cat(seqs), torch.cat([torch.arange(n, device=DEV) for n in lens]).to(torch.int32), lens, target


def gradients(student, data, lists, reverse, temperature):
    """One pass of the update: (stats by name, gradients by weight)."""
    tokens, positions, lens, target = data
    live = (target >= 0).float()
    for t in student.w.values():
        t.requires_grad_()
    z = student.train_logits(tokens, positions, lens)
    grad, stats = torch.empty_like(z), torch.empty(6, device=DEV)
    _lib.distill_loss(z.detach(), *lists, live / live.sum(), stats, grad, reverse=reverse, temperature=temperature)
    z.backward(grad)
    out = {n: t.grad for n, t in student.w.items()}
    for t in student.w.values():
        t.grad = None
        t.requires_grad_(False)
    return dict(zip(_lib.DISTILL_STATS, stats.tolist())), out


def main(reverse=0.0, prompts=4, samples=4, steps=24, updates=5, places=32, temperature=1.0, seed=0):
    gen = torch.Generator(DEV).manual_seed(seed)
    student, teacher = Model(seed=0), Model(seed=1)
    for t in teacher.w.values():
        t.requires_grad_(False)
    history = []
    for i in range(updates):
        with torch.no_grad():
            data = batch(student, prompts, samples, steps, gen)
            lists = teacher_lists(teacher, data[0], data[2], data[3], places, temperature)
        stats, grads = gradients(student, data, lists, reverse, temperature)
        with torch.no_grad():
            for n, t in student.w.items():
                t -= 0.5 * grads[n]
        history.append(stats)
        print(f"update {i}: " + "  ".join(f"{k} {v:.4f}" for k, v in stats.items()), flush=True)
    print(f"device status {_lib.read_device_status()}")
    return history


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--reverse", type=float, default=0.0)
    main(ap.parse_args().reverse)
