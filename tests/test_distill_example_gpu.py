"""examples/distill_step.py: the operators in a run together. It runs, and the gradients of its weights are those of the
same step with norms, teacher's lists and loss in plain torch."""

import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available()
    spec = importlib.util.spec_from_file_location("distill_step", os.path.join(ROOT, "examples", "distill_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("reverse", [0.0, 0.5])
def test_runs(example, reverse):
    history = example.main(reverse, updates=2)
    for h in history:
        assert all(math.isfinite(v) for v in h.values()) and abs(h["weight"] - 1) < 1e-5
        assert 0 < h["teacher_mass"] <= 1 + 1e-5 and 0 < h["student_mass"] <= 1 + 1e-5
        assert h["forward"] > 0 and h["reverse"] > 0
    assert example._lib.read_device_status() == 0


class Plain(torch.autograd.Function):
    """Marks where the plain step's norm stands in for the library's (a function of the same name and arguments)."""

    @staticmethod
    def apply(x, residual, weight):  # noqa: D102
        h = x + residual
        return h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + 1e-6) * weight, h


def plain_loss(z, ids, tau, w, b, temperature):
    """Divergences over the listed words and the rest, from their definition."""
    logp = torch.log_softmax(z.double() / temperature, dim=1)
    loss = 0.0
    for t in torch.nonzero(w)[:, 0].tolist():
        i, ta = ids[t].long(), tau[t].double()
        lp, p = logp[t, i], logp[t, i].exp()
        out = torch.ones(z.shape[1], dtype=torch.bool, device=z.device)
        out[i] = False
        rest, tr = logp[t][out].logsumexp(0), (1 - ta.exp().sum()).clamp(min=2.0 ** -24)
        f = (ta.exp() * (ta - lp)).sum() + tr * (tr.log() - rest)
        r = (p * (lp - ta)).sum() + rest.exp() * (rest - tr.log())
        loss = loss + w[t].double() * ((1 - b) * f + b * r)
    return loss


@pytest.mark.parametrize("reverse", [0.0, 0.5])
def test_gradients(example, reverse, monkeypatch):
    gen = torch.Generator("cuda").manual_seed(3)
    student, teacher = example.Model(seed=0), example.Model(seed=1)
    with torch.no_grad():
        data = example.batch(student, 3, 2, 10, gen)
        ids, tau = example.teacher_lists(teacher, data[0], data[2], data[3], 16, 0.9)
    live = data[3] >= 0
    assert ((ids >= 0).all(dim=1) == live).all() and (tau[~live] == -math.inf).all()
    stats, got = example.gradients(student, data, (ids, tau), reverse, 0.9)
    monkeypatch.setattr(example, "AddRMSNorm", Plain)
    for t in student.w.values():
        t.requires_grad_()
    z = student.train_logits(*data[:3])
    loss = plain_loss(z, ids, tau, live.float() / live.sum(), reverse, 0.9)
    loss.backward()
    # float32 products of up to 512 terms on both sides
    loss = loss.detach()
    assert abs(float(loss) - stats["loss"]) < 1e-5 * max(1.0, abs(float(loss)))
    for n, t in student.w.items():
        assert (got[n] - t.grad).norm() <= 1e-4 * t.grad.norm() + 1e-7, n
