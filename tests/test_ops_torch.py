"""The torch module of the calls around attention: it makes a call where every argument is as it has to be, and
leaves any other to the binding's own checks."""

import ctypes

import pytest
import torch

from paper_2605_20863_amd import _lib as L

M = L._pda_torch
DEV = "cuda:0"
INT32 = torch.int32


def rope_args(dev, T=3, hq=4, hkv=2, d=64):
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn((T, (hq + 2 * hkv), d), generator=g).to(dev)
    w = [1 + 0.1 * torch.randn(d, generator=g).to(dev) for _ in range(2)]
    table = torch.randn((16, d), generator=g).to(dev)
    return dict(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], wq=w[0], wk=w[1], table=table,
                pos=torch.arange(T, dtype=INT32, device=dev), v=qkv[:, hq + hkv:])


def calls(dev):
    """Every call's name and arguments."""
    a, f = rope_args(dev), dict(device=dev)
    T, hq, d = a["q"].shape
    hkv = a["k"].shape[1]
    empty = lambda *s: torch.zeros(s, **f)  # noqa: E731
    norm = [a["q"], a["k"], a["wq"], a["wk"], a["table"], a["pos"]]
    logits, y = torch.linspace(-1, 1, 60, **f).view(6, 10)[:, :9], torch.arange(6, **f)
    row = [torch.linspace(-2, 0, 6, **f), torch.ones(6, **f), torch.full((6,), 1 / 6, **f)]
    return {
        "paged_qk_norm_rope_append": [a["q"], a["k"], a["v"], a["wq"], a["wk"], a["table"], None,
                                      empty(T, hkv, 16, d), empty(T, hkv, d, 16), None,
                                      torch.arange(T, dtype=INT32, **f).view(T, 1), torch.ones(T, dtype=INT32, **f),
                                      empty(T, hq, d), 1e-6, False, None, 0],
        "qk_norm_rope": norm + [empty(T, hq, d), empty(T, hkv, d), 1e-6, False],
        "qk_norm_rope_backward": norm + [a["q"] * 2, a["k"] * 2, empty(T, hq, d), empty(T, hkv, d), empty(d), empty(d), 1e-6, True],
        "token_logprobs": [logits, y, empty(6), empty(6), 0.5],
        "policy_loss": [logits, y, *row, empty(8), empty(6, 9), empty(6), empty(6), row[0] - 0.1, 0.2, 0.2, 3.0, 0.1, 0.01, 1.0, 2.0],
    }


class Entry:
    """An entry that counts its calls and does nothing else."""

    def __init__(self, code=0):
        self.count = 0

        def f(*_):
            self.count += 1
            return code

        self.f = ctypes.CFUNCTYPE(ctypes.c_int)(f)
        self.address = ctypes.cast(self.f, ctypes.c_void_p).value


# arguments whose last dimension nothing else fixes: cos_sin, block_table, logits
WIDER = {("paged_qk_norm_rope_append", 5), ("paged_qk_norm_rope_append", 10), ("qk_norm_rope", 4), ("qk_norm_rope_backward", 4),
         ("token_logprobs", 0)}
NAMES = ["paged_qk_norm_rope_append", "qk_norm_rope", "qk_norm_rope_backward", "token_logprobs", "policy_loss"]


@pytest.mark.parametrize("name", NAMES)
def test_refuses_host_tensors_and_what_is_no_tensor(name):
    e, args = Entry(), calls("cpu")[name]
    f = getattr(M, name)
    assert f(e.address, 0, *args) is None
    assert f(e.address, 0, *[None] * len(args)) is None
    assert f(e.address, 0, *[1.5] * len(args)) is None
    assert f(e.address, 0) is None and f() is None
    assert e.count == 0


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_refuses_each_wrong_argument(name):
    """One argument at a time is of another type, shape, device or layout."""
    e, f = Entry(), getattr(M, name)
    good = calls(DEV)[name]
    assert f(e.address, 0, *good) == 0 and e.count == 1
    assert f(None, 0, *good) is None and f(e.address, "0", *good) is None
    for i, x in enumerate(good):
        if isinstance(x, torch.Tensor):
            bad = [x.cpu(), x.to(torch.float64), x[..., None], x.new_zeros(x.shape + (2,))[..., 0], x.tolist(),
                   x.new_zeros(1).expand(x.shape)]
            if (name, i) not in WIDER:
                bad.append(x.new_zeros(x.shape[:-1] + (x.shape[-1] + 1,)))
        elif x is None:
            bad = [torch.zeros(7, device=DEV), 3]
        elif isinstance(x, bool):
            bad = []
        else:
            bad = [None, "x", good[0]]
        for b in bad:
            args = good[:i] + [b] + good[i + 1:]
            assert f(e.address, 0, *args) is None, (i, b if not isinstance(b, torch.Tensor) else (b.shape, b.dtype, b.stride()))
    assert e.count == 1
    failing = Entry(-1)
    assert f(failing.address, 0, *good) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_same_results_as_through_the_checks(name, monkeypatch):
    """An ordinary call is made by the module; made by the binding instead it gives the same bits."""
    direct, checked = calls(DEV)[name], calls(DEV)[name]
    real = L._launch

    def no_launch(*_):
        raise AssertionError("left to the binding")

    def run(args):
        if name == "policy_loss":
            kw = dict(zip(("clip_low", "clip_high", "dual_clip", "kl_coef", "entropy_coef", "temperature", "grad_scale"), args[10:]))
            return L.policy_loss(*args[:9], ref_logprobs=args[9], **kw)
        return getattr(L, name)(*args)

    monkeypatch.setattr(L, "_launch", no_launch)
    run(direct)
    monkeypatch.setattr(L, "_launch", real)
    monkeypatch.setattr(L, "_direct", lambda *_: None)
    run(checked)
    torch.cuda.synchronize()
    for a, b in zip(direct, checked):
        if isinstance(a, torch.Tensor):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_library_errors_are_raised():
    args = calls(DEV)["token_logprobs"]
    with pytest.raises(L.PdaError, match="temperature"):
        L.token_logprobs(*args[:4], temperature=0.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    L.token_logprobs(*args[:4], stream=s)
    s.synchronize()
    want = torch.log_softmax(args[0].double(), 1)[torch.arange(6), args[1]]
    assert (args[2] - want).abs().max() < 1e-5
