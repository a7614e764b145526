"""The torch module's calls of include/pda_lm.h: made where every argument is as it has to be, any other left to the
binding's own checks; captured and replayed calls; calls on other streams."""

import pytest
import torch

from paper_2605_20863_amd import _lib as L
from tests.test_ops_torch import Entry

M = L._pda_torch
DEV = "cuda:0"
BF, INT32 = torch.bfloat16, torch.int32


def calls(dev, T=6, H=256, V=999, K=7):
    """Every call's name and arguments."""
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g).to(dev)  # noqa: E731
    e = lambda *s: torch.zeros(s, device=dev)  # noqa: E731
    x, w = r(T, H + 64).to(BF)[:, :H], 1 + 0.1 * r(H)
    z = r(T, V + 1)[:, :V]
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).to(INT32).to(dev)
    return {
        "add_rms_norm": [x, w, e(T, H).to(torch.float8_e4m3fn), r(T, H).to(BF), e(T, H).to(BF), e(T, 2), 1e-6],
        "add_rms_norm_backward": [x, w, r(T, H).to(BF), e(T, H).to(BF), e(H), r(T, H).to(BF), 1e-6],
        "top_logprobs": [z, e(T, K).to(INT32), e(T, K), torch.arange(T, device=dev), e(T), e(T), 0.8],
        "distill_loss": [z, ids, torch.log_softmax(r(T, K), 1) - 0.1, torch.full((T,), 1 / T, device=dev), e(6), e(T, V), e(T), 0.3, True,
                         0.8, 2.0],
    }


NAMES = ["add_rms_norm", "add_rms_norm_backward", "top_logprobs", "distill_loss"]
# arguments whose last dimension nothing else fixes, or that fix others' (wider ones are refused by those)
WIDER = {("add_rms_norm", 0), ("add_rms_norm_backward", 0), ("top_logprobs", 0)}


def run(name, args):
    if name == "distill_loss":
        return L.distill_loss(*args[:7], reverse=args[7], rest=args[8], temperature=args[9], grad_scale=args[10])
    if name == "top_logprobs":
        return L.top_logprobs(*args[:6], temperature=args[6])
    return getattr(L, name)(*args[:6], eps=args[6])


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
    """One argument at a time is of another type, shape, device or layout; the binding's checks refuse it too."""
    e, f = Entry(), getattr(M, name)
    good = calls(DEV)[name]
    assert f(e.address, 0, *good) == 0 and e.count == 1
    assert f(None, 0, *good) is None and f(e.address, "0", *good) is None
    for i, x in enumerate(good):
        if isinstance(x, torch.Tensor):
            bad = [x.cpu(), x.to(torch.float64), x[..., None], x.new_zeros(x.shape + (2,))[..., 0], x.new_zeros(1).expand(x.shape)]
            if (name, i) not in WIDER:
                bad.append(x.new_zeros(x.shape[:-1] + (x.shape[-1] + 1,)))
        elif isinstance(x, bool):
            bad = []
        else:
            bad = [None, "x", good[0]]
        for b in bad:
            args = good[:i] + [b] + good[i + 1:]
            assert f(e.address, 0, *args) is None, (i, b if not isinstance(b, torch.Tensor) else (b.shape, b.dtype, b.stride()))
            if isinstance(b, torch.Tensor):
                with pytest.raises((ValueError, TypeError)):
                    run(name, args)
    assert e.count == 1
    failing = Entry(-1)
    assert f(failing.address, 0, *good) == -1


def arguments_left_out(name, args):
    args = list(args)
    for i in {"add_rms_norm": (3, 4), "add_rms_norm_backward": (4, 5), "top_logprobs": (3, 4, 5), "distill_loss": (5, 6)}[name]:
        args[i] = None
    return args


@pytest.mark.gpu
@pytest.mark.parametrize("less", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_same_results_as_through_the_checks(name, less, monkeypatch):
    """An ordinary call is made by the module; made by the binding instead it gives the same bits."""
    direct, checked = calls(DEV)[name], calls(DEV)[name]
    if less:
        direct, checked = arguments_left_out(name, direct), arguments_left_out(name, checked)
    real = L._launch

    def no_launch(*_):
        raise AssertionError("left to the binding")

    monkeypatch.setattr(L, "_launch", no_launch)
    run(name, direct)
    monkeypatch.setattr(L, "_launch", real)
    monkeypatch.setattr(L, "_direct", lambda *_: None)
    run(name, checked)
    torch.cuda.synchronize()
    for a, b in zip(direct, checked):
        if isinstance(a, torch.Tensor):
            assert torch.equal(a.float(), b.float())


@pytest.mark.gpu
def test_scales_of_other_shapes():
    x, w = torch.randn((3, 256), device=DEV), torch.ones(256, device=DEV)
    o = torch.empty((3, 256), dtype=torch.uint8, device=DEV)
    a, b = torch.empty(3, device=DEV), torch.empty((3, 1), device=DEV)
    L.add_rms_norm(x, w, o, scales=a)
    L.add_rms_norm(x, w, o, scales=b)
    assert torch.equal(a, b[:, 0])
    for bad in (None, torch.empty((3, 3), device=DEV), torch.empty((3, 0), device=DEV), torch.empty((2, 2), device=DEV)):
        with pytest.raises(ValueError, match="scales"):
            L.add_rms_norm(x, w, o, scales=bad)
    with pytest.raises(ValueError, match="scales"):
        L.add_rms_norm(x, w, torch.empty_like(x), scales=a)
    with pytest.raises(L.PdaError, match="scale_group"):
        L.add_rms_norm(x, w, o, scales=torch.empty((3, 8), device=DEV))
    with pytest.raises(ValueError, match="targets"):
        L.top_logprobs(x, torch.empty((3, 2), dtype=INT32, device=DEV), torch.empty((3, 2), device=DEV), logprobs=a)
    with pytest.raises(L.PdaError, match="num_top"):
        L.top_logprobs(x, torch.empty((3, 300), dtype=INT32, device=DEV), torch.empty((3, 300), device=DEV))


SIZES = [dict(T=3, H=4096, V=131_072, K=20), dict(T=1, H=64, V=500, K=1), dict(T=40, H=1000, V=9000, K=256),
         dict(T=300, H=2048, V=20_001, K=64)]


def outputs(name, args):
    return [args[i] for i in {"add_rms_norm": (2, 4, 5), "add_rms_norm_backward": (3, 4), "top_logprobs": (1, 2, 4, 5),
                              "distill_loss": (4, 5, 6)}[name]]


def sized(dev, size):
    c = calls(dev, **size)
    if size["H"] % 128:
        c["add_rms_norm"][5] = torch.zeros(size["T"], device=dev)
    else:
        c["add_rms_norm"][5] = torch.zeros((size["T"], size["H"] // (128 if size["H"] > 64 else 64)), device=dev)
    return c


@pytest.mark.gpu
@pytest.mark.parametrize("size", range(len(SIZES)))
def test_captured_and_replayed(size):
    """All four calls in one graph, replayed with the program's own calls on other sizes between: each replay gives the
    eager call's bits, for inputs that changed in place too."""
    c = sized(DEV, SIZES[size])
    other = sized(DEV, SIZES[(size + 1) % len(SIZES)])
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for n in NAMES:
            run(n, c[n])
            run(n, other[n])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        for n in NAMES:
            run(n, c[n])
    for turn in range(4):
        for n in NAMES:
            c[n][0].mul_(0.9 if turn % 2 else -1.1)  # the inputs of the next replay
        want = {}
        for n in NAMES:
            run(n, c[n])
            want[n] = [t.float().clone() for t in outputs(n, c[n])]
            for t in outputs(n, c[n]):
                t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in NAMES:
            for a, b in zip(outputs(n, c[n]), want[n]):
                assert torch.equal(a.float(), b), (n, turn)
            run(n, other[n])


@pytest.mark.gpu
def test_calls_on_two_streams_at_once():
    """Each stream has a workspace of its own: calls that run beside each other do not touch each other's."""
    sets = [sized(DEV, SIZES[i]) for i in (0, 2)]
    want = []
    for c in sets:
        for n in NAMES:
            run(n, c[n])
        want.append({n: [t.float().clone() for t in outputs(n, c[n])] for n in NAMES})
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for c, s in zip(sets, streams):
        for n in NAMES:
            for t in outputs(n, c[n]):
                t.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip(sets, streams):
            with torch.cuda.stream(s):
                for n in NAMES:
                    run(n, c[n])
    torch.cuda.synchronize()
    for c, w in zip(sets, want):
        for n in NAMES:
            for a, b in zip(outputs(n, c[n]), w[n]):
                assert torch.equal(a.float(), b), n
