"""Calls whose workgroups count their arrivals, so that the last one finishes the work: one stream's calls of several
kinds share the counts, and give the same bits whatever call came before, as captured calls (finished by launches of
their own) do."""

import pytest
import torch

from tests._ops_ref import angles

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    from paper_2605_20863_amd import _lib
    return _lib


def rand(*shape, dtype=torch.float32, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(DEV).to(dtype)


def policy(lib, T, V, dtype, grad=True):
    z, y = rand(T, V, dtype=dtype, seed=T), (torch.arange(T, device=DEV) * 7) % V
    y[::5] = -1  # rows that take no part arrive too
    old, adv, w = rand(T, seed=1) - 5, rand(T, seed=2), torch.full((T,), 1 / T, device=DEV)
    out = [torch.zeros(8, device=DEV), torch.zeros_like(z) if grad else None, torch.zeros(T, device=DEV)]
    return lambda: lib.policy_loss(z, y, old, adv, w, out[0], out[1], out[2], kl_coef=0.0), [t for t in out if t is not None]


def logp(lib, T, V, dtype):
    z, y = rand(T, V, dtype=dtype, seed=T + 1), (torch.arange(T, device=DEV) * 11) % V
    y[::3] = -1
    out = [torch.zeros(T, device=DEV), torch.zeros(T, device=DEV)]
    return lambda: lib.token_logprobs(z, y, *out), out


def backward(lib, T, hq, hkv, d, dtype):
    q, k, gq, gk = (rand(T, h, d, dtype=dtype, seed=i) for i, h in enumerate((hq, hkv, hq, hkv)))
    w = rand(d, seed=9) + 1
    table, pos = angles(64, d).to(DEV), (torch.arange(T, device=DEV) % 64).to(torch.int32)
    out = [torch.zeros_like(q), torch.zeros_like(k), torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)]
    return lambda: lib.qk_norm_rope_backward(q, k, w, w, table, pos, gq, gk, *out), out


def decode(lib, B, tokens):
    hq, hkv, d, width = 8, 2, 128, (tokens + 15) // 16
    q, kc, vc = (rand(*s, dtype=torch.bfloat16, seed=i) for i, s in
                 enumerate(((B, hq, d), (B * width, hkv, 16, d), (B * width, hkv, d, 16))))
    table = torch.arange(B * width, dtype=torch.int32, device=DEV).view(B, width)
    lens, out = torch.full((B,), tokens, dtype=torch.int32, device=DEV), torch.zeros_like(q)
    return lambda: lib.paged_decode_attention(q, kc, vc, table, lens, None, out, d ** -0.5), [out]


def makers(lib):
    bf, f = torch.bfloat16, torch.float32
    return [policy(lib, 1, 100, bf), policy(lib, 130, 9000, bf), policy(lib, 31, 700, f), policy(lib, 32, 300, bf, False),
            policy(lib, 33, 300, bf), policy(lib, 513, 300, bf), policy(lib, 32, 50_001, bf), policy(lib, 32, 16_384, bf), policy(lib, 3, 50_001, f), policy(lib, 5, 17, f), decode(lib, 2, 700),
            policy(lib, 512, 9000, f), policy(lib, 170, 140_001, bf),
            logp(lib, 1, 60_000, bf), logp(lib, 192, 20_000, bf), logp(lib, 193, 20_000, bf), logp(lib, 64, 50_001, f),
            backward(lib, 1, 8, 2, 64, bf), backward(lib, 64, 28, 4, 128, bf), backward(lib, 51, 33, 3, 128, f), decode(lib, 5, 300),
            backward(lib, 400, 4, 1, 64, f)]


def test_same_bits_after_any_call_and_captured(lib):
    s = torch.cuda.Stream(DEV)
    with torch.cuda.stream(s):
        calls = makers(lib)
        for f, _ in calls:
            f()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            for f, _ in calls:
                f()
        for _, out in calls:
            for t in out:
                t.zero_()
        graph.replay()
        s.synchronize()
        want = [[t.clone() for t in out] for _, out in calls]
        g = torch.Generator().manual_seed(3)
        for turn in range(6):
            order = torch.randperm(len(calls), generator=g).tolist()
            for i in order + order[::-1]:
                for t in calls[i][1]:
                    t.zero_()
                calls[i][0]()
            s.synchronize()
            for i, (_, out) in enumerate(calls):
                assert all(torch.equal(a, b) for a, b in zip(out, want[i])), (turn, i)
            if turn % 2:
                for _, out in calls:
                    for t in out:
                        t.zero_()
                graph.replay()
                s.synchronize()
                for i, (_, out) in enumerate(calls):
                    assert all(torch.equal(a, b) for a, b in zip(out, want[i])), ("graph", turn, i)


def test_values_of_counted_calls(lib):
    """Against 64 bits: the weights' gradients (sums of up to 64 parts) and the loss's sums."""
    call, (_, _, dwq, dwk) = backward(lib, 51, 33, 3, 128, torch.float32)
    call()
    q, k, gq, gk = (rand(51, h, 128, seed=i).double() for i, h in enumerate((33, 3, 33, 3)))
    a = angles(64, 128).to(DEV).double()[torch.arange(51, device=DEV) % 64][:, None]
    cos, sin = a.chunk(2, -1)
    for x, g, got in ((q, gq, dwq), (k, gk, dwk)):
        u, v = g.chunk(2, -1)
        back = torch.cat([u * cos + v * sin, v * cos - u * sin], -1)
        n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        want, size = (back * n).sum((0, 1)), (back * n).abs().sum((0, 1))
        # a wave adds a few rows' terms, a workgroup four waves: below 32 roundings of a term, and the norm's
        assert ((got.double() - want).abs() <= 64 * 2.0 ** -24 * size).all()
    call, (stats, _, logps) = policy(lib, 31, 700, torch.float32)
    call()
    live = torch.ones(31, device=DEV)
    live[::5] = 0
    assert abs(float(stats[7]) - float(live.sum()) / 31) < 1e-6
    y = ((torch.arange(31, device=DEV) * 7) % 700)
    want = torch.log_softmax(rand(31, 700, seed=31).double(), 1)[torch.arange(31, device=DEV), y]
    assert ((logps.double() - want) * live).abs().max() < 1e-5
