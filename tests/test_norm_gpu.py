"""GPU parity of the residual stream's norm and its gradient (include/pda_lm.h) against 64-bit references with bounds
from the arithmetic (tests/_lm_ref.py)."""

import math

import pytest
import torch

from tests import _lm_ref as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
EPS = 1e-6


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    from paper_2605_20863_amd import _lib
    _lib.read_device_status()
    return _lib


def rand(shape, seed, dtype=torch.float32, amp=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * amp).to(dtype)


def apart(x, pad):
    """x on the device as a view of rows `pad` elements apart, with NaN between them."""
    if pad == 0:
        return x.to(DEV)
    full = torch.full((x.shape[0], x.shape[1] + pad), math.nan).to(x.dtype).to(DEV)
    full[:, :x.shape[1]] = x.to(DEV)
    return full[:, :x.shape[1]]


# one vector, around a wave's and a workgroup's vectors, beside every variant's limit
WIDTHS = [8, 64, 120, 504, 512, 520, 1000, 2048, 2056, 4096, 4104, 8192, 8200, 16384, 16392, 32768]


def inputs(T, H, dt, wt, seed, loud=True):
    x, res, w = rand((T, H), seed, dt), rand((T, H), seed + 1, dt, 3.0), (1 + rand((H,), seed + 2, amp=0.2)).to(wt)
    if loud and H > 64:
        res[:, 7] *= 30
    return x, res, w


@pytest.mark.parametrize("t,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("H", WIDTHS)
def test_norm(lib, t, out, H):
    for T, pad, wt, add in ((1, 0, torch.float32, True), (5, 8, torch.bfloat16, True), (67, 0, torch.bfloat16, False)):
        print(f"[norm] {t} -> {out} H={H} T={T}", flush=True)
        x, res, w = inputs(T, H, TYPES[t], wt, H + T)
        o = torch.full((T, H + pad), 9.0, dtype=TYPES[out], device=DEV)
        s = torch.full((T, H + pad), 9.0, dtype=TYPES[t], device=DEV)
        if add:
            lib.add_rms_norm(apart(x, pad), w.to(DEV), o[:, :H], apart(res, pad), s[:, :H], eps=EPS)
            x = (x.float() + res.float()).to(TYPES[t])
            assert torch.equal(s[:, :H].cpu(), x)
        else:
            lib.add_rms_norm(apart(x, pad), w.to(DEV), o[:, :H], eps=EPS)
        y, bound = R.norm(x, w, EPS)
        R.near(o[:, :H], y, bound, TYPES[out], "norm")
        assert (o[:, H:] == 9.0).all() and (s[:, H:] == 9.0).all()


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("H,group", [(h, g) for h in WIDTHS for g in (0, 64, 128) if g == 0 or h % g == 0])
def test_norm_fp8(lib, t, H, group):
    for T, pad in ((1, 0), (6, 8), (35, 0)):
        print(f"[norm fp8] {t} H={H} group={group} T={T}", flush=True)
        x, res, w = inputs(T, H, TYPES[t], TYPES[t], H + T)
        x[0, : min(H, 128)] = 0
        res[0, : min(H, 128)] = 0  # groups of zeros
        o = torch.zeros((T, H + pad), dtype=torch.uint8, device=DEV)
        scales = torch.full((T, H // group) if group else (T,), 9.0, device=DEV)
        stream = torch.empty((T, H), dtype=TYPES[t], device=DEV)
        lib.add_rms_norm(apart(x, pad), w.to(DEV), o[:, :H], apart(res, pad), stream, scales, eps=EPS)
        y, bound = R.norm(stream.cpu(), w, EPS)
        s, ds, z, dz = R.fp8(y, bound, group)
        R.near(scales.view(T, -1), s, ds, torch.float32, "scales")
        got = o[:, :H].contiguous().view(torch.float8_e4m3fn).cpu().double()
        assert ((got - z).abs() <= dz).all(), float(((got - z).abs() - dz).max())
        assert (o[:, H:] == 0).all()
        typed, again = torch.empty((T, H), dtype=TYPES["fp8"], device=DEV), torch.empty_like(scales)
        lib.add_rms_norm(stream, w.to(DEV), typed, scales=again, eps=EPS)  # the norm of what was kept
        assert torch.equal(typed.view(torch.uint8), o[:, :H]) and torch.equal(again, scales)


@pytest.mark.parametrize("H", [1000, 4096, 8192])
def test_norm_in_place(lib, H):
    x, res, w = (v.to(DEV) for v in inputs(9, H, torch.bfloat16, torch.bfloat16, 1))
    o, s = torch.empty_like(x), torch.empty_like(x)
    lib.add_rms_norm(x, w, o, res, s)
    a, b = x.clone(), res.clone()
    lib.add_rms_norm(a, w, a, b, b)  # out over x, the stream over the residual
    assert torch.equal(a, o) and torch.equal(b, s)
    a, b = x.clone(), res.clone()
    lib.add_rms_norm(a, w, b, b, a)  # out over the residual, the stream over x
    assert torch.equal(b, o) and torch.equal(a, s)
    a, b = x.clone(), torch.empty_like(x)
    lib.add_rms_norm(a, w, b, res)  # the stream is not kept
    assert torch.equal(b, o) and torch.equal(a, x)


@pytest.mark.parametrize("out", ["bf16", "fp8"])
def test_special_rows(lib, out):
    """Zeros, NaN, infinities and values whose squares pass float32 keep to their own rows."""
    H = 4096
    x = rand((6, H), 5)
    x[1] = 0
    x[2, 17] = math.nan
    x[3, 100] = math.inf
    x[4] *= 1e25
    o = torch.empty((6, H), dtype=TYPES[out], device=DEV)
    scales = torch.empty((6, H // 128), device=DEV) if out == "fp8" else None
    w = torch.ones(H, device=DEV)
    lib.add_rms_norm(x.to(DEV), w, o, scales=scales)
    y = o.float().cpu()
    assert (y[1] == 0).all() and (y[4] == 0).all() and y[2].isnan().all()
    assert y[3, 100].isnan() and (y[3].nan_to_num(0.0) == 0).all()
    if scales is not None:
        assert (scales[1] == 2.0 ** -126).all() and (scales[2] == 2.0 ** -126).all()
    alone = torch.empty((1, H), dtype=TYPES[out], device=DEV)
    for r in (0, 5):
        lib.add_rms_norm(x[r:r + 1].to(DEV), w, alone, scales=None if scales is None else scales[:1])
        assert torch.equal(alone.view(torch.uint8), o[r:r + 1].view(torch.uint8))


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("H", WIDTHS)
def test_gradient(lib, t, H):
    for T, pad, wt, add in ((1, 0, torch.float32, False), (5, 8, torch.bfloat16, True), (130, 0, torch.bfloat16, True)):
        print(f"[norm gradient] {t} H={H} T={T}", flush=True)
        dt = TYPES[t]
        q, h, w = inputs(T, H, dt, wt, H + T)
        g = rand((T, H), 3, dt, 0.1)
        dh, dw = torch.full((T, H + pad), 9.0, dtype=dt, device=DEV), torch.full((H,), 9.0, device=DEV)
        lib.add_rms_norm_backward(apart(h, pad), w.to(DEV), apart(g, pad), dh[:, :H], dw, apart(q, pad) if add else None, eps=EPS)
        want, bound, wdw, dwb = R.norm_grad(h, w, g, q if add else None, EPS)
        R.near(dh[:, :H], want, bound, dt, "gradient of the stream")
        R.near(dw, wdw, dwb, torch.float32, "gradient of the weights")
        assert (dh[:, H:] == 9.0).all()
        # over grad_out and over grad_residual, and without the weights': the same
        a, b = g.to(DEV), q.to(DEV)
        lib.add_rms_norm_backward(h.to(DEV), w.to(DEV), a, a, None, b if add else None, eps=EPS)
        assert torch.equal(a, dh[:, :H])
        if add:
            again = torch.empty_like(dw)
            lib.add_rms_norm_backward(h.to(DEV), w.to(DEV), g.to(DEV), b, again, b, eps=EPS)
            assert torch.equal(b, dh[:, :H]) and torch.equal(again, dw)


@pytest.mark.parametrize("T,H", [(4097, 128), (3000, 2048), (2100, 4096), (1500, 16384), (1029, 8), (1023, 4096), (1024, 4096), (1025, 8192),
                                 (1100, 6000), (4500, 1000), (300, 32768)])
def test_gradient_of_many_rows(lib, T, H):
    """More rows than workgroups."""
    q, h, w = inputs(T, H, torch.bfloat16, torch.bfloat16, T, loud=False)
    g = rand((T, H), 3, torch.bfloat16, 0.1)
    dh, dw = torch.empty((T, H), dtype=torch.bfloat16, device=DEV), torch.empty(H, device=DEV)
    lib.add_rms_norm_backward(h.to(DEV), w.to(DEV), g.to(DEV), dh, dw, q.to(DEV), eps=EPS)
    want, bound, wdw, dwb = R.norm_grad(h, w, g, q, EPS)
    R.near(dh, want, bound, torch.bfloat16, "gradient of the stream")
    R.near(dw, wdw, dwb, torch.float32, "gradient of the weights")
    o, s = torch.empty_like(dh), torch.empty_like(dh)
    lib.add_rms_norm(h.to(DEV), w.to(DEV), o, q.to(DEV), s, eps=EPS)
    y, bound = R.norm(s.cpu(), w, EPS)
    R.near(o, y, bound, torch.bfloat16, "norm")


@pytest.mark.parametrize("T,H,out", [(8191, 4096, "bf16"), (8192, 4096, "bf16"), (8192, 4096, "fp8"), (32800, 1024, "bf16"), (4100, 8192, "fp8"),
                                     (70000, 480, "bf16"), (1100, 32768, "bf16")])
def test_calls_past_the_caches(lib, T, H, out):
    """Both sides of the size from which rows are loaded and stored past the caches: as the same rows in smaller calls."""
    dev = lambda seed, amp=1.0: torch.randn((T, H), generator=torch.Generator(DEV).manual_seed(seed), device=DEV).mul_(amp).to(torch.bfloat16)  # noqa: E731
    x, res, g = dev(1), dev(2, 3.0), dev(3, 0.1)
    w = (1 + rand((H,), 4, amp=0.2)).to(DEV)
    o, s, dh, dw = torch.empty((T, H), dtype=TYPES[out], device=DEV), torch.empty_like(x), torch.empty_like(x), torch.empty(H, device=DEV)
    scales = torch.empty(T, device=DEV) if out == "fp8" else None
    lib.add_rms_norm(x, w, o, res, s, scales, eps=EPS)
    lib.add_rms_norm_backward(s, w, g, dh, dw, res, eps=EPS)
    assert torch.equal(s, (x.float() + res.float()).to(torch.bfloat16))
    total = torch.zeros(H, dtype=torch.float64)
    for i in range(0, T, 2000):
        at = slice(i, min(T, i + 2000))
        a, b, c, d = torch.empty_like(o[at]), torch.empty_like(dh[at]), torch.empty(H, device=DEV), scales if scales is None else torch.empty_like(scales[at])
        lib.add_rms_norm(s[at], w, a, scales=d, eps=EPS)
        lib.add_rms_norm_backward(s[at], w, g[at], b, c, res[at], eps=EPS)
        assert torch.equal(a.view(torch.uint8), o[at].view(torch.uint8)) and torch.equal(b, dh[at])
        total += c.cpu().double()
    _, _, wdw, dwb = R.norm_grad(s[:2000].cpu(), w.cpu(), g[:2000].cpu(), None, EPS)
    # more rows of the same kind: terms and bounds grow with their number, sums in a workgroup with its rows
    assert ((dw.cpu().double() - total).abs() <= 2 * dwb * (T / 2000 + 1) * (1 + T / 512 / 24) + 2 * R.EPS24 * total.abs()).all()


def test_gradient_against_differences(lib):
    """The norm's own differences agree with its gradient along random directions."""
    T, H = 7, 264
    q, h, w = inputs(T, H, torch.float32, torch.float32, 2)
    g = rand((T, H), 3)
    dh, dw = torch.empty((T, H), device=DEV), torch.empty(H, device=DEV)
    lib.add_rms_norm_backward(h.to(DEV), w.to(DEV), g.to(DEV), dh, dw, q.to(DEV), eps=EPS)

    def value(h, w):  # what the gradient is of: the stream goes on, the norm's result goes on
        y, _ = R.norm(h, w, EPS)
        return float((y * g.double()).sum() + (h * q.double()).sum())

    for seed in range(4):
        v, u, e = rand((T, H), 10 + seed).double(), rand((H,), 20 + seed).double(), 1e-5
        slope = (value(h.double() + e * v, w.double() + e * u) - value(h.double() - e * v, w.double() - e * u)) / (2 * e)
        dot = float((dh.cpu().double() * v).sum() + (dw.cpu().double() * u).sum())
        size = float((dh.cpu().double() * v).abs().sum() + (dw.cpu().double() * u).abs().sum())
        # float32 gradients, and differences of second order: 1e-5^2 of third derivatives of order 1
        assert abs(slope - dot) <= 64 * R.EPS24 * size + 1e-8 * (1 + size)


@pytest.mark.parametrize("out", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("H", [64, 512, 2048, 4096, 8192, 16384, 32768])
def test_a_row_is_the_same_in_every_call(lib, H, out):
    """Whatever the other rows, and however many: bit for bit, in calls around every limit on their number."""
    T = 1030 if H < 16384 else 40
    x, res, w = inputs(T, H, torch.bfloat16, torch.bfloat16, H)
    x, res, w = x.to(DEV), res.to(DEV), w.to(DEV)

    def run(n):
        o, s = torch.empty((n, H), dtype=TYPES[out], device=DEV), torch.empty((n, H), dtype=torch.bfloat16, device=DEV)
        scales = torch.empty(n, device=DEV) if out == "fp8" else None
        lib.add_rms_norm(x[:n], w, o, res[:n], s, scales, eps=EPS)
        return o.view(torch.uint8), s, scales

    want = run(T)
    for n in (1, 3, 4, 37, 1023, 1024):
        if n < T:
            for a, b in zip(run(n), want):
                assert a is None or torch.equal(a, b[:n]), n


@pytest.mark.parametrize("out", ["bf16", "fp8"])
def test_zeros_without_eps(lib, out):
    """A row of zeros has no norm with eps 0: NaN in its own row alone; its gradient likewise."""
    x, _, w = inputs(5, 256, torch.bfloat16, torch.float32, 3)
    x[2] = 0
    x, w = x.to(DEV), w.to(DEV)
    o, dx = torch.empty((5, 256), dtype=TYPES[out], device=DEV), torch.empty((5, 256), dtype=torch.bfloat16, device=DEV)
    lib.add_rms_norm(x, w, o, scales=torch.empty(5, device=DEV) if out == "fp8" else None, eps=0.0)
    lib.add_rms_norm_backward(x, w, x, dx, eps=0.0)
    for r in range(5):
        assert bool(o[r].float().isnan().all()) == (r == 2) and bool(dx[r].float().isnan().any()) == (r == 2)
        assert r == 2 or not o[r].float().isnan().any()


def test_no_rows(lib):
    H = 64
    e = torch.empty((0, H), dtype=torch.bfloat16, device=DEV)
    w, dw = torch.ones(H, device=DEV), torch.full((H,), 9.0, device=DEV)
    lib.add_rms_norm(e, w, e, e, e)
    lib.add_rms_norm_backward(e, w, e, e, dw, e)
    assert (dw == 0).all()
