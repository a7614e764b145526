"""The residual stream's norm and its gradient at the ends of their ranges (64-bit references and bounds of
tests/_lm_ref.py)."""

import pytest
import torch

from tests import _lm_ref as R
from tests.test_norm_gpu import DEV, EPS, TYPES, lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu


# rows' sizes: below the sum's limit (3.4e38 / H), past it, close to the mean's limit, past that (a norm of 0)
SIZES = [1.0, 1e16, 1e17, 5e17, 1e18, 9e18, 1.5e19, 4e19, 1e25, 1e37]


def large(T, H, dt, seed):
    x = rand((T, H), seed)
    x = x / (x * x).mean(dim=1, keepdim=True).sqrt()
    size = torch.tensor([SIZES[(i * 7 + 3) % len(SIZES)] for i in range(T)])
    x = (x * size[:, None]).clamp(-3e38, 3e38).to(dt)
    return x, size > 2e19


@pytest.mark.parametrize("out", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", [(13, 64), (21, 512), (30, 1000), (11, 2048), (15, 4096), (1030, 4096), (12, 8192), (11, 16384), (10, 32768)])
def test_rows_whose_squares_sum_past_float32(lib, T, H, t, out):
    """The norm of every row whose mean square float32 holds, and 0 for larger ones, with weights that take |h w| past it."""
    x, zero = large(T, H, TYPES[t], H)
    w = 50 * (1 + rand((H,), 2, amp=0.2))
    o = torch.empty((T, H), dtype=TYPES[out], device=DEV)
    y, bound = R.norm(x, w, EPS)
    y[zero], bound[zero] = 0, 0
    if out == "fp8":
        for group in (g for g in (0, 64, 128) if g == 0 or H % g == 0):
            s = torch.empty((T, H // group if group else 1), device=DEV)
            lib.add_rms_norm(x.to(DEV), w.to(DEV), o, scales=s, eps=EPS)
            scales, ds, z, dz = R.fp8(y, bound, group)
            R.near(s, scales, ds, torch.float32, "scales")
            assert ((o.float().cpu().double() - z).abs() <= dz).all()
    else:
        lib.add_rms_norm(x.to(DEV), w.to(DEV), o, eps=EPS)
        R.near(o, y, bound, TYPES[out], "norm")
    if t == "bf16" and out == "bf16":  # the sum as it is kept, with its residual
        half, kept = x / 2, torch.empty_like(x, device=DEV)
        lib.add_rms_norm(half.to(DEV), w.to(DEV), o, half.to(DEV), kept, eps=EPS)
        assert torch.equal(kept.cpu(), (half.float() * 2).to(torch.bfloat16))
        R.near(o, *[torch.where(zero[:, None], 0.0, v) for v in R.norm(kept.cpu(), w, EPS)], torch.bfloat16, "norm of the sum")


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", [(13, 64), (21, 512), (30, 1000), (11, 2048), (15, 4096), (1030, 4096), (12, 8192), (11, 16384), (10, 32768),
                                 (600, 16384)])
def test_gradient_of_rows_whose_squares_sum_past_float32(lib, T, H, t, add):
    """As the forward's: r is that of every row whose mean square float32 holds, and 0 for larger ones."""
    dt = TYPES[t]
    h, zero = large(T, H, dt, H)
    w, g = 1 + rand((H,), 2, amp=0.2), rand((T, H), 3, dt, 0.1)
    q = rand((T, H), 4, dt, 1e-3) if add else None
    dh, dw = torch.empty((T, H), dtype=dt, device=DEV), torch.empty(H, device=DEV)
    lib.add_rms_norm_backward(h.to(DEV), w.to(DEV), g.to(DEV), dh, dw, None if q is None else q.to(DEV), eps=EPS)
    want, bound, _, _ = R.norm_grad(h, w, g, q, EPS)
    want[zero] = q[zero].double() if add else 0.0
    R.near(dh, want, bound, dt, "gradient of the stream")
    _, _, wdw, dwb = R.norm_grad(h[~zero], w, g[~zero], None, EPS)
    R.near(dw, wdw, dwb, torch.float32, "gradient of the weights")


@pytest.mark.parametrize("group", [0, 64, 128])
@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", [(4, 256), (4, 4096), (1100, 4096), (3, 16384)])
def test_nan_rows_in_fp8(lib, T, H, t, group):
    """One NaN, of either sign, in the stream, the residual or the weights: every code of the row is 0x7f, every scale 2^-126."""
    x, res, w = rand((T, H), 1, TYPES[t]), rand((T, H), 2, TYPES[t]), rand((H,), 3)
    nan = torch.tensor([0x7FC0, 0xFFC0 - 0x10000], dtype=torch.int16).view(torch.bfloat16).to(TYPES[t])
    assert not nan[0].signbit() and nan[1].signbit()
    x[0, 9], x[1, H - 1], res[2, 77] = nan[0], nan[1], nan[1]

    def run(w):
        o = torch.empty((T, H), dtype=torch.uint8, device=DEV)
        s = torch.full((T, H // group) if group else (T, 1), 9.0, device=DEV)
        lib.add_rms_norm(x.to(DEV), w.to(DEV), o, res.to(DEV), scales=s, eps=EPS)
        return o.cpu(), s.cpu()

    codes, scales = run(w)
    assert (codes[:3] == 0x7F).all(), codes[:3].unique()
    assert (scales[:3] == 2.0 ** -126).all()
    assert (codes[3:] & 0x7F != 0x7F).all() and (scales[3:] > 2.0 ** -126).all()
    # a weight's NaN is its column's alone, and its group's scale that of the others
    x[:3], res[2] = rand((3, H), 4, TYPES[t]), rand((1, H), 5, TYPES[t])
    plain, plain_scales = run(w.clone().index_fill_(0, torch.tensor([70]), 0.0))
    for v in nan:
        codes, scales = run(w.clone().index_fill_(0, torch.tensor([70]), float(v)) if not v.signbit()
                            else torch.where(torch.arange(H) == 70, v.float(), w))
        assert (codes[:, 70] == 0x7F).all(), codes[:, 70].unique()
        rest = torch.arange(H) != 70
        assert torch.equal(codes[:, rest], plain[:, rest]) and torch.equal(scales, plain_scales)


def far_apart(x, stride):
    """x on the device as rows `stride` elements apart, 9 between them where anything is read back."""
    full = torch.empty((x.shape[0] - 1) * stride + x.shape[1], dtype=x.dtype, device=DEV)
    rows = full.as_strided(x.shape, (stride, 1))
    rows.copy_(x)
    return rows


@pytest.mark.parametrize("out", ["bf16", "fp8"])
@pytest.mark.parametrize("T,H,stride", [(700, 1024, 3_100_008), (5, 8192, (1 << 29) + 8)])
def test_rows_past_2_to_the_31_elements(lib, T, H, stride, out):
    """Offsets of rows that 32 bits do not hold: the bits of the same rows side by side."""
    assert (T - 1) * stride > 1 << 31
    x, res, g, w = (rand((T, H), i, torch.bfloat16) for i in (1, 2, 3, 4))
    w = w[0].float().to(DEV)

    def run(place):
        o, s = place(torch.zeros((T, H), dtype=TYPES[out])), place(torch.zeros_like(x))
        scales = torch.empty(T, device=DEV) if out == "fp8" else None
        lib.add_rms_norm(place(x), w, o, place(res), s, scales, eps=EPS)
        o, dh, dw = o.contiguous(), place(torch.zeros_like(x)), torch.empty(H, device=DEV)
        lib.add_rms_norm_backward(s, w, place(g), dh, dw, place(res), eps=EPS)
        return o.view(torch.uint8), s.contiguous(), scales, dh.contiguous(), dw

    for a, b in zip(run(lambda v: far_apart(v, stride)), run(lambda v: v.to(DEV))):
        assert a is None or torch.equal(a, b)
