"""GPU parity of the head norms with rotation (include/pda_ops.h): as a training
forward, its gradient, and into the paged cache, against 64-bit references with
bounds from the arithmetic (tests/_ops_ref.py)."""

import numpy as np
import pytest
import torch

from tests import _ops_ref as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device")
    from paper_2605_20863_amd import _lib
    _lib.read_device_status()
    return _lib


def rand(shape, dtype, seed, amp=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * amp).to(dtype)


def weights(d, dtype, norm, seed=9):
    if not norm:
        return None, None
    return tuple((1 + 0.3 * rand((d,), torch.float32, seed + i)).to(dtype) for i in range(2))


def dev(t):
    return None if t is None else t.to(DEV)


# head counts that fill a wave's rows, cross from q to k inside one, and are odd
SHAPES = [(1, 1, 1), (1, 28, 4), (3, 5, 3), (37, 4, 4), (130, 64, 8), (2100, 33, 1)]


@pytest.mark.parametrize("d,rot,inter", [(64, 64, False), (64, 32, True), (128, 128, False), (128, 96, False), (128, 16, True)])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_forward_and_gradient(lib, t, norm, d, rot, inter):
    dt = TYPES[t]
    for n, (T, hq, hkv) in enumerate(SHAPES):
        print(f"[rope] {t} norm={norm} D={d} R={rot} inter={inter} T={T} heads={hq}/{hkv}", flush=True)
        q, k = rand((T, hq, d), dt, 10 * n), rand((T, hkv, d), dt, 10 * n + 1, 3.0)
        gq, gk = rand((T, hq, d), dt, 10 * n + 2, 1e-3), rand((T, hkv, d), dt, 10 * n + 3)
        wq, wk = weights(d, dt if n % 2 else torch.float32, norm)
        pos = torch.randint(0, 500, (T,), generator=torch.Generator().manual_seed(n), dtype=torch.int32)
        table = R.angles(500, rot)
        args = [dev(x) for x in (q, k, wq, wk, table, pos)]
        qo, ko = torch.full((T, hq, d), 7.0, dtype=dt, device=DEV), torch.full((T, hkv, d), 7.0, dtype=dt, device=DEV)
        lib.qk_norm_rope(*args, qo, ko, interleaved=inter)
        dq, dk = torch.full_like(qo, 7.0), torch.full_like(ko, 7.0)
        dwq, dwk = (torch.full((d,), 7.0, device=DEV) for _ in "qk")
        lib.qk_norm_rope_backward(*args, dev(gq), dev(gk), dq, dk, dwq, dwk, interleaved=inter)
        for x, w, y, g, dx, dw, name in ((q, wq, qo, gq, dq, dwq, "q"), (k, wk, ko, gk, dk, dwk, "k")):
            want, bound = R.norm_turn(x, w, table, pos, 1e-6, inter)
            R.assert_within(y, want, bound, dt, f"{name} T={T}")
            want, bound, ww, wb = R.norm_turn_grad(x, w, table, pos, g, 1e-6, inter)
            R.assert_within(dx, want, bound, dt, f"d{name} T={T}")
            if norm:
                R.assert_within(dw, ww, wb, torch.float32, f"d{name} weight T={T}")
    assert lib.read_device_status() == 0


def test_gradient_against_differences(lib):
    """The forward's own differences along random directions, float32."""
    T, hq, hkv, d, rot = 5, 6, 2, 128, 64
    q, k = rand((T, hq, d), torch.float32, 1), rand((T, hkv, d), torch.float32, 2)
    gq, gk = rand((T, hq, d), torch.float32, 3), rand((T, hkv, d), torch.float32, 4)
    wq, wk = weights(d, torch.float32, True)
    table, pos = R.angles(64, rot), torch.arange(T, dtype=torch.int32) * 7
    c = [dev(x) for x in (q, k, wq, wk, table, pos)]
    dq, dk = torch.empty_like(c[0]), torch.empty_like(c[1])
    dwq, dwk = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    lib.qk_norm_rope_backward(*c, dev(gq), dev(gk), dq, dk, dwq, dwk)

    def value(step, direction):
        x = [c[i] + step * direction[i] for i in range(4)]
        qo, ko = torch.empty_like(c[0]), torch.empty_like(c[1])
        lib.qk_norm_rope(*x, c[4], c[5], qo, ko)
        return float((qo.double() * dev(gq).double()).sum() + (ko.double() * dev(gk).double()).sum())

    h = 1e-2
    for seed in range(4):
        u = [dev(rand(x.shape, torch.float32, 50 + 4 * seed + i)) for i, x in enumerate((q, k, wq, wk))]
        slope = (value(h, u) - value(-h, u)) / (2 * h)
        want = sum(float((a.double() * b.double()).sum()) for a, b in zip(u, (dq, dk, dwq, dwk)))
        # central differences: h^2 / 6 of the third derivative, and float32 outputs
        # (about 4,000 of size 1) over 2 h: 1e-3 and 2e-4 of the sums' sizes
        size = sum(float((a.double() * b.double()).square().sum().sqrt()) for a, b in zip(u, (dq, dk, dwq, dwk)))
        assert abs(slope - want) <= 2e-3 * size + 2e-3, (slope, want, size)


def test_views_of_packed_projections_and_in_place(lib):
    T, hq, hkv, d = 19, 6, 2, 64
    for dt in (torch.bfloat16, torch.float32):
        qkv = rand((T, (hq + 2 * hkv + 1) * d), dt, 3).to(DEV)
        x = qkv.view(T, -1, d)
        q, k = x[:, :hq], x[:, hq:hq + hkv]
        wq, wk = (dev(w) for w in weights(d, dt, True))
        table, pos = R.angles(T, 64).to(DEV), torch.arange(T, dtype=torch.int32, device=DEV)
        qo, ko = torch.empty((T, hq, d), dtype=dt, device=DEV), torch.empty((T, hkv, d), dtype=dt, device=DEV)
        lib.qk_norm_rope(q, k, wq, wk, table, pos, qo, ko)
        gq, gk = torch.empty_like(qo).normal_(), torch.empty_like(ko).normal_()
        dq, dk = torch.empty_like(qo), torch.empty_like(ko)
        dwq, dwk = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
        lib.qk_norm_rope_backward(q, k, wq, wk, table, pos, gq, gk, dq, dk, dwq, dwk)
        # gradients into the packed projection's gradient, then over the incoming ones
        packed = torch.full_like(qkv, 5.0)
        y = packed.view(T, -1, d)
        lib.qk_norm_rope_backward(q, k, wq, wk, table, pos, gq, gk, y[:, :hq], y[:, hq:hq + hkv], dwq, dwk)
        assert torch.equal(y[:, :hq], dq) and torch.equal(y[:, hq:hq + hkv], dk)
        assert (y[:, hq + hkv:] == 5.0).all()
        lib.qk_norm_rope_backward(q, k, wq, wk, table, pos, gq, gk, gq, gk, dwq, dwk)
        assert torch.equal(gq, dq) and torch.equal(gk, dk)
        rest = x[:, hq + hkv:].clone()
        lib.qk_norm_rope(q, k, wq, wk, table, pos, q, k)
        assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(x[:, hq + hkv:], rest)
        with pytest.raises(ValueError, match="overlap"):  # the strides of an expanded tensor
            lib.qk_norm_rope(qo[:1].expand(T, hq, d), ko, wq, wk, table, pos, dq, dk)


def test_positions_outside_the_table(lib):
    T, d = 4, 64
    q, k = rand((T, 2, d), torch.float32, 1).to(DEV), rand((T, 1, d), torch.float32, 2).to(DEV)
    table = R.angles(8, d).to(DEV)
    qo, ko, want_q, want_k = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k)
    lib.qk_norm_rope(q, k, None, None, table, torch.tensor([-3, 8, 7, 2 ** 31 - 1], dtype=torch.int32, device=DEV), qo, ko)
    assert lib.read_device_status() == lib.STATUS_BAD_POSITION
    lib.qk_norm_rope(q, k, None, None, table, torch.tensor([0, 7, 7, 7], dtype=torch.int32, device=DEV), want_q, want_k)
    assert torch.equal(qo, want_q) and torch.equal(ko, want_k) and lib.read_device_status() == 0


def test_rows_without_content(lib):
    """A row of zeros stays zeros, its gradient finite; a row with a NaN or an infinity keeps it to itself."""
    d = 128
    q = rand((3, 4, d), torch.bfloat16, 1)
    q[0, 0] = 0
    q[1, 1, 5] = float("nan")
    q[2, 2, 7] = float("inf")
    k = torch.zeros((3, 1, d), dtype=torch.bfloat16)
    wq, wk = weights(d, torch.bfloat16, True)
    table, pos = R.angles(3, d), torch.arange(3, dtype=torch.int32)
    qo, ko = torch.empty_like(q, device=DEV), torch.empty_like(k, device=DEV)
    lib.qk_norm_rope(dev(q), dev(k), dev(wq), dev(wk), dev(table), dev(pos), qo, ko)
    assert (qo[0, 0] == 0).all() and (ko == 0).all()
    bad = torch.zeros(3, 4, dtype=torch.bool)
    bad[1, 1] = bad[2, 2] = True
    assert torch.equal(qo.isfinite().all(dim=-1).cpu(), ~bad)
    g = torch.ones_like(qo)
    dq, dk = torch.empty_like(qo), torch.empty_like(ko)
    dw = torch.empty(d, device=DEV)
    lib.qk_norm_rope_backward(dev(q), dev(k), dev(wq), dev(wk), dev(table), dev(pos), g, torch.ones_like(ko), dq, dk, dw,
                              torch.empty_like(dw))
    assert torch.equal(dq.isfinite().all(dim=-1).cpu(), ~bad) and dk.isfinite().all()


def test_no_tokens(lib):
    q, k = torch.empty((0, 4, 64), device=DEV), torch.empty((0, 2, 64), device=DEV)
    table, pos = R.angles(4, 64).to(DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    w = torch.ones(64, device=DEV)
    dw = [torch.full((64,), 3.0, device=DEV) for _ in "qk"]
    lib.qk_norm_rope(q, k, w, w, table, pos, q, k)
    lib.qk_norm_rope_backward(q, k, w, w, table, pos, q, k, q, k, *dw)
    assert (dw[0] == 0).all() and (dw[1] == 0).all()


# ------------------------------------------------------------- into the cache


def cache_of(kv, nb, hkv, d, seed):
    """Host caches with earlier contents: K [nb, hkv, 16, d], V [nb, hkv, d, 16], scales."""
    rng = np.random.default_rng(seed)
    shapes = (nb, hkv, 16, d), (nb, hkv, d, 16)
    if kv == "fp8":
        k, v = (torch.from_numpy(rng.integers(0, 0x7F, s).astype(np.uint8)) for s in shapes)
        return k, v, torch.from_numpy(rng.uniform(0.001, 0.02, (2, nb, hkv)).astype(np.float32))
    return tuple(torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(TYPES[kv]) for s in shapes) + (None,)


def check_append(lib, kv, t, lens, counts, hq, hkv, d, rot, inter, norm, seed, positions=False, even=False, amp=None,
                 out=None):
    """One append against the reference; returns the device caches."""
    rng = np.random.default_rng(seed)
    dt, B = TYPES[t], len(lens)
    lens, counts = np.asarray(lens), np.asarray(counts)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    T, width = int(offsets[-1]), int(max(1, (lens.max() + 15) // 16))
    nb = B * width + 2
    table = rng.permutation(nb)[:B * width].reshape(B, width).astype(np.int32)
    q = rand((T, hq, d), dt, seed)
    a = torch.from_numpy(rng.choice(amp or [1.0], (T, 1, 1)).astype(np.float32))
    k, v = ((rand((T, hkv, d), torch.float32, seed + i) * a).to(dt) for i in (1, 2))
    wq, wk = weights(d, dt, norm)
    P = int(max(lens.max(), 1)) + 40
    cs = R.angles(P, rot)
    kc, vc, sc = cache_of(kv, nb, hkv, d, seed + 3)
    gk, gv, gs = kc.clone().to(DEV), vc.clone().to(DEV), None if sc is None else sc.clone().to(DEV)
    where = R.places(None if even else offsets, lens, T, width)
    pos = torch.tensor([max(p, 0) for _, _, p in where], dtype=torch.int32) + (17 if positions else 0)
    ot = out or dt
    qo = torch.full((T, hq, d), 9.0, dtype=ot, device=DEV)
    lib.paged_qk_norm_rope_append(dev(q), dev(k), dev(v), dev(wq), dev(wk), dev(cs),
                                  None if even else torch.from_numpy(offsets.astype(np.int32)).to(DEV), gk, gv, gs,
                                  torch.from_numpy(table).to(DEV), torch.from_numpy(lens.astype(np.int32)).to(DEV), qo,
                                  interleaved=inter, positions=dev(pos) if positions else None)
    what = f"{kv}/{t} D={d} R={rot} seed={seed}"
    want, bound = R.norm_turn(q, wq, cs, pos, 1e-6, inter)
    R.assert_within(qo, want, bound, ot, f"q {what}")
    want_k, bound_k = R.norm_turn(k, wk, cs, pos, 1e-6, inter)
    written = torch.zeros((nb, 16), dtype=torch.bool)
    tiles = {}
    for t_row, b, p in where:
        if p >= 0:
            written[table[b, p // 16], p % 16] = True
            tiles.setdefault((b, p // 16), []).append((p % 16, t_row))
    hk, hv = gk.cpu(), gv.cpu()
    rows_k, rows_v, kept = hk, hv.transpose(2, 3), ~written[:, None, :, None]
    if kv != "fp8":
        assert torch.equal(rows_k[kept.expand_as(rows_k)], kc[kept.expand_as(kc)]), f"K outside {what}"
        assert torch.equal(rows_v[kept.expand_as(rows_v)], vc.transpose(2, 3)[kept.expand_as(rows_v)]), f"V outside {what}"
        for (b, j), rows in tiles.items():
            slot, row = (torch.tensor(x) for x in zip(*rows))
            at = int(table[b, j])
            R.assert_within(rows_k[at, :, slot], want_k[row].transpose(0, 1), bound_k[row].transpose(0, 1), TYPES[kv], f"K {what}")
            assert torch.equal(rows_v[at, :, slot], v[row].transpose(0, 1).to(TYPES[kv])), f"V {what}"
        return gk, gv, gs
    hs = gs.cpu().numpy()
    ref_v, ref_s = vc.transpose(2, 3).contiguous().numpy(), sc.numpy().copy()
    touched = np.zeros((nb,), bool)
    for (b, j), rows in tiles.items():
        at = int(table[b, j])
        touched[at] = True
        slots, row = [s for s, _ in rows], [r for _, r in rows]
        for h in range(hkv):
            ref_v[at, h], ref_s[1, at, h] = R.write_fp8_tile(ref_v[at, h], ref_s[1, at, h], v[row, h].float().numpy(), slots, True)
            # K: the values differ by the arithmetic's bound, so a code may be the neighbour's
            x, e = want_k[row, h], bound_k[row, h]
            amax, old, s = float(x.abs().max()), float(sc[0, at, h]), float(hs[0, at, h])
            if slots[0] == 0 or amax > 448 * old:
                assert abs(s - max(amax / 448, R.MIN_SCALE)) <= float(e.max()) / 448 + 2.0 ** -23 * s, what
            else:
                assert s == np.float32(old), what
            got = R.decode(hk[at, h].numpy()).astype(np.float64) * s
            step = np.maximum(np.abs(x.numpy()) * 2.0 ** -4, s * 2.0 ** -10) + e.numpy()  # half a step of E4M3
            assert (np.abs(got[slots] - x.numpy()) <= step * 1.001).all(), f"K {what}"
            if slots[0] > 0:  # earlier tokens: as they were, or under the raised scale
                was = kc[at, h, :slots[0]].numpy()
                now = hk[at, h, :slots[0]].numpy()
                if s == np.float32(old):
                    assert np.array_equal(now, was), f"earlier K {what}"
                else:
                    assert np.array_equal(now, R.encode((R.decode(was) * np.float32(old)).astype(np.float32), np.float32(s))), f"earlier K {what}"
            assert torch.equal(hk[at, h, slots[-1] + 1:], kc[at, h, slots[-1] + 1:]), f"later K {what}"
    assert np.array_equal(rows_v.contiguous().numpy(), ref_v), f"V codes {what}"
    assert np.array_equal(hs[1], ref_s[1]), f"V scales {what}"
    assert torch.equal(hk[~touched], kc[~touched]) and np.array_equal(hs[0][~touched], ref_s[0][~touched]), f"K outside {what}"
    return gk, gv, gs


@pytest.mark.parametrize("d,rot,inter", [(64, 64, False), (128, 128, False), (128, 64, True), (64, 48, False)])
@pytest.mark.parametrize("kv,t", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("fp8", "bf16"), ("fp8", "f32"), ("f32", "bf16")])
def test_append(lib, kv, t, d, rot, inter):
    amp = [0.01, 0.5, 3.0, 40.0]
    print(f"[append] {kv} {t} D={d} R={rot}", flush=True)
    # a decode step, every slot of a block; a first token; a full block
    check_append(lib, kv, t, list(range(1, 34)), [1] * 33, 5, 3, d, rot, inter, True, 1, even=True, amp=amp)
    # speculative verification: 4 tokens, ending anywhere in a block
    check_append(lib, kv, t, [4, 5, 16, 17, 19, 20, 31, 64], [4] * 8, 8, 2, d, rot, inter, False, 2, even=True, amp=amp)
    # ragged chunks: none, one, part of a tile, whole tiles, several with odd ends, whole sequences
    check_append(lib, kv, t, [40, 7, 1, 16, 48, 100, 33, 200, 64], [0, 7, 1, 16, 32, 37, 2, 200, 15], 28, 4, d, rot, inter, True,
                 3, amp=amp)
    # positions of their own, more tokens than the sequence holds, an empty sequence
    check_append(lib, kv, t, [20, 3, 0, 90], [6, 5, 0, 70], 16, 1, d, rot, inter, True, 4, positions=True)
    # other type of the rotated queries
    check_append(lib, kv, t, [77, 15], [77, 15], 4, 4, d, rot, inter, True, 5, out=torch.float32 if t == "bf16" else torch.bfloat16)
    assert lib.read_device_status() == 0


@pytest.mark.parametrize("kv", ["f32", "bf16", "fp8"])
def test_append_of_many_sequences(lib, kv):
    """More sequences than a wave searches in one round, many of them without new tokens."""
    rng = np.random.default_rng(7)
    lens = rng.integers(0, 40, 4500)
    counts = np.minimum(rng.choice([0, 0, 0, 1, 1, 2, 5, 20], 4500), lens)
    check_append(lib, kv, "f32" if kv == "f32" else "bf16", lens, counts, 2, 1, 64, 64, False, True, 11)
    assert lib.read_device_status() == 0


@pytest.mark.parametrize("kv", ["f32", "bf16", "fp8"])
def test_one_token_equals_kv_append(lib, kv):
    """Unrotated (angle 0) and without norms, an append of one token per sequence leaves what paged_kv_append leaves."""
    B, hkv, d, width = 40, 4, 128, 4
    rng = np.random.default_rng(3)
    lens = rng.integers(1, 16 * width + 1, B).astype(np.int32)
    table = rng.permutation(B * width + 3)[:B * width].reshape(B, width).astype(np.int32)
    dt = torch.float32 if kv == "f32" else torch.bfloat16
    amp = torch.from_numpy(rng.choice([0.01, 1.0, 30.0], (B, hkv, 1)).astype(np.float32))
    k, v = ((rand((B, hkv, d), torch.float32, i) * amp).to(dt).to(DEV) for i in (1, 2))
    kc, vc, sc = cache_of(kv, B * width + 3, hkv, d, 5)
    a = [dev(x) if x is None else x.clone().to(DEV) for x in (kc, vc, sc)]
    b = [dev(x) if x is None else x.clone().to(DEV) for x in (kc, vc, sc)]
    q = rand((B, 8, d), dt, 3).to(DEV)
    qo = torch.empty_like(q)
    lib.paged_qk_norm_rope_append(q, k, v, None, None, R.angles(1, d).to(DEV), None, *a, torch.from_numpy(table).to(DEV),
                                  torch.from_numpy(lens).to(DEV), qo, positions=torch.zeros(B, dtype=torch.int32, device=DEV))
    lib.paged_kv_append(k, v, *b, torch.from_numpy(table).to(DEV), torch.from_numpy(lens - 1).to(DEV))
    assert torch.equal(q, qo)
    for x, y in zip(a, b):
        assert x is None or torch.equal(x, y)


def test_steps_of_decoding_fp8(lib):
    """48 one-token steps into empty fp8 tiles: caches and scales equal paged_kv_append's after every one."""
    B, hkv, d, width = 6, 2, 64, 3
    table = torch.randperm(B * width, generator=torch.Generator().manual_seed(1)).view(B, width).int().to(DEV)
    kc, vc, sc = cache_of("fp8", B * width, hkv, d, 1)
    a, b = ([x.clone().to(DEV) for x in (kc, vc, sc)] for _ in range(2))
    one, zero = R.angles(1, d).to(DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    for step in range(48):
        amp = torch.exp(rand((B, hkv, 1), torch.float32, step, 1.5))
        k, v = ((rand((B, hkv, d), torch.float32, 100 + 2 * step + i) * amp).to(DEV) for i in range(2))
        q = rand((B, 4, d), torch.float32, step).to(DEV)
        lib.paged_qk_norm_rope_append(q, k, v, None, None, one, None, *a, table, zero + step + 1, q, positions=zero)
        lib.paged_kv_append(k, v, *b, table, zero + step)
        for x, y in zip(a, b):
            assert torch.equal(x, y), step


def test_device_checks(lib):
    """Bad block ids, lengths past the table, offsets that go back: nothing outside is written, and the status says so."""
    B, hq, hkv, d, width, nb = 3, 4, 2, 64, 2, 8
    q, k, v = (rand((6, h, d), torch.bfloat16, h).to(DEV) for h in (hq, hkv, hkv))
    cs = R.angles(64, d).to(DEV)
    table = torch.tensor([[0, 1], [2, 99], [-1, 4]], dtype=torch.int32, device=DEV)

    def call(offsets, lens):
        kc = torch.zeros((nb, hkv, 16, d), dtype=torch.bfloat16, device=DEV)
        vc, qo = torch.zeros((nb, hkv, d, 16), dtype=torch.bfloat16, device=DEV), torch.zeros_like(q)
        lib.paged_qk_norm_rope_append(q, k, v, None, None, cs, torch.tensor(offsets, dtype=torch.int32, device=DEV), kc, vc,
                                      None, table, torch.tensor(lens, dtype=torch.int32, device=DEV), qo)
        return qo, kc.abs().sum(dim=(1, 3)).ne(0).cpu(), lib.read_device_status()

    qo, at, st = call([0, 2, 4, 6], [17, 17, 18])      # blocks 0, 1 / 2, 99 / 4
    assert st == lib.STATUS_BAD_BLOCK and at.nonzero().tolist() == [[0, 15], [1, 0], [2, 15], [4, 0], [4, 1]]
    assert (qo.abs().sum(dim=(1, 2)) > 0).all()
    qo, at, st = call([0, 2, 4, 6], [100, -5, 18])     # clamped to 32; to 0
    assert st == lib.STATUS_LEN_CLAMPED and at.nonzero().tolist() == [[1, 14], [1, 15], [4, 0], [4, 1]]
    qo, at, st = call([0, 4, 2, 6], [4, 4, 20])        # sequence 1 goes back
    assert st & lib.STATUS_BAD_OFFSETS
    assert not at[2].any()
    qo, at, st = call([1, 1, 1, 3], [9, 9, 18])        # rows of no sequence keep q_out's content
    assert st == 0 and at.nonzero().tolist() == [[4, 0], [4, 1]]
    assert (qo.abs().sum(dim=(1, 2)) > 0).tolist() == [False, True, True, False, False, False]
    call([0, 2, 4, 900], [17, 17, 18])
    call([-7, 2, 4, 6], [17, 17, 18])
    lib.read_device_status()


def test_graph_and_streams(lib):
    """Captured once on a side stream, replayed with lengths and tokens changed in place; every replay equals the eager call."""
    B, hq, hkv, d, width = 5, 8, 2, 128, 8
    table = torch.arange(B * width, dtype=torch.int32, device=DEV).view(B, width)
    kc, vc, _ = cache_of("bf16", B * width, hkv, d, 1)
    ga, gb = [kc.clone().to(DEV), vc.clone().to(DEV)], [kc.clone().to(DEV), vc.clone().to(DEV)]
    q, k, v = (rand((B, h, d), torch.bfloat16, h).to(DEV) for h in (hq, hkv, hkv))
    w = torch.ones(d, device=DEV)
    cs, lens = R.angles(width * 16, d).to(DEV), torch.full((B,), 3, dtype=torch.int32, device=DEV)
    qa, qb = torch.empty_like(q), torch.empty_like(q)
    s = torch.cuda.Stream(DEV)
    s.wait_stream(torch.cuda.current_stream())

    def call(c, o):
        lib.paged_qk_norm_rope_append(q, k, v, w, w, cs, None, *c, None, table, lens, o)

    with torch.cuda.stream(s):
        call([x.clone() for x in ga], qa)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call(ga, qa)
    for r in range(4):
        lens += 5
        q.normal_()
        k.normal_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        call(gb, qb)
        torch.cuda.synchronize()
        assert torch.equal(qa, qb) and torch.equal(ga[0], gb[0]) and torch.equal(ga[1], gb[1]), r


def test_cache_past_32_bits(lib):
    """Tiles at element offsets past 2^32 of a large cache."""
    hkv, d, nb = 8, 128, (1 << 32) // (8 * 16 * 128) + 40
    kc = torch.zeros((nb, hkv, 16, d), dtype=torch.bfloat16, device=DEV)
    vc = torch.zeros((nb, hkv, d, 16), dtype=torch.bfloat16, device=DEV)
    table = torch.tensor([[nb - 1, 3], [nb - 2, nb - 30]], dtype=torch.int32, device=DEV)
    q, k, v = (rand((4, h, d), torch.bfloat16, h).to(DEV) for h in (8, hkv, hkv))
    lib.paged_qk_norm_rope_append(q, k, v, None, None, R.angles(40, d).to(DEV), None, kc, vc, None, table,
                                  torch.tensor([17, 32], dtype=torch.int32, device=DEV), torch.empty_like(q),
                                  positions=torch.zeros(4, dtype=torch.int32, device=DEV))
    for row, (b, s) in enumerate(((nb - 1, 15), (3, 0), (nb - 30, 14), (nb - 30, 15))):
        assert torch.equal(kc[b, :, s], k[row]) and torch.equal(vc[b, :, :, s], v[row])
    assert int(kc.ne(0).any(dim=3).sum()) == 4 * hkv
