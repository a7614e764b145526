"""Cache append with offsets that go back or leave [0, T]: the status says so, and whatever is written belongs to a
sequence whose own offsets are in order (other tokens of such sequences may be left out)."""

import numpy as np
import pytest
import torch

from tests import _ops_ref as R
from tests.test_rope_gpu import DEV, lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu


def offsets_of(seed):
    if seed == 0:
        return [-7, 2, 4, 6], 6
    if seed == 1:
        return [0, 900, 4, 6], 6
    if seed == 2:
        return [0, 2, 4, 900], 6
    if seed == 3:
        return [0, 5, 2, 6], 6  # two sequences claim the same rows
    if seed == 4:
        return [2 ** 31 - 1, -2 ** 31, 0, 6], 6
    rng = np.random.default_rng(seed)
    B = int(rng.integers(1, 200))
    off = np.concatenate([[0], rng.choice([0, 1, 2, 17, 40], B)]).cumsum()
    T = int(off[-1]) + 1
    for i in rng.choice(B + 1, min(B + 1, 3), replace=False):
        off[i] = rng.choice([-5, -2 ** 31, T + 1, 2 ** 31 - 1, 0, int(off[0]), T])
    return off.tolist(), T


@pytest.mark.parametrize("seed", range(15))
def test_offsets_out_of_order(lib, seed):
    off, T = offsets_of(seed)
    B, hq, hkv, d, width = len(off) - 1, 2, 2, 64, 8
    print(f"[offsets] seed {seed}: {B} sequences, {T} rows", flush=True)
    good = [0 <= a <= b <= T for a, b in zip(off, off[1:])]
    rng = np.random.default_rng(seed + 100)
    lens = rng.integers(0, 16 * width + 1, B)
    table = rng.permutation(B * width).reshape(B, width)
    q, k, v = (rand((T, h, d), torch.bfloat16, h + i).to(DEV) for i, h in enumerate((hq, hkv, hkv)))
    kc, vc = (torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in ((B * width, hkv, 16, d), (B * width, hkv, d, 16)))
    qo = torch.zeros_like(q)
    as_int = lambda x: torch.from_numpy(np.asarray(x).astype(np.int32)).to(DEV)  # noqa: E731
    lib.paged_qk_norm_rope_append(q, k, v, None, None, R.angles(16 * width, d).to(DEV), as_int(off), kc, vc, None, as_int(table),
                                  as_int(lens), qo, positions=torch.zeros(T, dtype=torch.int32, device=DEV))
    assert lib.read_device_status() == (0 if all(good) else lib.STATUS_BAD_OFFSETS)
    owner = {}  # slot -> the row that may be there
    rows = np.zeros(T, bool)
    for b in range(B):
        if good[b]:
            rows[off[b]:off[b + 1]] = True
            for i in range(off[b], off[b + 1]):
                p = int(lens[b]) - (off[b + 1] - i)
                if p >= 0:
                    owner[int(table[b, p // 16]), p % 16] = i
    for t in range(T):
        assert torch.equal(qo[t], q[t]) or not qo[t].any()
        assert rows[t] or not qo[t].any()
    hk, hv, ck, cv = kc.cpu(), vc.cpu().transpose(2, 3), k.cpu(), v.cpu()
    for block, slot in (hk.ne(0).any(dim=3).any(dim=1) | hv.ne(0).any(dim=3).any(dim=1)).nonzero().tolist():
        i = owner[block, slot]
        for got, want in ((hk, ck), (hv, cv)):
            assert torch.equal(got[block, :, slot], want[i]) or not got[block, :, slot].any()
    if all(good):
        assert len(owner) == int(hk.ne(0).any(dim=3).any(dim=1).sum())
