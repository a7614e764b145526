"""Cache append of head norms with rotation (include/pda_ops.h) in the sizes that choose its kernels: on both sides of
the rows from which a wave takes many of them, on both sides of the rule that hands few tokens to a wave per token, without offsets
as with them; and that kernel's device checks."""

import numpy as np
import pytest
import torch

from tests import _ops_ref as R
from tests.test_rope_gpu import DEV, TYPES, check_append, lib, rand  # noqa: F401

pytestmark = pytest.mark.gpu

KINDS = [("f32", "f32"), ("bf16", "bf16"), ("fp8", "bf16"), ("bf16", "f32"), ("fp8", "f32"), ("f32", "bf16")]
AMP = [0.01, 0.5, 3.0, 40.0]  # sizes of tokens, so that fp8 scales rise in the middle of tiles


@pytest.mark.parametrize("T", [1985, 1986])  # 65,505 and 65,538 rows of queries
@pytest.mark.parametrize("d,rot,inter", [(64, 64, False), (128, 128, False), (128, 64, True)])
@pytest.mark.parametrize("kv,t", KINDS)
def test_many_rows_with_offsets(lib, kv, t, d, rot, inter, T):
    counts = [0, 1, 15, 16, 17, 333, 0, 64, 2, 700, 31, 48]
    counts.append(T - sum(counts))
    lens = [c + x for c, x in zip(counts, (5, 0, 3, 16, 31, 7, 0, 0, 62, 9, 33, 8, 1))]
    print(f"[append] {kv} {t} D={d} R={rot} T={T}", flush=True)
    check_append(lib, kv, t, lens, counts, 33, 3, d, rot, inter, True, T, amp=AMP)
    assert lib.read_device_status() == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv,t", KINDS)
def test_many_rows_without_offsets(lib, kv, t, d):
    """4 x 512 tokens that end anywhere in a block, one sequence of its new tokens alone."""
    check_append(lib, kv, t, [512, 519, 600, 801], [512] * 4, 33, 2, d, d, False, True, 3, even=True, amp=AMP)
    assert lib.read_device_status() == 0


@pytest.mark.parametrize("kv,t", [("f32", "f32"), ("bf16", "bf16"), ("fp8", "bf16")])
@pytest.mark.parametrize("n,B,hkv", [(3, 100, 5), (4, 32, 8), (4, 33, 8), (59, 5, 4), (8, 16, 8), (8, 17, 8), (2, 70, 16), (33, 31, 1),
                                     (32, 32, 1), (16, 65, 1)])
def test_tokens_of_every_sequence(lib, kv, t, n, B, hkv):
    """n new tokens each without offsets: up to 3, and up to 1,024 (token, KV head) pairs in all, go by tokens into a
    cache without scales, others by tiles."""
    rng = np.random.default_rng(n * B)
    for d, rot, inter in ((64, 32, True), (128, 128, False)):
        lens = n + rng.integers(0, 50, B)
        lens[:2] = n, n + 16 - n % 16  # from the first slot on; up to the end of a block
        check_append(lib, kv, t, lens, [n] * B, 6, hkv, d, rot, inter, True, n + B, even=True, amp=AMP)
        # more tokens than a sequence holds, an empty one; positions of their own
        lens[2:4] = n - 1, 0
        check_append(lib, kv, t, lens, [n] * B, 6, hkv, d, rot, inter, False, n + B + 1, even=True, positions=True)
    assert lib.read_device_status() == 0


@pytest.mark.parametrize("kv", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("n,hkv", [(1, 2), (2, 2), (3, 5), (4, 128), (7, 64), (40, 2)])
def test_device_checks_without_offsets(lib, kv, n, hkv):
    """Bad block ids, lengths outside the table and below the token count: what is outside is not written, the rest is,
    and the status says so."""
    B, d, width, nb = 3, 64, 4, 12
    dt = torch.float32 if kv == "f32" else torch.bfloat16
    q, k, v = (rand((B * n, h, d), dt, h + i).to(DEV) for i, h in enumerate((1, hkv, hkv)))
    table = torch.tensor([[0, 1, 8, 3], [2, 99, 7, -1], [-1, 4, nb, 5]], dtype=torch.int32)
    cs, zeros = R.angles(64, d).to(DEV), torch.zeros(B * n, dtype=torch.int32, device=DEV)
    for lens in ([17, 17, 18], [100, -5, 18], [64, 64, 64], [16, 33, 0], [n, n, max(n - 1, 0)], [2 ** 31 - 1, -2 ** 31, 1]):
        kc = torch.zeros((nb, hkv, 16, d), device=DEV).to(torch.uint8 if kv == "fp8" else dt)
        vc, qo = torch.zeros((nb, hkv, d, 16), device=DEV).to(kc.dtype), torch.zeros_like(q)
        sc = torch.zeros((2, nb, hkv), device=DEV) if kv == "fp8" else None
        lib.paged_qk_norm_rope_append(q, k, v, None, None, cs, None, kc, vc, sc, table.to(DEV),
                                      torch.tensor(lens, dtype=torch.int32, device=DEV), qo, positions=zeros)
        want, status = {}, 0
        for b, x in enumerate(lens):
            x, status = min(max(x, 0), 16 * width), status | (lib.STATUS_LEN_CLAMPED if not 0 <= x <= 16 * width else 0)
            for i in range(n):
                p = x - n + i
                if p < 0:
                    continue
                block = int(table[b, p // 16])
                if 0 <= block < nb:
                    want[block, p % 16] = b * n + i
                else:
                    status |= lib.STATUS_BAD_BLOCK
        assert lib.read_device_status() == status, lens
        assert torch.equal(qo, q)  # turned by angle 0
        at = kc.view(torch.uint8).view(nb, hkv, 16, -1).ne(0).any(dim=3).any(dim=1).cpu().nonzero().tolist()
        assert [tuple(x) for x in at] == sorted(want), lens
        if kv != "fp8":
            for (block, slot), row in want.items():
                assert torch.equal(kc[block, :, slot], k[row]) and torch.equal(vc[block, :, :, slot], v[row]), lens
        else:
            got = {(b, 0) for b, _ in want}
            assert {(int(b), 0) for b in sc.amax(dim=(0, 2)).nonzero()} == got


@pytest.mark.parametrize("kv", ["f32", "bf16"])
def test_cache_past_32_bits_by_tiles(lib, kv):
    """Tiles at element offsets past 2^32 of a large cache, with offsets."""
    hkv, d, nb = 8, 128, (1 << 32) // (8 * 16 * 128) + 40
    kc, vc = (torch.zeros(s, dtype=TYPES[kv], device=DEV) for s in ((nb, hkv, 16, d), (nb, hkv, d, 16)))
    table = torch.tensor([[nb - 1, 3], [nb - 2, nb - 30]], dtype=torch.int32, device=DEV)
    q, k, v = (rand((5, h, d), TYPES[kv], h + i).to(DEV) for i, h in enumerate((8, hkv, hkv)))
    lib.paged_qk_norm_rope_append(q, k, v, None, None, R.angles(40, d).to(DEV), torch.tensor([0, 2, 5], dtype=torch.int32, device=DEV),
                                  kc, vc, None, table, torch.tensor([17, 18], dtype=torch.int32, device=DEV), torch.empty_like(q),
                                  positions=torch.zeros(5, dtype=torch.int32, device=DEV))
    for row, (b, s) in enumerate(((nb - 1, 15), (3, 0), (nb - 2, 15), (nb - 30, 0), (nb - 30, 1))):
        assert torch.equal(kc[b, :, s], k[row]) and torch.equal(vc[b, :, :, s], v[row])
    assert int(kc.ne(0).any(dim=3).sum()) == 5 * hkv
