"""How much one call of include/pda_ops.h takes, as its header says, and what the refusal names (no GPU needed: a NULL
pointer ends the calls that are within the limits)."""

import pytest

from paper_2605_20863_amd import _lib as L
from tests import test_ops_abi as A


def error(rc):
    assert rc == L.EINVAL
    return L.last_error()


@pytest.mark.parametrize("hq,hkv,d,per", [(8, 2, 128, 4), (64, 8, 128, 20), (4, 4, 64, 3)])
def test_tokens(hq, hkv, d, per):
    def call(T, fn, **more):
        pr = A.rope(num_tokens=T, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, rotary_dim=d)
        return error(fn(pr, **{**dict(q=None), **more}))

    def append(pr, **kw):
        return A.append(pr, A.cache(num_seqs=1, max_blocks_per_seq=1 << 20, num_blocks=1 << 20), **kw)

    most = (1 << 25) // per
    assert call(most, append) == "q is NULL"
    assert "num_tokens" in call(most + 1, append)
    for fn in (A.forward, A.backward):
        assert call(2 * most, fn) == "q is NULL"
        assert "num_tokens" in call((1 << 26) // per + 1, fn)


def test_tiles():
    def call(B, T, **kw):
        return error(A.append(A.rope(num_tokens=T), A.cache(num_seqs=B), q=None, **kw))

    most = (1 << 25) // 4 // 2  # 2 tiles a sequence, of 2 KV heads
    assert call(most, 0 + 15) == "q is NULL"
    assert "cache tiles" in call(most + 1, 15)
    n = (1 << 25) // 4  # one token each: one tile
    assert "num_tokens" in call(n + 1, n + 1, off=None)
    assert call(n, n, off=None) == "q is NULL"


def test_rows():
    assert "num_tokens" in error(A.logprobs(A.logits(num_tokens=(1 << 22) + 1)))
    assert "num_tokens" in error(A.policy(A.logits(num_tokens=(1 << 20) + 1), A.options()))
