"""The training forward with results of another type than its inputs (include/pda_ops.h: out_dtype), in rows of few and
of many, in strided results."""

import pytest
import torch

from tests import _ops_ref as R
from tests.test_rope_gpu import DEV, TYPES, dev, lib, rand, weights  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,o", [("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("d,rot,inter", [(64, 32, False), (128, 128, False), (128, 64, True)])
@pytest.mark.parametrize("T,hq,hkv", [(1, 3, 1), (70, 28, 4), (2100, 31, 3)])
def test_results_of_another_type(lib, t, o, d, rot, inter, T, hq, hkv):
    dt, ot = TYPES[t], TYPES[o]
    q, k = rand((T, hq, d), dt, 1), rand((T, hkv, d), dt, 2, 3.0)
    table, pos = R.angles(100, rot), torch.arange(T, dtype=torch.int32) % 100
    for norm in (True, False):
        wq, wk = weights(d, torch.float32, norm)
        out = torch.full((T, hq + hkv + 1, d), 7.0, dtype=ot, device=DEV)
        lib.qk_norm_rope(*[dev(x) for x in (q, k, wq, wk, table, pos)], out[:, :hq], out[:, hq:hq + hkv], interleaved=inter)
        for x, w, y, name in ((q, wq, out[:, :hq], "q"), (k, wk, out[:, hq:hq + hkv], "k")):
            want, bound = R.norm_turn(x, w, table, pos, 1e-6, inter)
            R.assert_within(y, want, bound, ot, f"{name} norm={norm}")
        assert (out[:, hq + hkv:] == 7.0).all()
    assert lib.read_device_status() == 0
