"""Policy loss with gradients on both sides of the size from which they are stored past the caches (10 MiB), of rows in
registers and in parts, the gradient in rows of its own alignment and with padding."""

import pytest
import torch

from tests.test_policy_gpu import check_policy, lib, TYPES  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,T,V", [
    ("bf16", 1310, 4001), ("bf16", 1311, 4001), ("bf16", 349, 15_000), ("bf16", 350, 15_000), ("bf16", 165, 31_700), ("bf16", 166, 31_700),
    ("f32", 655, 4001), ("f32", 656, 4001), ("f32", 320, 8191), ("f32", 321, 8191),
    ("bf16", 104, 50_001), ("bf16", 105, 50_001), ("f32", 52, 50_001), ("f32", 53, 50_001)])
def test_both_sides_of_the_size(lib, t, T, V):
    check_policy(lib, TYPES[t], T, V, 3, 1.0, True, 0.0, 0.1, 0.01, 1.0, 0.02, 1.0, V + T)
