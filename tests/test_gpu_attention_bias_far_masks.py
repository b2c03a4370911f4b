"""Attention with a bias by distance where keys behind a far finite mask come first and those that count have logits far below 0: the masked ones weigh nothing.
Tolerances as in test_gpu_attention_bias_masks.py."""
import numpy as np
import pytest

from test_gpu_attention_bias_masks import LOWEST, check, masked

pytestmark = pytest.mark.gpu

# few queries over more keys than the waves of a workgroup take at once, and many queries; the keys that count come last
LONG = [dict(B_=1, H=2, Hk=2, dh=64, Lq=1, Lk=1024, first=[1018]), dict(B_=2, H=4, Hk=1, dh=128, Lq=3, Lk=1500, first=[1490, 700]),
        dict(B_=1, H=1, Hk=1, dh=64, Lq=16, Lk=5000, first=[4970]), dict(B_=1, H=2, Hk=2, dh=64, Lq=40, Lk=1024, first=[980])]


@pytest.mark.parametrize("level", [-150.0, -300.0])
@pytest.mark.parametrize("low", [-1e10, LOWEST])
@pytest.mark.parametrize("i", range(len(LONG)))
def test_low_logits_behind_masked_keys(i, low, level):
    """Masked keys, far more of them than of the others, come first and weigh nothing."""
    c = masked(LONG[i], low, 5)
    c.table[:-1] += np.float32(level)
    check(c)
