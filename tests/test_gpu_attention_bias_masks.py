"""Attention with a bias by distance where finite biases mask: values from -1e4 to the lowest of the type in front of keys that count, rows that such a
bias leaves nothing else to, and rows whose logits are all large. Tolerances as in test_gpu_attention_bias.py, whose terms they are; beyond them:
  a logit of size x is rounded to 24 bits in the sum with its bias: for |x| <= 2^12 by 2^-12 in powers of two, twice with its reference, ln 2 of that in
  its weight, and once more for the sum: 2^-10 A, which the allowance of 2^-10 A there has room for (2^-15 A of it are used there);
  gradients: 2^-10 of size instead of 2^-14, and so for the table."""
import numpy as np
import pytest

from oracle import encoder as OE
from paper_2604_04451_amd import binding as B
from gpu_util import host, host_bf16
from test_gpu_attention_bias import U, Case, backward

pytestmark = pytest.mark.gpu

LOWEST = float(np.finfo(np.float32).min)
SHAPES = [
    dict(B_=1, H=2, Hk=2, dh=64, Lq=130, Lk=130), dict(B_=2, H=8, Hk=8, dh=64, Lq=300, Lk=300, lens=[300, 140]), dict(B_=1, H=2, Hk=1, dh=128, Lq=200, Lk=260, causal=True, first=[60]),
    dict(B_=1, H=2, Hk=2, dh=64, Lq=20, Lk=1500, first=[1400]), dict(B_=2, H=4, Hk=2, dh=128, Lq=1, Lk=1300, first=[1200, 3]), dict(B_=1, H=4, Hk=1, dh=64, Lq=3, Lk=5000, first=[4300]),
]


def masked(shape, low, keep, far=8):
    """Keys further than `keep` to either side get the bias `low`; the others that of their distance."""
    bucket = np.full(2 * far + 1, 2 * far + 1, np.int32)
    bucket[far - keep:far + keep + 1] = np.arange(far - keep, far + keep + 1)
    c = Case(**shape, far=far, bucket=bucket, buckets=2 * far + 2, scale=None)
    c.table[-1] = low
    return c


def sizes(c, p):
    n = c.lens if c.lens is not None else [c.Lk] * c.B
    A = np.zeros(c.q.shape)
    for b in range(c.B):
        for h in range(c.H):
            A[b, :, h] = p[b, h] @ np.where((np.arange(c.Lk) < n[b])[:, None], np.abs(c.v[b, :, h // (c.H // c.Hk)]), 0.0)
    return A


def check(c):
    o, want_lse, p = OE.attention_bias(*c.plain())
    tol = U * sizes(c, p) + U * np.abs(o) + 2.0 ** -10 * sizes(c, p)
    for train in (False, True):
        O, lse, _, _ = c.forward(train)
        off = np.abs(host_bf16(O) - o)
        assert (off <= tol).all(), (train, float((off - tol).max()))
    got = host(lse).astype(np.float64)
    few = np.abs(want_lse) < 2.0 ** 12
    assert (np.abs(got - want_lse)[few] <= 2.0 ** -16 * (1 + np.abs(want_lse[few]))).all()
    grads, _ = backward(c)
    want, size = OE.attention_bias_backward(*c.plain(), c.do)
    for name, g, w, m in zip(("dq", "dk", "dv"), grads, want, size):
        t = (1.1 * U + 2.0 ** -10) * m + U * np.abs(w) + 1e-30
        off = np.abs(host_bf16(g) - w)
        assert (off <= t).all(), (name, float((off - t).max()))
    off = np.abs(host(grads[3]).astype(np.float64) - want[3])
    assert (off <= 2.0 ** -10 * size[3] + 1e-30).all(), float((off - 2.0 ** -10 * size[3]).max())


@pytest.mark.parametrize("low", [-1e4, -1e6, -1e9, LOWEST])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_masked_keys_in_front_of_others(i, low):
    """Many keys behind a finite mask, then the 11 that count."""
    check(masked(SHAPES[i], low, 5))


@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_rows_with_nothing_but_the_lowest_value(i):
    """Whole rows are masked by the lowest value, which leaves all their keys the same weight; half of the others see only some keys so."""
    c = masked(SHAPES[i], LOWEST, 0)
    c.table[:] = LOWEST
    c.table[c.bucket[8], 0] = 0.25  # the first head has its own position
    check(c)


@pytest.mark.parametrize("level", [-2800.0, 400.0, 2800.0])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_large_logits(i, level):
    c = Case(**SHAPES[i])
    c.table += np.float32(level)
    check(c)


def test_highest_value():
    """Keys with the highest value of the type are all that counts in their rows."""
    for i in (0, 3, 4):
        c = masked(SHAPES[i], 0.0, 5)
        c.table[c.bucket[8 - 5:8 + 2]] = -LOWEST
        check(c)


@pytest.mark.parametrize("far", [0, 1])
def test_few_distances(far):
    c = Case(B_=2, H=2, Hk=1, dh=64, Lq=150, Lk=170, lens=[170, 80], far=far, bucket=np.arange(2 * far + 1), buckets=2 * far + 1)
    check(c)
