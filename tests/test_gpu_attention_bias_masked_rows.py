"""Attention with a bias by distance in rows that only keys behind a finite mask of -1e10 to -1e17 are left to: their products still tell them apart. Tolerances as in
test_gpu_attention_bias.py, whose terms they are; beyond them, for products near 832 and -896 before their scale of 1/8:
  a sum of up to 128 products below 1024 in fp32, one behind the other, is off by at most 128 x 2^-15 = 2^-8, after the scale by 2^-11, in a weight by as much of
  it, and so the sum of the weights: 2^-10; 2^-9 A is allowed, and 2^-9 of size for the gradients, for the table too
  a logarithm that far from 0 has the 24 bits of fp32 twice: 2^-22 of itself."""
import numpy as np
import pytest

from oracle import encoder as OE
from gpu_util import host, host_bf16
from test_gpu_attention_bias import U, Case, backward
from test_gpu_attention_bias_masks import sizes

pytestmark = pytest.mark.gpu

ROWS = [dict(B_=2, H=2, Hk=2, dh=64, Lq=70, Lk=150, lens=[150, 33]), dict(B_=1, H=2, Hk=1, dh=128, Lq=130, Lk=140, causal=True, first=[10]),
        dict(B_=1, H=2, Hk=2, dh=64, Lq=20, Lk=1100, first=[1000]), dict(B_=2, H=4, Hk=2, dh=128, Lq=2, Lk=1300, first=[1200, 3]), dict(B_=1, H=8, Hk=1, dh=64, Lq=1, Lk=90)]


def masked_row(shape, low, product):
    """Every bias is `low`, but for the nearest distances', which is as many steps of `low`'s last place further down as no product makes up for. The
    products are near `product`, before their scale."""
    c = Case(**shape, far=8, bucket=np.where(np.abs(np.arange(-8, 9)) < 3, 1, 0), buckets=2, scale=0.125)
    c.q[..., 0], c.k[..., 0] = 32.0, product / 32.0
    low = np.float32(low)
    c.table[0], c.table[1] = low, np.float32(low * 1.125)
    return c


@pytest.mark.parametrize("product", [832.0, -896.0])
@pytest.mark.parametrize("low", [-1e10, -1e15, -1e17])
@pytest.mark.parametrize("i", range(len(ROWS)))
def test_rows_with_masked_keys_alone(i, low, product):
    c = masked_row(ROWS[i], low, product)
    # the softmax does not see what all biases of a row have in common: without it 64 bits hold the products beside them
    plain = list(c.plain())
    base = c.table[0, 0].astype(np.float64)
    plain[3] = c.table.astype(np.float64) - base
    o, moved, p = OE.attention_bias(*plain)
    A = sizes(c, p)
    tol = U * A + U * np.abs(o) + 2.0 ** -9 * A
    for train in (False, True):
        O, lse, _, _ = c.forward(train)
        got = host_bf16(O)
        assert np.isfinite(got).all(), train
        off = np.abs(got - o)
        assert (off <= tol).all(), (train, float((off - tol).max()))
    want = base + moved
    assert (np.abs(host(lse).astype(np.float64) - want) <= 2.0 ** -22 * np.abs(want)).all()
    grads, _ = backward(c)
    want, size = OE.attention_bias_backward(*plain, c.do)
    for name, g, w, m in zip(("dq", "dk", "dv"), grads, want, size):
        t = (1.1 * U + 2.0 ** -9) * m + U * np.abs(w) + 1e-30
        off = np.abs(host_bf16(g) - w)
        assert (off <= t).all(), (name, float((off - t).max()))
    off = np.abs(host(grads[3]).astype(np.float64) - want[3])
    assert (off <= 2.0 ** -9 * size[3] + 1e-30).all(), float((off - 2.0 ** -9 * size[3]).max())
