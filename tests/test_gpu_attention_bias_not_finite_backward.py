"""Gradients of attention with a bias by distance where keys and values hold infinities and NaN in places that a query does not see, or that no query sees,
and where the gradient that comes in does. Where gradients are finite, the tolerances of test_gpu_attention_bias.py."""
import numpy as np
import pytest
import torch

from oracle import encoder as OE
from gpu_util import host, host_bf16
from test_gpu_attention_bias import Case, U, _bits, backward
from test_gpu_attention_bias_not_finite import CAUSAL, seen_rows, spoil, with_room

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["apart", "packed"])
@pytest.mark.parametrize("i", range(len(CAUSAL)))
def test_keys_that_no_query_sees(i, layout):
    """Causal, over a cache with room that no length cuts off: what stands behind the last query's own key changes no bit of the gradients, whose rows there
    are zeros."""
    c = Case(**CAUSAL[i], causal=True, layout=layout)
    last = with_room(c)
    want, _ = backward(c)
    spoil(c, last)
    got, _ = backward(c)
    for a, b in zip(got, want):
        assert torch.equal(_bits(a.contiguous()), _bits(b.contiguous())) and np.isfinite(host(a.float())).all()
    assert not host_bf16(got[1])[0, last:].any() and not host_bf16(got[2])[0, last:].any()


@pytest.mark.parametrize("of", ["key", "value"])
@pytest.mark.parametrize("i", range(len(CAUSAL)))
def test_gradients_of_queries_behind_which_a_key_is_not_finite(i, of):
    """Causal: the gradients of queries that do not see the key are what they are without it."""
    c = Case(**CAUSAL[i], causal=True)
    j = (c.first[0] if c.first else 0) + c.Lq - max(2, c.Lq // 2)
    rows = seen_rows(c, j)
    c.do[:, rows] = 0.0
    want, size = OE.attention_bias_backward(*c.plain(), c.do)
    (c.k if of == "key" else c.v)[0, j, :, 9] = np.nan
    got = host_bf16(backward(c)[0][0])
    tol = 1.1 * U * size[0] + U * np.abs(want[0]) + 1e-30
    assert (np.abs(got - want[0]) <= tol)[:, ~rows].all()


def test_gradients_behind_the_last_key():
    """An infinity in a gradient that comes in leaves the rows of keys behind a sequence's length zeros."""
    c = Case(2, 2, 1, 64, 70, 150, lens=[100, 9])
    c.do[0, 3, 0, 5], c.do[1, 60, 1, 7] = np.inf, np.nan
    (_, dK, dV, _), _ = backward(c)
    for b, n in enumerate(c.lens):
        assert not host_bf16(dK)[b, n:].any() and not host_bf16(dV)[b, n:].any()
    assert not np.isfinite(host_bf16(dV)[0, :100]).all()


@pytest.mark.parametrize("dh", [64, 128])
def test_gradients_of_keys_that_no_query_sees(dh):
    """The same, causal: of keys behind the last query's own."""
    c = Case(1, 2, 2, dh, 70, 150, first=[20], causal=True)
    c.do[0, 3, 0, 5], c.do[0, 60, 1, 7] = np.inf, np.nan
    (_, dK, dV, _), _ = backward(c)
    assert not host_bf16(dK)[0, 90:].any() and not host_bf16(dV)[0, 90:].any()
