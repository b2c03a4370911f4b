"""Attention with a bias by distance with infinities and NaN in keys and values: in those that count they come through as the definition has them,
and in places that a query does not see they change nothing. Where results are finite, the tolerances of test_gpu_attention_bias.py, whose terms they are."""
import numpy as np
import pytest
import torch

from oracle import encoder as OE
from gpu_util import host, host_bf16
from test_gpu_attention_bias import Case, U, _bits
from test_gpu_attention_bias_masks import sizes

pytestmark = pytest.mark.gpu

# the few queries' kernel, the tiled one, in one piece and in slices of the keys, both widths of heads
WHOLE = [dict(B_=2, H=2, Hk=1, dh=64, Lq=3, Lk=200, lens=[130, 3]), dict(B_=2, H=2, Hk=2, dh=128, Lq=1, Lk=1500, lens=[1473, 1]),
         dict(B_=2, H=2, Hk=2, dh=64, Lq=100, Lk=200, lens=[130, 3]), dict(B_=1, H=2, Hk=2, dh=128, Lq=40, Lk=1500, lens=[1473])]


def check_row_by_row(c, got, o, A):
    """Finite places within their tolerance, infinities and NaN at the same places."""
    finite = np.isfinite(o)
    assert np.array_equal(np.isnan(got), np.isnan(o)) and np.array_equal(got[np.isinf(o)], o[np.isinf(o)])
    tol = U * A + U * np.abs(o) + 2.0 ** -10 * A
    with np.errstate(invalid="ignore"):
        off = np.abs(got - o)
    assert (off <= tol)[finite].all(), float((off - tol)[finite].max())


@pytest.mark.parametrize("train", [False, True])
@pytest.mark.parametrize("i", range(len(WHOLE)))
def test_last_key(i, train):
    """An infinity in the last key's values is one in its column of the result, and nowhere else."""
    c = Case(**WHOLE[i])
    for b, n in enumerate(c.lens):
        c.v[b, n - 1, :, 5], c.v[b, n - 1, :, 40] = np.inf, -np.inf
    O, lse, _, _ = c.forward(train)
    plain = c.plain()
    with np.errstate(invalid="ignore"):
        o, want, p = OE.attention_bias(*plain)
        A = sizes(c, p)
    assert np.isinf(o[..., 5]).all() and np.isinf(o[..., 40]).all() and np.isfinite(np.delete(o, [5, 40], 3)).all()
    check_row_by_row(c, host_bf16(O), o, A)
    if train:
        assert (np.abs(host(lse) - want) <= 2.0 ** -16 * (1 + np.abs(want))).all()


CAUSAL = [dict(B_=1, H=2, Hk=1, dh=64, Lq=8, Lk=300, first=[250]), dict(B_=1, H=2, Hk=2, dh=128, Lq=5, Lk=1500, first=[1495]),
          dict(B_=1, H=2, Hk=2, dh=64, Lq=200, Lk=200), dict(B_=1, H=2, Hk=2, dh=128, Lq=40, Lk=1500, first=[1450]), dict(B_=1, H=3, Hk=3, dh=64, Lq=16, Lk=40, first=[-6])]


def seen_rows(c, j):
    """Rows of queries that see key j."""
    return np.arange(c.Lq) + (c.first[0] if c.first else 0) >= j


def by_definition(c):
    """Rows one by one over the keys that they see, and their A."""
    o, A, lse = np.zeros(c.q.shape), np.zeros(c.q.shape), np.full((c.B, c.H, c.Lq), -np.inf)
    for i in range(c.Lq):
        n = max(0, min(c.Lk, (c.first[0] if c.first else 0) + i + 1))
        if n == 0:
            continue
        with np.errstate(invalid="ignore"):
            r, l, p = OE.attention_bias(c.q[:, i:i + 1], c.k[:, :n], c.v[:, :n], c.table, c.bucket, [n], [(c.first[0] if c.first else 0) + i], True, c.scale)
        o[:, i:i + 1], lse[:, :, i:i + 1] = r, l
        for h in range(c.H):
            A[0, i, h] = p[0, h, 0] @ np.abs(c.v[0, :n, h // (c.H // c.Hk)])
    return o, A, lse


@pytest.mark.parametrize("train", [False, True])
@pytest.mark.parametrize("where", ["value inf", "value nan", "key nan", "key inf"])
@pytest.mark.parametrize("i", range(len(CAUSAL)))
def test_keys_ahead(i, where, train):
    """Causal: a key and value with an infinity or NaN reach the rows from their own on and no row ahead of it."""
    c = Case(**CAUSAL[i], causal=True)
    of, what = where.split()
    j = (c.first[0] if c.first else 0) + c.Lq - max(2, c.Lq // 2)
    t = c.v if of == "value" else c.k
    t[0, j, :, 7] = np.inf if what == "inf" else np.nan
    O, lse, _, _ = c.forward(train)
    o, A, want = by_definition(c)
    got, rows = host_bf16(O), seen_rows(c, j)
    assert rows.any() and not rows.all()
    check_row_by_row(c, got[:, ~rows], o[:, ~rows], A[:, ~rows])
    assert np.isfinite(got[:, ~rows]).all()
    if of == "value":
        with np.errstate(invalid="ignore"):
            check_row_by_row(c, got[:, rows], o[:, rows], A[:, rows])
    elif what == "nan":
        assert np.isnan(got[:, rows]).all()
    if train:
        some = np.isfinite(want) & ~rows
        assert (np.abs(host(lse).astype(np.float64)[some] - want[some]) <= 2.0 ** -16 * (1 + np.abs(want[some]))).all()


def with_room(c):
    """A cache with room behind, and the first key that no query sees."""
    c.k, c.v = (np.concatenate((t, np.ones((1, 70) + t.shape[2:], np.float32)), 1) for t in (c.k, c.v))
    c.Lk += 70
    return (c.first[0] if c.first else 0) + c.Lq


def spoil(c, last):
    c.k[0, last:last + 20], c.k[0, last + 20:], c.v[0, last:last + 10], c.v[0, last + 10:] = np.nan, np.inf, -np.inf, np.nan


@pytest.mark.parametrize("train", [False, True])
@pytest.mark.parametrize("layout", ["apart", "packed"])
@pytest.mark.parametrize("i", range(len(CAUSAL)))
def test_keys_that_no_query_sees(i, layout, train):
    """Causal, over a cache with room that no length cuts off: what stands behind the last query's own key changes no bit of the results."""
    c = Case(**CAUSAL[i], causal=True, layout=layout)
    last = with_room(c)
    want = c.forward(train)[0].clone()
    spoil(c, last)
    assert torch.equal(_bits(c.forward(train)[0].contiguous()), _bits(want.contiguous()))


@pytest.mark.parametrize("Lq", [4, 40])
def test_rows_that_see_no_key(Lq):
    """Queries ahead of the first key are rows of zeros, whatever the keys hold."""
    c = Case(1, 2, 2, 64, Lq, 90, first=[-Lq + 1], causal=True)
    c.k[0, 0], c.v[0, 0] = np.nan, np.inf
    O, lse, rest, _ = c.forward()
    assert not host_bf16(O)[0, :-1].any() and not rest.view(torch.int16)[0, :-1].any() and np.isneginf(host(lse)[0, :, :-1]).all()
    assert not host_bf16(c.forward(False)[0])[0, :-1].any() and np.isnan(host_bf16(O)[0, -1]).all()
