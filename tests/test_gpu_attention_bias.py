"""Attention with a bias by distance on the GPU through the C ABI, against plain fp64 forms. Tolerances, u = 2^-8 (half a step of bf16):
  weights are rounded to bf16 behind the matrix pipe's sums and the result once more: u A + u |O|, A the attention with |V| for V;
  a logit of up to 32 (in powers of two) from at most 128 products, its bias and the reference is off by at most 2^-16, of which the
  sum of the weights has as much: 2^-15 A together, 2^-10 A taken; lse: 2^-16 (1 + |lse|) for logits of that size
  with `rest` the result is not rounded
  gradients (delta is off by u |do| A in dq, where it comes from o, and by 2^-14 of its terms elsewhere): a weight is off by 2^-15 of itself, the gradient of a logit, ds = p (dp - delta), by 2^-14 of size = p (|do| |v| + |do o|) and is
  rounded to bf16 for the products: u |ds| + u 2^-6 size, whose sums against |k| and |q| the oracle returns (mq, mk), with those of p |do|
  (mv) and of size (mt): u of the first three, one more u of the result, 1.1 for sums in fp32; 2^-14 mt for the table, whose terms are
  not rounded to bf16."""
import numpy as np
import pytest
import torch

from oracle import encoder as OE
import paper_2604_04451_amd as P
from paper_2604_04451_amd import binding as B
from gpu_util import DEV, dev_bf16, dev_f32, host_bf16, host
import synth

pytestmark = pytest.mark.gpu

U = 2.0 ** -8
BF = torch.bfloat16


def _bf(a):
    return synth.round_bf16(np.ascontiguousarray(a, dtype=np.float32))


def _i32(a):
    return None if a is None else torch.tensor(list(a), dtype=torch.int32, device=DEV)


def _bits(t):
    return t.view(torch.int16 if t.dtype == BF else torch.int32)


class Case:
    def __init__(self, B_, H, Hk, dh, Lq, Lk, lens=None, first=None, causal=False, scale=None, buckets=32, far=128, both=True, seed=0, layout="apart",
                 bucket=None):
        rng = np.random.default_rng(seed + B_ * 1000 + H * 100 + dh + Lq * 7 + Lk)
        self.B, self.H, self.Hk, self.dh, self.Lq, self.Lk = B_, H, Hk, dh, Lq, Lk
        self.scale = dh ** -0.5 if scale is None else scale
        std = (2.0 / (self.scale * dh ** 0.5)) ** 0.5
        self.q, self.k, self.v = (_bf(rng.standard_normal(s) * std) for s in ((B_, Lq, H, dh), (B_, Lk, Hk, dh), (B_, Lk, Hk, dh)))
        self.do = _bf(rng.standard_normal((B_, Lq, H, dh)))
        self.table = rng.standard_normal((buckets, H)).astype(np.float32)
        self.bucket = OE.bias_buckets(buckets, far, both) if bucket is None else np.asarray(bucket, np.int32)
        self.lens, self.first, self.causal, self.layout = lens, first, causal, layout

    def plain(self):
        return (self.q, self.k, self.v, self.table, self.bucket, self.lens if self.lens is not None else [self.Lk] * self.B,
                self.first if self.first is not None else [0] * self.B, self.causal, self.scale)

    def place(self, a, fill=3.0):
        """A device tensor of a's shape: rows with room beside and behind ("apart"), or one behind the other."""
        n, L, heads, dh = a.shape
        if self.layout == "apart":
            room = torch.full((n, L + 3, heads * dh + 64), fill, dtype=BF, device=DEV)
            t = room[:, :L, 8:8 + heads * dh].view(n, L, heads, dh)
            t.copy_(dev_bf16(a))
            return t, room
        t = dev_bf16(a)
        return t, t

    def how(self):
        return dict(lens=_i32(self.lens), first=_i32(self.first), causal=self.causal, scale=self.scale)

    def forward(self, train=True):
        (Q, _), (K, _), (V, _), (O, room) = (self.place(t) for t in (self.q, self.k, self.v, np.full(self.q.shape, 5.0)))
        lse = torch.full((self.B, self.H, self.Lq), 9.0, device=DEV) if train else None
        rest = self.place(np.full(self.q.shape, 5.0))[0] if train else None
        self.dev = (Q, K, V, O, dev_f32(self.table), _i32(self.bucket))
        B.chorus_attention_bias(*self.dev, lse=lse, rest=rest, **self.how())
        return O, lse, rest, room


def check_forward(c, train=True):
    O, lse, rest, room = c.forward(train)
    o, want_lse, p = OE.attention_bias(*c.plain())
    _, Hk, group = c.k, c.Hk, c.H // c.Hk
    n = c.lens if c.lens is not None else [c.Lk] * c.B
    A = np.zeros(o.shape)
    for b in range(c.B):
        for h in range(c.H):
            A[b, :, h] = p[b, h] @ np.where((np.arange(c.Lk) < n[b])[:, None], np.abs(c.v[b, :, h // group]), 0.0)
    tol = U * A + U * np.abs(o) + 2.0 ** -10 * A
    got = host_bf16(O)
    assert (np.abs(got - o) <= tol).all(), float((np.abs(got - o) - tol).max())
    if c.layout == "apart":
        assert (room[:, c.Lq:] == 3).all() and (room[:, :, :8] == 3).all() and (room[:, :, 8 + c.H * c.dh:] == 3).all()
    if train:
        got = host(lse).astype(np.float64)
        some = np.isfinite(want_lse)
        assert np.array_equal(np.isneginf(got), ~some)
        assert (np.abs(got[some] - want_lse[some]) <= 2.0 ** -16 * (1 + np.abs(want_lse[some]))).all()
        bits = (O.contiguous().view(torch.int16).int() << 16) + rest.contiguous().view(torch.int16).int()  # both halves of the fp32 result
        assert (np.abs(host(bits.view(torch.float32)).astype(np.float64) - o) <= U * A + 2.0 ** -10 * A).all()
        assert torch.equal(bits.view(torch.float32).to(BF), O.contiguous())
    return c


FORWARD = [
    dict(B_=1, H=1, Hk=1, dh=64, Lq=1, Lk=1), dict(B_=1, H=2, Hk=2, dh=128, Lq=2, Lk=1), dict(B_=2, H=2, Hk=1, dh=64, Lq=5, Lk=63),
    dict(B_=1, H=2, Hk=2, dh=128, Lq=127, Lk=129), dict(B_=2, H=4, Hk=2, dh=64, Lq=130, Lk=130, lens=[130, 65]),
    dict(B_=3, H=2, Hk=2, dh=64, Lq=77, Lk=200, lens=[0, 1, 200], scale=1.0), dict(B_=1, H=2, Hk=2, dh=64, Lq=700, Lk=700),
    dict(B_=1, H=1, Hk=1, dh=128, Lq=513, Lk=513, causal=True, both=False), dict(B_=2, H=2, Hk=2, dh=64, Lq=40, Lk=300, causal=True, lens=[300, 17], first=[260, -23]),
    dict(B_=4, H=2, Hk=2, dh=64, Lq=1, Lk=1000, causal=True, lens=[1000, 999, 64, 0], first=[999, 998, 63, -1], both=False),
    dict(B_=1, H=3, Hk=3, dh=128, Lq=16, Lk=2100), dict(B_=2, H=2, Hk=2, dh=128, Lq=17, Lk=1500, lens=[1500, 300], first=[700, 100]),
    dict(B_=1, H=2, Hk=2, dh=64, Lq=260, Lk=1300, first=[520], far=512, buckets=64), dict(B_=1, H=2, Hk=2, dh=64, Lq=90, Lk=90, far=3, buckets=4),
    dict(B_=1, H=1, Hk=1, dh=64, Lq=300, Lk=1200, first=[-2000000000]), dict(B_=1, H=1, Hk=1, dh=64, Lq=300, Lk=1200, first=[2000000000], far=512),
    dict(B_=2, H=12, Hk=2, dh=128, Lq=3, Lk=2500, lens=[2500, 1100], first=[2497, 1090], causal=True, both=False), dict(B_=1, H=40, Hk=1, dh=128, Lq=1, Lk=300, far=512),
    dict(B_=1, H=5, Hk=1, dh=64, Lq=7, Lk=4100, scale=1.0, first=[-3], far=512, buckets=64), dict(B_=5, H=64, Hk=64, dh=64, Lq=1, Lk=130, lens=[130, 0, 64, 65, 1]),
    dict(B_=3, H=8, Hk=8, dh=64, Lq=200, Lk=200, lens=[200, 77, 0]), dict(B_=1, H=16, Hk=8, dh=128, Lq=140, Lk=1500, first=[900]),
    dict(B_=2, H=16, Hk=16, dh=64, Lq=30, Lk=700, lens=[700, 65], causal=True, first=[670, 35]),
    dict(B_=2, H=8, Hk=2, dh=64, Lq=1, Lk=777, lens=[777, 401], first=[776, 400], causal=True),
]


@pytest.mark.parametrize("layout", ["apart", "packed"])
@pytest.mark.parametrize("i", range(len(FORWARD)))
def test_forward(i, layout):
    check_forward(Case(**FORWARD[i], layout=layout), train=layout == "apart" or i % 2 == 0)


def test_rows_without_a_finite_logit():
    """Biases of -inf, the lowest value of the type and far beyond the exponential's range: rows of zeros, rows of one key, no NaN."""
    bucket = np.zeros(2 * 4 + 1, np.int32)
    bucket[4] = 1      # the key at the query's own position
    bucket[5:] = 2     # keys ahead
    for low, behind in ((-np.inf, -np.inf), (np.finfo(np.float32).min, -np.inf), (-np.inf, 0.5)):
        c = Case(1, 2, 2, 64, 100, 100, far=4, bucket=bucket, buckets=3)
        c.table[:] = np.array([behind, low, -np.inf])[:, None]
        with np.errstate(invalid="ignore"):
            O, lse, rest, _ = c.forward()
            o, want, _ = OE.attention_bias(*c.plain())
        got = host_bf16(O)
        assert np.isfinite(got).all()
        if low == -np.inf and behind == -np.inf:
            assert not got.any() and np.isneginf(host(lse)).all()
        else:
            worst = float(np.abs(got - o).max())
            assert worst <= 4 * U * np.abs(c.v).max()


def test_what_no_query_sees_is_not_read():
    """NaN in keys and values behind a sequence's length, infinities in a cache's room."""
    c = Case(2, 2, 2, 64, 100, 200, lens=[130, 3])
    want = c.forward()[0].clone()
    c.k[0, 130:], c.v[0, 130:], c.k[1, 3:], c.v[1, 3:] = np.nan, np.inf, np.inf, np.nan
    assert torch.equal(c.forward()[0], want)


def test_buckets_outside_the_table_have_no_bias():
    c = Case(1, 2, 2, 64, 150, 150, far=8, buckets=4)
    c.bucket[::2] = -1
    c.bucket[1] = 4
    keep = c.table.copy()
    wide = np.concatenate((keep, np.zeros((1, 2), np.float32)))
    O = c.forward()[0]
    plain = list(c.plain())
    plain[3], plain[4] = wide, np.where((c.bucket < 0) | (c.bucket >= 4), 4, c.bucket)
    o, _, p = OE.attention_bias(*plain)
    assert np.abs(host_bf16(O) - o).max() <= 3 * U * np.abs(c.v).max()


def test_buckets_of_the_host_call():
    for n, far, both in ((32, 128, True), (32, 128, False), (8, 8, False), (64, 512, True), (16, 500, True), (12, 100, True), (2, 7, False), (4, 3, True)):
        assert B.chorus_bias_buckets(n, far, both).tolist() == OE.bias_buckets(n, far, both).tolist(), (n, far, both)


def backward(c, ws=None):
    O, lse, rest, _ = c.forward()
    Q, K, V, _, table, bucket = c.dev
    dO = c.place(c.do)[0]
    (dQ, rq), (dK, rk), (dV, rv) = (c.place(np.full(t.shape, 7.0)) for t in (c.q, c.k, c.v))
    dtable = torch.full(c.table.shape, float("nan"), device=DEV)
    B.chorus_attention_bias_backward(Q, K, V, O, rest, lse, dO, table, bucket, dQ, dK, dV, dtable, ws=ws, **c.how())
    return (dQ, dK, dV, dtable), (rq, rk, rv)


@pytest.mark.parametrize("layout", ["apart", "packed"])
@pytest.mark.parametrize("i", range(len(FORWARD)))
def test_backward(i, layout):
    c = Case(**FORWARD[i], layout=layout)
    got, rooms = backward(c)
    want, size = OE.attention_bias_backward(*c.plain(), c.do)
    for name, g, w, m in zip(("dq", "dk", "dv"), got, want, size):
        tol = 1.1 * U * m + U * np.abs(w) + 1e-30
        off = np.abs(host_bf16(g) - w)
        assert (off <= tol).all(), (name, float((off - tol).max()))
    off = np.abs(host(got[3]).astype(np.float64) - want[3])
    print("[parity] dtable", float(np.linalg.norm(off) / max(np.linalg.norm(want[3]), 1e-30)))
    assert (off <= 2.0 ** -14 * size[3] + 1e-30).all(), float((off - 2.0 ** -14 * size[3]).max())
    if layout == "apart":
        for room, rows, width in zip(rooms, (c.Lq, c.Lk, c.Lk), (c.H, c.Hk, c.Hk)):
            assert (room[:, rows:] == 3).all() and (room[:, :, :8] == 3).all() and (room[:, :, 8 + width * c.dh:] == 3).all()


def test_gradients_of_what_is_not_seen_are_zeros():
    c = Case(3, 2, 1, 64, 70, 150, lens=[0, 150, 9], first=[0, 500, 0], causal=True)
    c.k[2, 9:], c.v[2, 9:], c.k[0], c.v[0] = np.nan, np.nan, np.inf, np.nan
    (dQ, dK, dV, dtable), _ = backward(c)
    assert not host_bf16(dQ)[0].any() and not host_bf16(dK)[0].any() and not host_bf16(dV)[0].any()
    assert not host_bf16(dK)[2, 9:].any() and not host_bf16(dV)[2, 9:].any()
    assert all(np.isfinite(host(t.float())).all() for t in (dQ, dK, dV, dtable))


def test_table_gradients_are_exact_enough_to_cancel():
    """The sums of a row's gradients are 0: so is the sum of a head's table gradients, against terms that are not small."""
    c = Case(2, 4, 4, 64, 500, 500, lens=[500, 400])
    (_, _, _, dtable), _ = backward(c)
    _, size = OE.attention_bias_backward(*c.plain(), c.do)
    assert (np.abs(host(dtable).sum(0)) <= 2.0 ** -14 * size[3].sum(0)).all()


@pytest.mark.parametrize("Lq,Lk", [(1, 900), (200, 200)])
def test_results_do_not_depend_on_the_call(Lq, Lk):
    """Twice eagerly, on another stream, and in a captured graph that is replayed with eager calls between: equal bits; new lengths at a replay."""
    c = Case(2, 4, 2, 64, Lq, Lk, lens=[Lk, Lk // 2], first=[0, 5], causal=Lq > 1)
    Q, K, V, dO = (c.place(t)[0] for t in (c.q, c.k, c.v, c.do))
    table, bucket, lens, first = dev_f32(c.table), _i32(c.bucket), _i32(c.lens), _i32(c.first)

    def buffers():
        e = lambda t: torch.zeros(t.shape, dtype=BF, device=DEV)  # noqa: E731
        return [e(Q), e(Q), torch.zeros(2, 4, Lq, device=DEV), e(Q), e(K), e(V), torch.zeros(c.table.shape, device=DEV)]

    def step(o, rest, lse, dq, dk, dv, dt):
        how = dict(lens=lens, first=first, causal=c.causal, scale=c.scale)
        B.chorus_attention_bias(Q, K, V, o, table, bucket, lse=lse, rest=rest, **how)
        B.chorus_attention_bias_backward(Q, K, V, o, rest, lse, dO, table, bucket, dq, dk, dv, dt, **how)

    want, other, captured = buffers(), buffers(), buffers()
    step(*want)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step(*captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(*captured)
    for n in (c.lens, [Lk // 3, 0], [1, Lk], c.lens):
        lens.copy_(_i32(n))
        for t in captured:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        step(*other)
        torch.cuda.synchronize()
        for a, b in zip(other, captured):
            assert torch.equal(_bits(a), _bits(b))
    for a, b in zip(want, other):
        assert torch.equal(_bits(a), _bits(b))
