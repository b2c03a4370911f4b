"""The forms in which the choice of key blocks and the attention over them are launched for large calls, against the plain fp64 forms: workgroups
of 4 to 32 rows of queries, lists some of which go whole and some in slices, lists that are read more than 64 entries at a time. Which form a case
takes is checked first, so that it cannot quietly take another. Tolerance of the attention: the weights and the result are rounded to bf16 and the sum may
be that of the rounded weights, u A + 2 u |O| with A the attention with |V| for V; fp32 logits and sums 2^-10 A. The choice is exact."""
import numpy as np
import pytest
import torch

from oracle import blocks as OB
from paper_2604_04451_amd import binding as B
from gpu_util import DEV, dev_bf16, host_bf16
import synth

pytestmark = pytest.mark.gpu

U = 2.0 ** -8
BF = torch.bfloat16


def _bf(a):
    return synth.round_bf16(np.ascontiguousarray(a, dtype=np.float32))


# ------------------------------------------------------------------------------------------------ choice

def _rows(nq, H, nk):
    """Rows of queries to a workgroup: as few as let all workgroups run at once, 32 or what 155 KB of scores hold at most."""
    R = 4
    while R < 32 and -(-nq // R) * H > 256:
        R *= 2
    while R > 1 and R * (-(-nk // 64) * 64 + 4) * 4 > 155 * 1024:
        R //= 2
    return R


def _choose(Qm, Km, keep, rule=None):
    """OB.block_select row by row with numpy's sort."""
    H, nq, _ = Qm.shape
    Hk, nk, _ = Km.shape
    cls = np.zeros(nk, int) if rule is None else np.where(rule == 1, 0, np.where(rule == 2, 2, 1))
    may = np.flatnonzero(cls != 2)
    out = np.full((H, nq, keep), -1, np.int32)
    for h in range(H):
        s = Qm[h].astype(np.float64) @ Km[h // (H // Hk)].astype(np.float64).T
        order = np.lexsort((np.broadcast_to(may, (nq, may.size)), -s[:, may], np.broadcast_to(cls[may], (nq, may.size))), axis=1)
        best = np.sort(may[order[:, :keep]], axis=1)
        out[h, :, :best.shape[1]] = best
    return out


def _select(Qm, Km, keep, rule):
    H, nq, _ = Qm.shape
    out = torch.full((H, nq, keep), -9, dtype=torch.int32, device=DEV)
    B.chorus_block_select(dev_bf16(Qm), dev_bf16(Km), out, None if rule is None else torch.from_numpy(rule).to(DEV))
    got, want = out.cpu().numpy(), _choose(Qm, Km, keep, rule)
    wrong = np.argwhere((got != want).any(2))
    assert not wrong.size, f"rows {wrong[:8].tolist()} of {len(wrong)}"


SHAPES = [  # H, Hk, nq, nk, rows of a workgroup
    (40, 40, 33, 70, 8), (12, 6, 250, 70, 16), (40, 8, 203, 70, 32), (1, 1, 8200, 130, 32),
    (40, 40, 33, 600, 8), (12, 12, 256, 512, 16), (40, 40, 203, 600, 32), (40, 10, 203, 1216, 32), (40, 10, 203, 1217, 16),
    (40, 20, 203, 1300, 16), (4, 4, 500, 2560, 8), (4, 2, 500, 2600, 8),
]


@pytest.mark.parametrize("H,Hk,nq,nk,R", SHAPES)
@pytest.mark.parametrize("dh", [64, 128])
def test_select_rows_of_a_workgroup(H, Hk, nq, nk, R, dh):
    assert _rows(nq, H, nk) == R
    print(f"[case] block_select H={H} Hk={Hk} nq={nq} nk={nk} dh={dh}, {R} rows a workgroup", flush=True)
    rng = np.random.default_rng(nq + nk + dh)
    Qm, Km = _bf(rng.standard_normal((H, nq, dh))), _bf(rng.standard_normal((Hk, nk, dh)))
    np.testing.assert_array_equal(_choose(Qm[:1, :3], Km[:1], 9), OB.block_select(Qm[:1, :3], Km[:1], 9))
    rule = rng.choice([0, 0, 0, 0, 1, 2], nk).astype(np.uint8)
    for keep, r in ((max(1, nk // 9), None), (nk // 2, rule), (3, rule), (nk + 5, rule)):  # 3: fewer than go ahead of all others
        _select(Qm, Km, keep, r)


@pytest.mark.parametrize("H,Hk,nq,nk,R", [s for s in SHAPES if s[4] > 4 and s[3] != 512])
def test_select_rows_of_a_workgroup_with_ties(H, Hk, nq, nk, R):
    """Neighbouring rows that are settled in three ways: scores equal by the hundred, in threes, and far apart."""
    assert _rows(nq, H, nk) == R
    print(f"[case] block_select ties H={H} nq={nq} nk={nk}, {R} rows a workgroup", flush=True)
    rng = np.random.default_rng(nk)
    dh = 128
    Km = _bf(rng.standard_normal((Hk, nk, dh)))
    Km[:, :, :8] = rng.integers(0, 3, (Hk, nk, 8))
    same = rng.integers(0, max(1, nk // 3), nk)
    Km = Km[:, same]  # each about three times, anywhere
    Qm = _bf(rng.standard_normal((H, nq, dh)))
    kind = rng.integers(0, 3, (H, nq))
    Qm[kind == 0] = np.eye(dh, dtype=np.float32)[rng.integers(0, 8, (kind == 0).sum())]
    Qm[kind == 1, :8] = 0.0
    rule = np.zeros(nk, np.uint8)
    rule[::11], rule[5::13] = 1, 2
    for keep, r in ((nk // 7, None), (nk // 3, rule), (4, rule)):
        _select(Qm, Km, keep, r)


# ------------------------------------------------------------------------------------------------ attention

def _vt(V, pad):
    Hk, L, dh = V.shape
    out = torch.empty(Hk * dh, pad, dtype=BF, device=DEV)
    return B.chorus_v_transpose(dev_bf16(V.transpose(1, 0, 2).reshape(L, Hk * dh)), 0, out, L)


def _pad(X, pad):
    out = np.zeros((X.shape[0], pad, X.shape[2]), np.float32)
    out[:, :X.shape[1]] = X
    return out


def _plan(Lq, H, dh, keep):
    """(lists that go whole, slices of the others) from the workspace, which holds the slices' results."""
    lists = -(-Lq // 128) * H
    need = B.chorus_attention_blocks_workspace_bytes(Lq, H, dh, keep)
    if need == 0:
        return lists, 1
    slices, over = divmod(need, lists % 512 * 128 * (4 * dh + 8))
    assert not over
    return lists - lists % 512, slices


def _allowed(O, A):
    return (U + 2.0 ** -10) * A + 2 * U * np.abs(O) + 1e-30


def _attend(Q, K, V, lists, Lq, Lk, prescaled):
    H, _, dh = Q.shape
    keep, pad = lists.shape[2], -(-Lk // 64) * 64
    need = B.chorus_attention_blocks_workspace_bytes(Lq, H, dh, keep)
    ws = torch.full((max(need, 256),), 0xff, dtype=torch.uint8, device=DEV)  # NaN
    got = torch.full((Lq + 2, H * dh), 7.0, dtype=BF, device=DEV)
    B.chorus_attention_blocks(dev_bf16(Q), dev_bf16(_pad(K, pad)), _vt(V, pad), got,
                              torch.from_numpy(np.ascontiguousarray(lists, dtype=np.int32)).to(DEV), Lq, Lk, prescaled, ws=ws)
    assert (got[Lq:] == 7.0).all()
    return host_bf16(got[:Lq])


def _near(got, O, A):
    assert np.isfinite(got).all()
    off = np.abs(got - O) - _allowed(O, A)
    assert off.max() <= 0, f"{off.max():.3e} over its tolerance at {np.unravel_index(off.argmax(), off.shape)}"


def _scattered(rng, H, nq, nk, keep, most):
    """Up to `most` blocks a list, some lists without any, among entries that are none."""
    out = rng.choice([-1, nk, nk + 70, -2 ** 31, 2 ** 31 - 1], (H, nq, keep))
    for h in range(H):
        for a in range(nq):
            n = rng.integers(0, min(most, nk, keep) + 1)
            out[h, a, rng.permutation(keep)[:n]] = rng.permutation(nk)[:n]
    return out


@pytest.mark.parametrize("H,Hk,dh,Lq,Lk,keep,most", [
    (40, 40, 128, 128 * 14 + 1, 1500, 40, 12),   # 512 whole, 88 cut, the last of each head with one query
    (40, 10, 64, 128 * 27 + 1, 1500, 40, 12),    # 1024 whole, 96 cut
    (3, 3, 128, 128 * 174 - 5, 900, 30, 5),      # 512 whole, 10 cut: a joined row is four waves' work
    (5, 1, 64, 128 * 206 + 77, 2000, 150, 9),    # whole lists of 150 entries
])
@pytest.mark.parametrize("prescaled", [False, True])
def test_attention_whole_and_cut_lists(H, Hk, dh, Lq, Lk, keep, most, prescaled):
    whole, slices = _plan(Lq, H, dh, keep)
    assert whole in (512, 1024) and slices > 1
    print(f"[case] attention_blocks H={H} Hk={Hk} dh={dh} Lq={Lq} Lk={Lk} keep={keep} prescaled={prescaled}: {whole} lists whole, the others in "
          f"{slices} slices", flush=True)
    rng = np.random.default_rng(Lq + dh)
    c = float(np.log2(np.e) / np.sqrt(dh)) if prescaled else 1.0
    Q, K, V = _bf(rng.standard_normal((H, Lq, dh)) * c), _bf(rng.standard_normal((Hk, Lk, dh))), _bf(rng.standard_normal((Hk, Lk, dh)))
    lists = _scattered(rng, H, -(-Lq // 128), -(-Lk // 64), keep, most)
    _near(_attend(Q, K, V, lists, Lq, Lk, prescaled), *OB.attention_blocks(Q, K, V, lists, Lq, Lk, prescaled))


@pytest.mark.parametrize("H,Hk,dh,Lq,Lk,keep,entries", [
    (2, 2, 128, 1, 20001, 313, 7), (3, 3, 64, 1, 20001, 400, 8),
    (1, 1, 128, 5, 64 * 4500 - 9, 4500, 70), (1, 1, 64, 3, 64 * 4300, 4300, 70),  # slices that are read 64 entries at a time
])
def test_attention_misses_no_block(H, Hk, dh, Lq, Lk, keep, entries):
    """Every block of a long list is seen in the result: the values of every second block are 1 in one column, by the block's number, all others 0, and
    logits are small, so that leaving out any of those blocks takes its whole share from that column, which is more than the tolerance allows."""
    whole, slices = _plan(Lq, H, dh, keep)
    assert whole == 0 and keep // slices >= entries
    print(f"[case] attention_blocks counts H={H} dh={dh} Lq={Lq} Lk={Lk} keep={keep}: {slices} slices", flush=True)
    rng = np.random.default_rng(keep)
    nk = -(-Lk // 64)
    Q, K = _bf(rng.standard_normal((H, Lq, dh)) / 8), _bf(rng.standard_normal((Hk, Lk, dh)) / 8)
    lists = np.full((H, 1, keep), -1)
    for h in range(H):
        lists[h, 0, :min(keep, nk)] = rng.permutation(nk)[:keep]
    for part in (0, 1):
        block = np.arange(Lk) // 64
        V = np.zeros((Hk, Lk, dh), np.float32)
        V[:, np.flatnonzero(block % 2 == part), (block // 2 % dh)[block % 2 == part]] = 1.0
        O, A = OB.attention_blocks(Q, K, V, lists, Lq, Lk)
        for h in range(H):
            z = np.exp(Q[h].astype(np.float64) @ K[h // (H // Hk)].astype(np.float64).T / np.sqrt(dh))
            share = np.add.reduceat(z, np.arange(0, Lk, 64), axis=1)
            seen = lists[h, 0][lists[h, 0] >= 0]
            share = share / share[:, seen].sum(1, keepdims=True)
            seen = seen[seen % 2 == part]
            o = O.reshape(Lq, H, dh)[:, h, seen // 2 % dh]
            assert (share[:, seen] > 1.5 * _allowed(o, o)).all()
        _near(_attend(Q, K, V, lists, Lq, Lk, False), O, A)


@pytest.mark.parametrize("H,dh,Lq,keep", [(2, 128, 130, 60), (3, 64, 1, 60), (20, 128, 300, 60)])
def test_attention_joins_far_references(H, dh, Lq, keep):
    """Slices whose logits are a hundred and more apart, up and down, slices of logits of -inf alone, and slices without a block."""
    whole, slices = _plan(Lq, H, dh, keep)
    assert whole == 0 and slices > 1
    print(f"[case] attention_blocks far references H={H} dh={dh} Lq={Lq} keep={keep}: {slices} slices", flush=True)
    rng = np.random.default_rng(dh + Lq)
    nk = 64
    Q = np.abs(_bf(rng.standard_normal((H, Lq, dh)))) + np.float32(2.0 ** -6)
    Q[:, :, 0] = 8.0
    Q = _bf(Q)
    K, V = _bf(rng.standard_normal((H, nk * 64, dh))), _bf(rng.standard_normal((H, nk * 64, dh)))
    K[:, :, 0] = np.repeat(_bf(rng.uniform(-128, 128, nk) * np.sqrt(dh) / 8), 64)
    K[:, 5 * 64:21 * 64] = -np.inf
    nq = -(-Lq // 128)
    lists = np.full((H, nq, keep), -1)
    for h in range(H):
        for a in range(nq):
            for e in range(slices):  # entry e, e + slices, ... are a slice's
                kind = rng.integers(0, 4) if e else 3
                at = np.arange(e, keep, slices)
                of = np.r_[0:5, 21:nk] if kind == 3 else np.arange(5, 21) if kind else np.array([-1])
                lists[h, a, at] = rng.choice(of, at.size)
    lists[-1, -1] = rng.integers(5, 21, keep)  # -inf only: zeros
    O, A = OB.attention_blocks(Q, K, V, lists, Lq, nk * 64)
    got = _attend(Q, K, V, lists, Lq, nk * 64, False)
    _near(got, O, A)
    assert not got[(nq - 1) * 128:, -dh:].any()
