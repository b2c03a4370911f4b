"""Attention over selected blocks of keys and what feeds it (axis rotations, block means, block choice) on the GPU through the C ABI,
against plain fp64 forms. Tolerances, in roundings of bf16 (u = 2^-8 relative, half a step):
  attention  the weights and the result are rounded to bf16 and the sum of the weights may be that of the rounded ones: u A + 2 u |O| where A
             is the attention with |V| for V; fp32 logits of up to 32 (in powers of two) from 128 products are off by at most 2^-12
             and sums of 64 thousand weights by 2^-12 in practice: 2^-10 A together
  rotation   one rounding of the result, u |y|; in fp32 the angle's fraction of a turn (2^-24), sine, norm and four products: 2^-19 of the
             largest magnitude of the head
  mean       one rounding, u |y|; at most 128 fp32 additions: 2^-17 mean|x|
  choice     exact"""
import numpy as np
import pytest
import torch

from oracle import blocks as OB
import paper_2604_04451_amd as P
from paper_2604_04451_amd import binding as B
from gpu_util import DEV, dev_bf16, dev_f32, host_bf16
import synth

pytestmark = pytest.mark.gpu

U = 2.0 ** -8
BF = torch.bfloat16


def _bf(a):
    return synth.round_bf16(np.ascontiguousarray(a, dtype=np.float32))


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _vt(V, pad):
    """V [Hk, L, dh] -> device [Hk*dh, pad] by the library's transposition."""
    Hk, L, dh = V.shape
    out = torch.empty(Hk * dh, pad, dtype=BF, device=DEV)
    return B.chorus_v_transpose(dev_bf16(V.transpose(1, 0, 2).reshape(L, Hk * dh)), 0, out, L)


def _pad(X, pad, fill=0.0):
    out = np.full((X.shape[0], pad, X.shape[2]), fill, np.float32)
    out[:, :X.shape[1]] = X
    return out


def _lists(rng, H, Lq, Lk, keep, kind):
    nq, nk = -(-Lq // 128), -(-Lk // 64)
    out = np.full((H, nq, keep), -1, np.int64)
    for h in range(H):
        for a in range(nq):
            n = min(keep, nk) if kind == "full" else rng.integers(0, min(keep, nk) + 1)
            b = rng.permutation(nk)[:n]
            if kind == "full":
                out[h, a, :n] = np.sort(b)
            else:  # any order, gaps anywhere, entries beyond the last block
                at = np.sort(rng.permutation(keep)[:n])
                out[h, a] = rng.choice([-1, nk, nk + 70, -2 ** 31, 2 ** 31 - 1], keep)
                out[h, a, at] = b
    return out


def _near(got, O, A):
    assert np.isfinite(got).all()
    off = np.abs(got - O) - ((U + 2.0 ** -10) * A + 2 * U * np.abs(O) + 1e-30)
    assert off.max(initial=-1.0) <= 0, f"{off.max():.3e} over its tolerance at {np.unravel_index(off.argmax(), off.shape)}"


CASES = [  # H, Hk, dh, Lq, Lk, keep, kind
    (4, 2, 64, 130, 130, 3, "full"), (1, 1, 128, 1, 1, 1, "full"), (2, 2, 128, 1, 64, 1, "full"), (2, 1, 64, 5, 65, 2, "full"),
    (3, 1, 64, 129, 1000, 20, "gaps"), (5, 5, 128, 300, 777, 13, "gaps"), (8, 4, 128, 128, 4096, 64, "full"),
    (2, 2, 128, 1, 20001, 313, "full"), (3, 3, 64, 1, 20001, 400, "gaps"), (2, 2, 128, 127, 9000, 141, "gaps"),
    (12, 12, 128, 1500, 1500, 6, "full"), (6, 3, 64, 2000, 3001, 47, "gaps"), (1, 1, 128, 4096, 128, 2, "full"),
]


@pytest.mark.parametrize("H,Hk,dh,Lq,Lk,keep,kind", CASES)
@pytest.mark.parametrize("prescaled", [False, True])
def test_attention_blocks(H, Hk, dh, Lq, Lk, keep, kind, prescaled):
    print(f"[case] attention_blocks H={H} Hk={Hk} dh={dh} Lq={Lq} Lk={Lk} keep={keep} {kind} prescaled={prescaled}", flush=True)
    rng = np.random.default_rng(Lq * 7 + Lk)
    c = float(np.log2(np.e) / np.sqrt(dh)) if prescaled else 1.0
    Q, K, V = _bf(rng.standard_normal((H, Lq, dh)) * c), _bf(rng.standard_normal((Hk, Lk, dh))), _bf(rng.standard_normal((Hk, Lk, dh)))
    lists = _lists(rng, H, Lq, Lk, keep, kind)
    O, A = OB.attention_blocks(Q, K, V, lists, Lq, Lk, prescaled)
    pad = -(-Lk // 64) * 64
    got = torch.full((Lq + 3, H * dh), 7.0, dtype=BF, device=DEV)
    B.chorus_attention_blocks(dev_bf16(_pad(Q, Lq + 5)), dev_bf16(_pad(K, pad)), _vt(V, pad), got, _i32(lists), Lq, Lk, prescaled)
    _near(host_bf16(got[:Lq]), O, A)
    assert (got[Lq:] == 7.0).all()  # rows behind the last query stay as they were


@pytest.mark.parametrize("dh", [64, 128])
def test_attention_blocks_reads_what_is_listed(dh):
    """NaN in every block that no list names, a block named twice, blocks of logits of -inf, large logits of both signs."""
    print(f"[case] attention_blocks unlisted NaN, twice, -inf dh={dh}", flush=True)
    rng = np.random.default_rng(dh)
    H, Lq, Lk = 2, 200, 640
    Q, K, V = (_bf(rng.standard_normal((H, n, dh))) for n in (Lq, Lk, Lk))
    lists = np.array([[[1, 4, 4, -1], [7, -1, -1, 2]], [[-1, 9, -1, 5], [-1, -1, -1, -1]]])
    for h in range(H):
        for b in set(range(10)) - set(lists[h].ravel().tolist()):
            K[h, b * 64:(b + 1) * 64] = np.nan
            V[h, b * 64:(b + 1) * 64] = np.nan
    O, A = OB.attention_blocks(Q, K, V, lists, Lq, Lk)
    got = torch.empty(Lq, H * dh, dtype=BF, device=DEV)
    B.chorus_attention_blocks(dev_bf16(Q), dev_bf16(K), _vt(V, Lk), got, _i32(lists), Lq, Lk)
    _near(host_bf16(got), O, A)
    assert not host_bf16(got)[128:, dh:].any()  # no block at all
    # positive queries see -inf keys as no keys, whichever block comes first; a row that sees nothing else is zeros
    Q, K, V = np.abs(Q), np.nan_to_num(K), np.nan_to_num(V)
    K[:, 64:128] = -np.inf
    lists = np.array([[[1, 4, -1], [4, 1, 2]], [[1, -1, -1], [3, 5, 1]]])
    O, A = OB.attention_blocks(Q, K, V, lists, Lq, Lk)
    B.chorus_attention_blocks(dev_bf16(Q), dev_bf16(K), _vt(V, Lk), got, _i32(lists), Lq, Lk)
    _near(host_bf16(got), O, A)
    assert not host_bf16(got)[:128, dh:].any()
    # logits around -1000 and +1000 (powers of 64: exact products): the running maximum moves far, up and down
    Q = np.full((H, Lq, dh), 8.0, np.float32)
    K = np.zeros((H, Lk, dh), np.float32)
    for b in range(10):
        K[:, b * 64:(b + 1) * 64, 0] = (-1) ** b * 64.0 * np.sqrt(dh) / 8 * (b + 1) / 8
    K = _bf(K)
    for order in ([0, 2, 4, 8], [8, 4, 2, 0], [1, 3, 5, 7], [9, 7, 1, 3]):
        lists = np.broadcast_to(np.array(order), (H, 2, 4))
        O, A = OB.attention_blocks(Q, K, V, lists, Lq, Lk)
        B.chorus_attention_blocks(dev_bf16(Q), dev_bf16(K), _vt(V, Lk), got, _i32(lists), Lq, Lk)
        _near(host_bf16(got), O, A)


def test_attention_blocks_all_blocks_is_dense_attention():
    print("[case] attention_blocks with every block against chorus_attention", flush=True)
    rng = np.random.default_rng(5)
    H, dh, L = 4, 128, 1000
    Q, K, V = (_bf(rng.standard_normal((H, L, dh))) for _ in range(3))
    dQ, dK, dV = dev_bf16(_pad(Q, 1024)), dev_bf16(_pad(K, 1024)), _vt(V, 1024)
    a, b = torch.empty(L, H * dh, dtype=BF, device=DEV), torch.empty(L, H * dh, dtype=BF, device=DEV)
    B.chorus_attention(dQ, dK, dV, a, None, L, L)
    lists = torch.arange(16, dtype=torch.int32, device=DEV).expand(H, 8, 16).contiguous()
    B.chorus_attention_blocks(dQ, dK, dV, b, lists, L, L)
    O, A = OB.attention_blocks(Q, K, V, lists.cpu().numpy(), L, L)
    _near(host_bf16(a), O, A)
    _near(host_bf16(b), O, A)


def test_attention_blocks_beyond_32_bits():
    """Keys and values of more than 2^31 values: the last head's last blocks."""
    H, dh, Lk, Lq = 40, 128, 430016, 3
    print(f"[case] attention_blocks {H} heads of {Lk} keys", flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    K = torch.zeros(H, Lk, dh, dtype=BF, device=DEV)
    Vt = torch.zeros(H * dh, Lk, dtype=BF, device=DEV)
    Q = torch.empty(H, Lq, dh, device=DEV).normal_(generator=g).to(BF)
    tail = 256
    K[-1, -tail:] = torch.empty(tail, dh, device=DEV).normal_(generator=g).to(BF)
    V = torch.empty(tail, dh, device=DEV).normal_(generator=g).to(BF)
    vt = torch.empty(dh, tail, dtype=BF, device=DEV)
    Vt[-dh:, -tail:] = B.chorus_v_transpose(V, 0, vt, tail)
    nk = Lk // 64
    lists = torch.full((H, 1, 6), -1, dtype=torch.int32, device=DEV)
    lists[-1, 0] = torch.tensor([-1, nk - 4, nk - 2, nk, nk - 1, nk + 1], dtype=torch.int32)
    got = torch.empty(Lq, H * dh, dtype=BF, device=DEV)
    B.chorus_attention_blocks(Q, K, Vt, got, lists, Lq, Lk)
    O, A = OB.attention_blocks(host_bf16(Q[-1:]), host_bf16(K[-1:, -tail:]), host_bf16(V)[None], np.array([[[0, 2, 3]]]), Lq, tail)
    _near(host_bf16(got[:, -dh:]), O, A)
    assert not got[:, :-dh].any()


# ------------------------------------------------------------------------------------------------ choice

@pytest.mark.parametrize("H,Hk,dh,nq,nk,keep", [(1, 1, 64, 1, 1, 1), (2, 1, 128, 3, 2, 5), (4, 2, 64, 17, 63, 20), (3, 3, 128, 16, 64, 64),
                                                 (2, 2, 128, 33, 65, 7), (4, 1, 64, 5, 700, 130), (1, 1, 128, 40, 1182, 118),
                                                 (1, 1, 64, 2, 5000, 800), (1, 1, 128, 2, B.BLOCK_SELECT_MAX, 3000)])
@pytest.mark.parametrize("rules", [False, True])
def test_block_select(H, Hk, dh, nq, nk, keep, rules):
    print(f"[case] block_select H={H} Hk={Hk} dh={dh} nq={nq} nk={nk} keep={keep} rules={rules}", flush=True)
    rng = np.random.default_rng(nk + keep)
    Qm, Km = _bf(rng.standard_normal((H, nq, dh))), _bf(rng.standard_normal((Hk, nk, dh)))
    rule = rng.choice([0, 0, 0, 1, 2, 200], nk).astype(np.uint8) if rules else None
    out = torch.full((H, nq, keep), -9, dtype=torch.int32, device=DEV)
    B.chorus_block_select(dev_bf16(Qm), dev_bf16(Km), out, None if rule is None else torch.from_numpy(rule).to(DEV))
    np.testing.assert_array_equal(out.cpu().numpy(), OB.block_select(Qm, Km, keep, rule))


@pytest.mark.parametrize("nk,keep", [(64, 9), (300, 40), (1500, 700)])
def test_block_select_ties(nk, keep):
    """Scores of 0, 1 and 2 times 2^-12, equal by the hundred, between terms of 2^12 and -2^12 that fp32 sums do not cancel in every order;
    zeros of both signs, NaN and infinities."""
    print(f"[case] block_select ties nk={nk} keep={keep}", flush=True)
    rng = np.random.default_rng(nk)
    H, nq, dh = 2, 6, 128
    Qm = np.ones((H, nq, dh), np.float32)
    Qm[:, :, 0::2] = rng.choice([1.0, -1.0], (H, nq, dh // 2))
    Km = np.zeros((H, nk, dh), np.float32)
    Km[:, :, 1] = rng.integers(0, 3, (H, nk)) * 2.0 ** -12
    for h in range(H):
        for k in range(nk):
            i, j = rng.permutation(np.arange(3, dh, 2))[:2]
            Km[h, k, [i, j]] = 4096.0, -4096.0
    Km = _bf(Km)
    Km[:, 5, :] = 0.0
    Km[:, 6, :] = -0.0
    Km[0, 7, 2] = np.nan
    Km[0, 8, 1] = np.inf
    Km[0, 9, 1] = -np.inf
    rule = np.zeros(nk, np.uint8)
    rule[[3, 11]] = 1
    rule[[4, 20]] = 2
    for r in (None, rule):
        out = torch.empty(H, nq, keep, dtype=torch.int32, device=DEV)
        B.chorus_block_select(dev_bf16(Qm), dev_bf16(Km), out, None if r is None else torch.from_numpy(r).to(DEV))
        np.testing.assert_array_equal(out.cpu().numpy(), OB.block_select(Qm, Km, keep, r))


def test_block_select_neighbours_closer_than_fp32():
    """Scores around 2^14 whose differences are 2^-12 of a unit and less: what fp32 sums cannot tell apart decides here."""
    print("[case] block_select near ties", flush=True)
    rng = np.random.default_rng(3)
    nq, nk, dh, keep = 20, 500, 128, 60
    Qm = np.ones((1, nq, dh), np.float32)
    Km = np.full((1, nk, dh), 128.0, np.float32)
    Km[0, :, 5] = rng.permutation(nk) * 2.0 ** -20 * 8
    Km[0, :, 9] = rng.choice([64.0, 128.0], nk)
    Km, Qm = _bf(Km), _bf(Qm)
    Qm[0, :, 5] = _bf(rng.uniform(0.5, 2.0, nq))
    out = torch.empty(1, nq, keep, dtype=torch.int32, device=DEV)
    B.chorus_block_select(dev_bf16(Qm), dev_bf16(Km), out)
    np.testing.assert_array_equal(out.cpu().numpy(), OB.block_select(Qm, Km, keep))


@pytest.mark.parametrize("q_scale,k_scale", [(1.0, 1e-30), (1e-20, 1e-18), (1.0, 1e-39), (1e18, 1e18), (3e18, 3e18), (1e19, 1e19), (1.0, 1e38), (1e-30, 3e38), (0.0, 1.0)])
def test_block_select_far_scales(q_scale, k_scale):
    """Scores that fp32 does not hold, barely holds or flushes, and scores that are all zero: fp64 decides."""
    print(f"[case] block_select scales {q_scale} {k_scale}", flush=True)
    rng = np.random.default_rng(17)
    Qm = _bf(np.clip(rng.standard_normal((2, 5, 128)) / 3, -1, 1) * q_scale)
    Km = _bf(np.clip(rng.standard_normal((2, 300, 128)) / 3, -1, 1) * k_scale)
    out = torch.empty(2, 5, 40, dtype=torch.int32, device=DEV)
    B.chorus_block_select(dev_bf16(Qm), dev_bf16(Km), out)
    np.testing.assert_array_equal(out.cpu().numpy(), OB.block_select(Qm, Km, 40))


# ------------------------------------------------------------------------------------------------ means, rotations

@pytest.mark.parametrize("H,dh,L,block", [(1, 64, 1, 64), (2, 128, 63, 64), (3, 64, 64, 128), (2, 128, 129, 128), (5, 64, 1000, 64),
                                          (4, 128, 1300, 128), (12, 128, 4099, 64)])
def test_block_mean(H, dh, L, block):
    print(f"[case] block_mean H={H} dh={dh} L={L} block={block}", flush=True)
    X = _bf(np.random.default_rng(L).standard_normal((H, L, dh)) * 3 + 0.5)
    n = -(-L // block)
    out = torch.empty(H, n, dh, dtype=BF, device=DEV)
    B.chorus_block_mean(dev_bf16(_pad(X, L + 7, np.nan)), out, L, block)  # padding is not part of a mean
    ref, mag = OB.block_mean(X, L, block), OB.block_mean(np.abs(X), L, block)
    assert (np.abs(host_bf16(out) - ref) <= U * np.abs(ref) + 2.0 ** -17 * mag).all()


@pytest.mark.parametrize("scale", [2.0 ** 126, 2.0 ** -127, 2.0 ** -131])
@pytest.mark.parametrize("dh,block", [(64, 128), (128, 64)])
def test_block_mean_far_scales(dh, block, scale):
    """Values whose sum fp32 does not hold though it holds their mean, and subnormal ones (steps of 2^-133: half a one is allowed)."""
    print(f"[case] block_mean dh={dh} block={block} scale={scale}", flush=True)
    L = 3 * block - 5
    X = _bf(np.random.default_rng(block).uniform(0.25, 3.9, (2, L, dh)) * scale)
    out = torch.empty(2, 3, dh, dtype=BF, device=DEV)
    B.chorus_block_mean(dev_bf16(X), out, L, block)
    ref = OB.block_mean(X, L, block)
    assert (np.abs(host_bf16(out) - ref) <= (U + 2.0 ** -17) * np.abs(ref) + 2.0 ** -134).all()


@pytest.mark.parametrize("H,dh,L,dims", [(4, 64, 130, (16, 24)), (12, 128, 301, (44, 42, 42)), (1, 64, 1, (64,)), (4, 128, 77, (16, 32, 32, 48)),
                                         (40, 128, 33, (96,)), (5, 64, 9, (16, 0, 16)), (7, 128, 5, ())])
@pytest.mark.parametrize("norm", ["none", "width", "head"])
@pytest.mark.parametrize("halves", [False, True])
def test_rope_axes(H, dh, L, dims, norm, halves):
    if halves and sum(dims) % 16:
        dims = tuple(d // 16 * 16 for d in dims)
    print(f"[case] rope_axes H={H} dh={dh} L={L} dims={dims} norm={norm} halves={halves}", flush=True)
    rng = np.random.default_rng(L + dh)
    D, Lpad = H * dh, L + 6
    x = _bf(rng.standard_normal((L, 2 * D + 8)) * 1.5)
    n_axes = max(1, len(dims))
    pos = rng.uniform(-300, 300, (L, n_axes)).astype(np.float32)
    pos[0] = 100003.0  # far along every axis
    if dims:
        freq, axis = (t.numpy() for t in B.chorus_rope_axes_table(dims, device="cpu"))
    else:
        freq, axis = np.zeros(0), np.zeros(0, np.int32)
    if axis.size > 9:
        axis = axis.copy()
        axis[[2, 9]] = [-1, n_axes]  # no such axes: these pairs do not turn
    gain = {"none": None, "width": rng.uniform(0.5, 2, D), "head": rng.uniform(0.5, 2, dh)}[norm]
    gain = None if gain is None else gain.astype(np.float32)
    out = torch.full((H, Lpad, dh), 3.0, dtype=BF, device=DEV)
    B.chorus_rope_axes(dev_bf16(x), D + 8, None if gain is None else dev_f32(gain), {"none": 0, "width": 1, "head": 2}[norm], out, L, H, dh,
                       dev_f32(pos), torch.from_numpy(freq).to(DEV), _i32(axis), B.ROPE_HALVES if halves else B.ROPE_PAIRS, 0.25)
    ref = OB.rope_axes(x[:, D + 8:], gain, norm, H, dh, pos, freq, axis, halves, 0.25)
    got = host_bf16(out)
    assert (np.abs(got[:, :L] - ref) <= U * np.abs(ref) + 2.0 ** -19 * np.abs(ref).max(2, keepdims=True)).all()
    assert not got[:, L:].any()


@pytest.mark.parametrize("H", [9, 14, 18, 27, 30, 41])
@pytest.mark.parametrize("norm,halves", [("width", False), ("width", True), ("head", False), ("head", True)])
def test_rope_axes_widths(H, norm, halves):
    """Rows that fill the registers they are held in partly, and one that is too wide for them."""
    test_rope_axes(H, 128, 5, (16, 48, 32), norm, halves)


def test_rope_axes_of_grid_positions_is_qk_norm_rope():
    """The framework's own rotation is the one of three axes with the grid's positions: same values but for the last roundings."""
    print("[case] rope_axes against qk_norm_rope", flush=True)
    H, dh, grid = 12, 128, (5, 12, 20)
    L = grid[0] * grid[1] * grid[2]
    rng = np.random.default_rng(8)
    x, gain = dev_bf16(rng.standard_normal((L, H * dh))), dev_f32(rng.uniform(0.5, 2, H * dh))
    idx = torch.arange(L, device=DEV)
    pos = torch.stack((idx // 240, idx // 20 % 12, idx % 20), 1).float().contiguous()
    a, b = torch.empty(H, 1280, dh, dtype=BF, device=DEV), torch.empty(H, 1280, dh, dtype=BF, device=DEV)
    B.chorus_qk_norm_rope(x, 0, gain, a, L, H, dh, None, grid, True, 0.3)
    freq, axis = B.chorus_rope_axes_table((44, 42, 42))
    B.chorus_rope_axes(x, 0, gain, B.ROPE_NORM_WIDTH, b, L, H, dh, pos, freq, axis, out_scale=0.3)
    a, b = host_bf16(a), host_bf16(b)
    assert (np.abs(a - b) <= 2 * U * np.abs(b) + 2.0 ** -16 * np.abs(b).max(2, keepdims=True)).all()


# ------------------------------------------------------------------------------------------------ together

def test_attention_blocks_two_calls_at_once():
    """Cut lists on two streams and in two captured graphs, each with a workspace of its own and kept busy for many calls: the bits of a call alone."""
    print("[case] attention_blocks at once", flush=True)
    rng = np.random.default_rng(21)
    H, dh, Lq, Lk, keep = 3, 128, 200, 6400, 90
    need = B.chorus_attention_blocks_workspace_bytes(Lq, H, dh, keep)
    assert need > 0

    def inputs():
        Q, K, V = (_bf(rng.standard_normal((H, n, dh))) for n in (Lq, Lk, Lk))
        return dev_bf16(Q), dev_bf16(K), _vt(V, Lk), torch.zeros(Lq, H * dh, dtype=BF, device=DEV), _i32(_lists(rng, H, Lq, Lk, keep, "gaps"))

    sides = [(inputs(), torch.full((need,), 0xff, dtype=torch.uint8, device=DEV), torch.cuda.Stream()) for _ in range(2)]
    want = []
    for a, ws, _ in sides:
        want.append(B.chorus_attention_blocks(*a, Lq, Lk).clone())
        a[3].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for a, ws, s in sides:
            with torch.cuda.stream(s):
                B.chorus_attention_blocks(*a, Lq, Lk, ws=ws)
    torch.cuda.synchronize()
    assert all(torch.equal(a[3], w) for (a, _, _), w in zip(sides, want))
    graphs = []
    for a, ws, _ in sides:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            B.chorus_attention_blocks(*a, Lq, Lk, ws=ws)
    for _ in range(5):
        for a, _, _ in sides:
            a[3].zero_()
        torch.cuda.synchronize()
        for g, (_, _, s) in zip(graphs, sides):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a[3], w) for (a, _, _), w in zip(sides, want))


def _pipeline(x, V0, gains, pos, freq, axis, L, H, dh, keep, bufs):
    """Projection rows -> attention output, as a caller that runs a block's operations itself calls them."""
    D = H * dh
    B.chorus_rope_axes(x, 0, gains[0], B.ROPE_NORM_WIDTH, bufs["q"], L, H, dh, pos, freq, axis, out_scale=float(np.log2(np.e) / np.sqrt(dh)))
    B.chorus_rope_axes(x, D, gains[1], B.ROPE_NORM_WIDTH, bufs["k"], L, H, dh, pos, freq, axis)
    B.chorus_v_transpose(x, V0, bufs["vt"], L)
    B.chorus_block_mean(bufs["q"], bufs["qm"], L, B.BLOCK_QUERIES)
    B.chorus_block_mean(bufs["k"], bufs["km"], L, B.BLOCK_KEYS)
    B.chorus_block_select(bufs["qm"], bufs["km"], bufs["blocks"], bufs["rule"])
    B.chorus_attention_blocks(bufs["q"], bufs["k"], bufs["vt"], bufs["o"], bufs["blocks"], L, L, prescaled=True, ws=bufs["ws"])


def test_together_on_a_stream_and_in_a_graph():
    """The whole path, stage by stage against the plain forms on what the stage before left; the same bits on another stream and from
    each replay of a captured graph, with eager work on other inputs between the replays."""
    H, dh, L, keep = 4, 64, 1301, 6
    print(f"[case] together H={H} dh={dh} L={L} keep={keep}", flush=True)
    D, pad = H * dh, 1536
    rng = np.random.default_rng(2)
    xs = [_bf(rng.standard_normal((L, 3 * D)) * 1.2) for _ in range(3)]
    gains = [dev_f32(rng.uniform(0.5, 1.5, D)) for _ in range(2)]
    idx = np.arange(L)
    pos = np.stack((idx // 260, idx // 20 % 13 * 1.5, idx % 20 * 1.5), 1).astype(np.float32)
    freq, axis = B.chorus_rope_axes_table((24, 20, 20))
    dpos = dev_f32(pos)
    nq, nk = -(-L // 128), -(-L // 64)
    need = B.chorus_attention_blocks_workspace_bytes(L, H, dh, keep)

    def buffers():
        e = lambda *s: torch.full(s, 5.0, dtype=BF, device=DEV)  # noqa: E731
        rule = torch.zeros(nk, dtype=torch.uint8, device=DEV)
        rule[0] = 1
        return {"q": e(H, pad, dh), "k": e(H, pad, dh), "vt": e(D, pad), "qm": e(H, nq, dh), "km": e(H, nk, dh), "rule": rule,
                "blocks": torch.zeros(H, nq, keep, dtype=torch.int32, device=DEV), "o": e(L, D),
                "ws": torch.full((max(need, 256),), 0xab, dtype=torch.uint8, device=DEV)}

    args = lambda x, b: (x, 2 * D, gains, dpos, freq, axis, L, H, dh, keep, b)  # noqa: E731
    x, b = dev_bf16(xs[0]), buffers()
    _pipeline(*args(x, b))
    want = {n: b[n].clone() for n in ("q", "k", "qm", "km", "blocks", "o")}
    c = float(np.log2(np.e) / np.sqrt(dh))
    for name, col, gain, scale in (("q", 0, gains[0], c), ("k", D, gains[1], 1.0)):
        ref = OB.rope_axes(xs[0][:, col:col + D], gain.cpu().numpy(), "width", H, dh, pos, freq.cpu().numpy(), axis.cpu().numpy(), False, scale)
        assert (np.abs(host_bf16(b[name])[:, :L] - ref) <= U * np.abs(ref) + 2.0 ** -19 * np.abs(ref).max(2, keepdims=True)).all()
    for name, of, block in (("qm", "q", 128), ("km", "k", 64)):
        X = host_bf16(b[of])
        ref = OB.block_mean(X, L, block)
        assert (np.abs(host_bf16(b[name]) - ref) <= U * np.abs(ref) + 2.0 ** -17 * OB.block_mean(np.abs(X), L, block)).all()
    lists = OB.block_select(host_bf16(b["qm"]), host_bf16(b["km"]), keep, b["rule"].cpu().numpy())
    np.testing.assert_array_equal(b["blocks"].cpu().numpy(), lists)
    V = xs[0][:, 2 * D:].reshape(L, H, dh).transpose(1, 0, 2)
    O, A = OB.attention_blocks(host_bf16(b["q"]), host_bf16(b["k"]), V, lists, L, L, True)
    _near(host_bf16(b["o"]), O, A)

    side = torch.cuda.Stream()
    b2 = buffers()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _pipeline(*args(x, b2))
    torch.cuda.synchronize()
    assert all(torch.equal(b2[n], want[n]) for n in want)

    graph, fixed, b3 = torch.cuda.CUDAGraph(), x.clone(), buffers()
    with torch.cuda.graph(graph):
        _pipeline(*args(fixed, b3))
    for i in (0, 1, 2, 0, 1):
        other = dev_bf16(xs[(i + 1) % 3])
        _pipeline(*args(other, b))  # eager work of the same shape between the replays
        torch.cuda.synchronize()
        fixed.copy_(dev_bf16(xs[i]))
        graph.replay()
        torch.cuda.synchronize()
        _pipeline(*args(dev_bf16(xs[i]), b))
        assert all(torch.equal(b3[n], b[n]) for n in want), i
