"""CPU checks of attention over selected blocks and what feeds it: refusals (each call returns before any device work), the table of
rotation frequencies, and the plain forms that the GPU tests compare with against brute force."""
import ctypes as C

import numpy as np
import pytest

from oracle import blocks as OB
import paper_2604_04451_amd as P
from paper_2604_04451_amd import binding as B

NULL, P16, P8 = C.c_void_p(0), C.c_void_p(16), C.c_void_p(8)


def _rope(lib, inp=P16, ld=256, gain=P16, norm=0, out=P16, L=4, Lpad=8, H=4, dh=64, pos=P16, n_axes=2, freq=P16, axis=P16, n_pairs=20,
          layout=0, scale=1.0):
    return lib.chorus_rope_axes(inp, ld, gain, norm, out, L, Lpad, H, dh, pos, n_axes, freq, axis, n_pairs, layout, scale, NULL)


@pytest.mark.parametrize("change,want", [
    (dict(L=-1), B.E_ARG), (dict(Lpad=3), B.E_ARG), (dict(H=0), B.E_ARG), (dict(n_axes=0), B.E_ARG), (dict(n_pairs=-1), B.E_ARG),
    (dict(norm=3), B.E_ARG), (dict(norm=-1), B.E_ARG), (dict(layout=2), B.E_ARG), (dict(scale=0.0), B.E_ARG),
    (dict(scale=float("nan")), B.E_ARG), (dict(scale=float("inf")), B.E_ARG), (dict(inp=NULL), B.E_ARG), (dict(out=NULL), B.E_ARG),
    (dict(pos=NULL), B.E_ARG), (dict(freq=NULL), B.E_ARG), (dict(axis=NULL), B.E_ARG), (dict(norm=1, gain=NULL), B.E_ARG),
    (dict(norm=2, gain=NULL), B.E_ARG), (dict(inp=P8), B.E_ARG), (dict(out=P8), B.E_ARG), (dict(pos=P8), B.E_ARG),
    (dict(dh=96), B.E_SHAPE), (dict(dh=256), B.E_SHAPE), (dict(n_pairs=33), B.E_SHAPE), (dict(layout=1, n_pairs=20), B.E_SHAPE),
    (dict(ld=260), B.E_SHAPE), (dict(ld=248), B.E_SHAPE), (dict(L=0, Lpad=0), B.OK), (dict(L=0, Lpad=1 << 40), B.E_SHAPE),
])
def test_rope_axes_refuses(change, want):
    assert _rope(P.load(), **change) == want


def _mean(lib, X=P16, out=P16, L=100, Lpad=128, H=2, dh=64, block=64):
    return lib.chorus_block_mean(X, out, L, Lpad, H, dh, block, NULL)


@pytest.mark.parametrize("change,want", [
    (dict(L=-1), B.E_ARG), (dict(Lpad=99), B.E_ARG), (dict(H=0), B.E_ARG), (dict(X=NULL), B.E_ARG), (dict(out=P8), B.E_ARG),
    (dict(dh=80), B.E_SHAPE), (dict(block=32), B.E_SHAPE), (dict(block=0), B.E_SHAPE), (dict(L=1 << 40, Lpad=1 << 40), B.E_SHAPE),
    (dict(L=0, X=NULL, out=NULL), B.OK),
])
def test_block_mean_refuses(change, want):
    assert _mean(P.load(), **change) == want


def _select(lib, Qm=P16, Km=P16, rule=NULL, blocks=P16, nq=3, nk=9, H=4, Hk=2, dh=64, keep=4):
    return lib.chorus_block_select(Qm, Km, rule, blocks, nq, nk, H, Hk, dh, keep, NULL)


@pytest.mark.parametrize("change,want", [
    (dict(nq=-1), B.E_ARG), (dict(nk=-1), B.E_ARG), (dict(H=0), B.E_ARG), (dict(Hk=0), B.E_ARG), (dict(keep=0), B.E_ARG),
    (dict(Qm=NULL), B.E_ARG), (dict(Km=NULL), B.E_ARG), (dict(blocks=NULL), B.E_ARG), (dict(Km=P8), B.E_ARG), (dict(rule=P8), B.E_ARG),
    (dict(Hk=3), B.E_SHAPE), (dict(Hk=8), B.E_SHAPE), (dict(dh=32), B.E_SHAPE), (dict(nk=0), B.E_SHAPE),
    (dict(nk=B.BLOCK_SELECT_MAX + 1), B.E_SHAPE), (dict(nq=1 << 30), B.E_SHAPE), (dict(nq=0, Qm=NULL, blocks=NULL), B.OK),
])
def test_block_select_refuses(change, want):
    assert _select(P.load(), **change) == want


def _attend(lib, Q=P16, K=P16, Vt=P16, O=P16, blocks=P16, keep=4, Lq=100, Lk=200, LqPad=128, LkPad=256, H=4, Hk=2, dh=64, pre=0,
            ws=NULL, ws_bytes=0):
    return lib.chorus_attention_blocks(Q, K, Vt, O, blocks, keep, Lq, Lk, LqPad, LkPad, H, Hk, dh, pre, ws, ws_bytes, NULL)


@pytest.mark.parametrize("change,want", [
    (dict(Lq=-1), B.E_ARG), (dict(Lk=-1), B.E_ARG), (dict(LqPad=99), B.E_ARG), (dict(LkPad=192), B.E_ARG), (dict(H=0), B.E_ARG),
    (dict(Hk=0), B.E_ARG), (dict(keep=0), B.E_ARG), (dict(Q=NULL), B.E_ARG), (dict(K=NULL), B.E_ARG), (dict(Vt=NULL), B.E_ARG),
    (dict(O=NULL), B.E_ARG), (dict(blocks=NULL), B.E_ARG), (dict(Q=P8), B.E_ARG), (dict(Vt=P8), B.E_ARG), (dict(blocks=P8), B.E_ARG),
    (dict(ws=P8), B.E_ARG), (dict(Lk=0), B.E_SHAPE), (dict(LkPad=224), B.E_SHAPE), (dict(dh=96), B.E_SHAPE), (dict(Hk=3), B.E_SHAPE),
    (dict(LkPad=1 << 32, Lk=1 << 32), B.E_SHAPE), (dict(LkPad=(1 << 22) + 64), B.E_SHAPE), (dict(Lq=1 << 40, LqPad=1 << 40), B.E_SHAPE),
    (dict(Lq=(1 << 31) - 1, LqPad=1 << 31, H=400, Hk=400), B.E_SHAPE), (dict(Lq=0), B.OK),
    # few lists of many blocks are cut into slices, which need a workspace
    (dict(Lq=1, keep=1000), B.E_WORKSPACE), (dict(Lq=1, keep=1000, ws=P16, ws_bytes=1 << 16), B.E_WORKSPACE),
])
def test_attention_blocks_refuses(change, want):
    assert _attend(P.load(), **change) == want


def test_attention_blocks_workspace():
    """Slices only where lists leave compute units idle, 64 of them at most, 128 rows of fp32 results and 8 bytes each."""
    need = P.load().chorus_attention_blocks_workspace_bytes
    row = lambda dh: 128 * (4 * dh + 8)  # noqa: E731
    assert need(32768, 2, 128, 100) == need(16384, 4, 64, 1000) == 0            # 512 lists: a full round
    for Lq, H, dh, keep in ((1, 1, 128, 5000), (60, 12, 128, 256), (128, 40, 64, 600), (5000, 16, 128, 900)):
        lists = -(-Lq // 128) * H % 512
        n, over = divmod(need(Lq, H, dh, keep), lists * row(dh))
        assert not over and 2 <= n <= min(64, keep), (Lq, H, dh, keep, n)
    assert need(1, 1, 128, 1) == need(128, 4, 64, 3) == 0                       # nothing to cut
    assert need(0, 4, 64, 100) == need(-1, 4, 64, 100) == need(1, 0, 64, 100) == need(1, 4, 96, 100) == need(1, 4, 64, 0) == 0
    assert need(1 << 40, 4, 64, 100) == need((1 << 31) - 1, 1 << 20, 64, 100) == 0


def test_refuses_more_than_a_launch_holds():
    """Rows, lists and entries whose number does not fit a launch or 32 bits are refused, lengths at the end of 64 bits included."""
    lib, most = P.load(), (1 << 63) - 1
    for Lpad in ((1 << 26), most - 2, most):
        assert _rope(lib, Lpad=Lpad) == B.E_SHAPE
    assert _mean(lib, L=1, Lpad=1, H=1 << 26) == _mean(lib, L=most, Lpad=most) == B.E_SHAPE
    assert _select(lib, nq=1, H=1 << 30, Hk=1) == _select(lib, nq=1 << 28) == _select(lib, nq=most) == _select(lib, keep=(1 << 31) - 1) == B.E_SHAPE
    ws = dict(ws=P16, ws_bytes=1 << 62)
    assert _attend(lib, Lq=1, H=1 << 24, Hk=1, **ws) == _attend(lib, Lq=(1 << 31) - 1, LqPad=most, H=1, Hk=1, **ws) == B.E_SHAPE
    assert _attend(lib, Lq=most, LqPad=most, **ws) == _attend(lib, keep=(1 << 31) - 1, **ws) == B.E_SHAPE


def test_rope_axes_table():
    freq, axis = B.chorus_rope_axes_table((16, 24), device="cpu")
    want = [10000.0 ** (-2.0 * i / 16) for i in range(8)] + [10000.0 ** (-2.0 * i / 24) for i in range(12)]
    np.testing.assert_allclose(freq.numpy(), want, rtol=1e-15)
    assert axis.tolist() == [0] * 8 + [1] * 12
    freq, axis = B.chorus_rope_axes_table((44, 42, 42), theta=256.0, device="cpu")
    assert freq.numel() == axis.numel() == 64 and freq[22] == 1.0 and abs(freq[23].item() - 256.0 ** (-2 / 42)) < 1e-15
    assert B.chorus_rope_axes_table((0, 8), device="cpu")[1].tolist() == [1] * 4  # an axis without values has no pairs
    lib = P.load()
    f, a, n = (C.c_double * 64)(), (C.c_int32 * 64)(), C.c_int32(-5)
    call = lambda dims, theta=1e4: lib.chorus_rope_axes_table(len(dims), (C.c_int32 * max(1, len(dims)))(*dims), theta, f, a, C.byref(n))  # noqa: E731
    assert call([]) == B.E_ARG and call([3]) == B.E_ARG and call([-2]) == B.E_ARG and call([64, 66]) == B.E_SHAPE
    assert call([8], 0.0) == B.E_ARG and call([8], float("nan")) == B.E_ARG and call([8], float("inf")) == B.E_ARG
    assert call([2 ** 31 - 2, 2 ** 31 - 2]) == B.E_SHAPE
    assert lib.chorus_rope_axes_table(1, None, 1e4, f, a, C.byref(n)) == B.E_ARG
    assert n.value == -5
    assert call([128]) == B.OK and n.value == 64


def test_plain_forms_against_brute_force():
    """The rotation turns by the angle and keeps the length; the choice is what a full sort of (class, score, index) gives; attention
    over all blocks is dense attention, and over a block listed twice weights it twice."""
    rng = np.random.default_rng(0)
    x, pos = rng.standard_normal((5, 128)), rng.uniform(-50, 50, (5, 2))
    freq, axis = np.array([0.3, 0.01]), np.array([1, 0])
    for halves in (False, True):
        y = OB.rope_axes(x, None, "none", 2, 64, pos, freq, axis, halves)
        a, b = (1, 3) if halves else (2, 3)
        z = (x.reshape(5, 2, 64)[:, 1, a] + 1j * x.reshape(5, 2, 64)[:, 1, b]) * np.exp(1j * pos[:, 0] * 0.01)
        np.testing.assert_allclose(y[1, :, a] + 1j * y[1, :, b], z, atol=1e-12)
        np.testing.assert_allclose(np.linalg.norm(y), np.linalg.norm(x))
        np.testing.assert_array_equal(y[0, :, 4:], x.reshape(5, 2, 64)[:, 0, 4:])
    Km = np.array([[[2.0], [5.0], [5.0], [np.nan], [-1.0], [9.0]]])
    Qm = np.ones((1, 1, 1))
    assert OB.block_select(Qm, Km, 3)[0, 0].tolist() == [1, 2, 5]
    assert OB.block_select(Qm, Km, 2)[0, 0].tolist() == [1, 5]
    assert OB.block_select(Qm, Km, 6)[0, 0].tolist() == [0, 1, 2, 3, 4, 5]
    assert OB.block_select(Qm, Km, 4, np.array([0, 0, 2, 1, 1, 2]))[0, 0].tolist() == [0, 1, 3, 4]
    assert OB.block_select(Qm, Km, 1, np.array([0, 0, 2, 1, 1, 2]))[0, 0].tolist() == [4]
    assert OB.block_select(Qm, Km, 3, np.full(6, 2))[0, 0].tolist() == [-1, -1, -1]
    Q, K, V = rng.standard_normal((2, 70, 8)), rng.standard_normal((1, 130, 8)), rng.standard_normal((1, 130, 8))
    z = Q @ K[0].T / np.sqrt(8)
    w = np.exp(z)
    dense = (w / w.sum(2, keepdims=True)) @ V[0]
    got, _ = OB.attention_blocks(Q, K, V, np.array([[[0, 1, 2]]] * 2), 70, 130)
    np.testing.assert_allclose(got, dense.transpose(1, 0, 2).reshape(70, 16), atol=1e-12)
    w[:, :, :64] *= 2
    w[:, :, 64:128] = 0
    twice = (w / w.sum(2, keepdims=True)) @ V[0]
    got, _ = OB.attention_blocks(Q, K, V, np.array([[[0, 2, 0, -1, 3]]] * 2), 70, 130)
    np.testing.assert_allclose(got, twice.transpose(1, 0, 2).reshape(70, 16), atol=1e-12)
    got, _ = OB.attention_blocks(Q, K, V, np.array([[[-1, 3]]] * 2), 70, 130)
    assert not got.any()
    assert OB.block_mean(np.arange(12.0).reshape(1, 6, 2), 5, 2).tolist() == [[[1, 2], [5, 6], [8, 9]]]
