"""CPU checks of a text encoder's operators and of the 8-bit products: refusals (each call returns before any device work), and the plain
forms that the GPU tests compare with against differences and brute force."""
import ctypes as C

import numpy as np
import pytest

from oracle import encoder as OE
import paper_2604_04451_amd as P
from paper_2604_04451_amd import binding as B

NULL, P16, P8 = C.c_void_p(0), C.c_void_p(16), C.c_void_p(8)


def _quant(lib, X=P16, ld=256, out=P16, scale=P16, M=4, K=200, Kp=256):
    return lib.chorus_quant_rows_i8(X, ld, out, scale, M, K, Kp, NULL)


@pytest.mark.parametrize("change,want", [
    (dict(M=-1), B.E_ARG), (dict(K=0), B.E_ARG), (dict(Kp=192), B.E_ARG), (dict(ld=192), B.E_ARG), (dict(X=NULL), B.E_ARG),
    (dict(out=NULL), B.E_ARG), (dict(scale=NULL), B.E_ARG), (dict(X=P8), B.E_ARG), (dict(out=P8), B.E_ARG), (dict(scale=P8), B.E_ARG),
    (dict(K=196), B.E_SHAPE), (dict(Kp=260), B.E_SHAPE), (dict(ld=260), B.E_SHAPE), (dict(M=1 << 23), B.E_SHAPE), (dict(M=0, X=NULL), B.OK),
])
def test_quant_rows_refuses(change, want):
    assert _quant(P.load(), **change) == want


def _i8(lib, A=P16, sa=P16, W=P16, sw=P16, M=4, N=64, K=256, epilogue=0, out=P16, bias=NULL, gate0=NULL, gate1=NULL, scale=1.0):
    return lib.chorus_gemm_i8(A, sa, W, sw, M, N, K, epilogue, out, bias, gate0, gate1, scale, NULL)


@pytest.mark.parametrize("change,want", [
    (dict(M=-1), B.E_ARG), (dict(N=0), B.E_ARG), (dict(K=0), B.E_ARG), (dict(epilogue=4), B.E_ARG), (dict(epilogue=-1), B.E_ARG),
    (dict(A=NULL), B.E_ARG), (dict(sa=NULL), B.E_ARG), (dict(W=NULL), B.E_ARG), (dict(sw=NULL), B.E_ARG), (dict(out=NULL), B.E_ARG),
    (dict(A=P8), B.E_ARG), (dict(W=P8), B.E_ARG), (dict(sa=P8), B.E_ARG), (dict(sw=P8), B.E_ARG), (dict(out=P8), B.E_ARG),
    (dict(bias=P8), B.E_ARG), (dict(gate0=P8), B.E_ARG), (dict(gate1=P8), B.E_ARG), (dict(K=64), B.E_SHAPE), (dict(K=320), B.E_SHAPE),
    (dict(K=131072 + 128), B.E_SHAPE), (dict(N=12), B.E_SHAPE), (dict(M=1 << 40, N=1 << 20), B.E_SHAPE), (dict(M=0, A=NULL), B.OK),
])
def test_gemm_i8_refuses(change, want):
    assert _i8(P.load(), **change) == want


def _gated(lib, X=P16, W=P16, act=0, H=P16, pre=NULL, M=4, F=128, K=64):
    return lib.chorus_gated_ffn(X, W, act, H, pre, M, F, K, NULL)


def _gated_back(lib, X=P16, W=P16, pre=P16, dH=P16, act=0, dX=P16, dW=P16, epilogue=0, M=4, F=128, K=64, ws=P16, ws_bytes=1 << 30):
    return lib.chorus_gated_ffn_backward(X, W, pre, dH, act, dX, dW, epilogue, M, F, K, ws, ws_bytes, NULL)


SIZES = [(dict(M=-1), B.E_ARG), (dict(F=0), B.E_ARG), (dict(K=-64), B.E_ARG), (dict(act=2), B.E_ARG), (dict(act=-1), B.E_ARG), (dict(X=NULL), B.E_ARG),
         (dict(W=NULL), B.E_ARG), (dict(X=P8), B.E_ARG), (dict(W=P8), B.E_ARG), (dict(pre=P8), B.E_ARG), (dict(K=96), B.E_SHAPE), (dict(F=96), B.E_SHAPE),
         (dict(K=(1 << 20) + 64), B.E_SHAPE), (dict(F=(1 << 20) + 64), B.E_SHAPE), (dict(M=(1 << 22) + 1), B.E_SHAPE)]


@pytest.mark.parametrize("change,want", SIZES + [(dict(H=NULL), B.E_ARG), (dict(H=P8), B.E_ARG), (dict(M=0, X=NULL), B.OK)])
def test_gated_refuses(change, want):
    assert _gated(P.load(), **change) == want


@pytest.mark.parametrize("change,want", SIZES + [
    (dict(pre=NULL), B.E_ARG), (dict(dH=NULL), B.E_ARG), (dict(dH=P8), B.E_ARG), (dict(dX=P8), B.E_ARG), (dict(dW=P8), B.E_ARG), (dict(ws=P8), B.E_ARG),
    (dict(epilogue=1), B.E_ARG), (dict(epilogue=4), B.E_ARG), (dict(ws=NULL), B.E_WORKSPACE), (dict(ws_bytes=1000), B.E_WORKSPACE), (dict(M=0), B.E_SHAPE),
])
def test_gated_backward_refuses(change, want):
    assert _gated_back(P.load(), **change) == want


def _bias(**change):
    a = B.BiasAttention(40, 50, 2, 4, 2, 64, 32, 128, 0, 1.0, 256, 40 * 256, 128, 50 * 128, 128, 50 * 128, 256, 40 * 256)
    for n, v in change.items():
        setattr(a, n, v)
    return a


def _attend(lib, a, Q=P16, K=P16, V=P16, O=P16, rest=NULL, lse=NULL, table=P16, bucket=P16, lens=NULL, first=NULL, ws=NULL, ws_bytes=0):
    return lib.chorus_attention_bias(C.byref(a) if a is not None else None, Q, K, V, O, rest, lse, table, bucket, lens, first, ws, ws_bytes, NULL)


SHAPES = [(dict(B=-1), B.E_ARG), (dict(Lq=-1), B.E_ARG), (dict(Lk=-1), B.E_ARG), (dict(H=0), B.E_ARG), (dict(Hk=0), B.E_ARG), (dict(n_buckets=0), B.E_ARG),
          (dict(far=-1), B.E_ARG), (dict(scale=0.0), B.E_ARG), (dict(scale=-1.0), B.E_ARG), (dict(scale=float("nan")), B.E_ARG),
          (dict(scale=float("inf")), B.E_ARG), (dict(scale=2.0 ** -31), B.E_ARG), (dict(scale=2.0 ** 31), B.E_ARG), (dict(dh=96), B.E_SHAPE), (dict(dh=32), B.E_SHAPE), (dict(Hk=3), B.E_SHAPE), (dict(far=513), B.E_SHAPE),
          (dict(Lq=(1 << 28) + 1), B.E_SHAPE), (dict(Lk=(1 << 28) + 1), B.E_SHAPE), (dict(q_row=248), B.E_SHAPE), (dict(k_row=120), B.E_SHAPE),
          (dict(v_row=132), B.E_SHAPE), (dict(o_row=(1 << 23) + 8), B.E_SHAPE), (dict(q_batch=4), B.E_SHAPE), (dict(k_batch=-8), B.E_SHAPE),
          (dict(B=1 << 20, Lq=1 << 12), B.E_SHAPE), (dict(B=1 << 20, Lk=1 << 12), B.E_SHAPE), (dict(H=1 << 17, q_row=1 << 23, o_row=1 << 23), B.E_SHAPE)]


@pytest.mark.parametrize("change,want", SHAPES + [(dict(B=0), B.OK), (dict(Lq=0), B.OK)])
def test_attention_bias_refuses_shapes(change, want):
    assert _attend(P.load(), _bias(**change)) == want


@pytest.mark.parametrize("change,want", [(dict(Q=NULL), B.E_ARG), (dict(K=NULL), B.E_ARG), (dict(V=NULL), B.E_ARG), (dict(O=NULL), B.E_ARG),
                                         (dict(table=NULL), B.E_ARG), (dict(bucket=NULL), B.E_ARG), (dict(Q=P8), B.E_ARG), (dict(K=P8), B.E_ARG),
                                         (dict(V=P8), B.E_ARG), (dict(O=P8), B.E_ARG), (dict(rest=P8), B.E_ARG), (dict(lse=P8), B.E_ARG),
                                         (dict(table=P8), B.E_ARG), (dict(bucket=P8), B.E_ARG), (dict(lens=P8), B.E_ARG), (dict(first=P8), B.E_ARG),
                                         (dict(ws=P8), B.E_ARG)])
def test_attention_bias_refuses_pointers(change, want):
    assert _attend(P.load(), _bias(), **change) == want
    assert _attend(P.load(), None) == B.E_ARG


def test_attention_bias_workspace():
    lib = P.load()
    size = lib.chorus_attention_bias_workspace_bytes
    few = _bias(Lk=4096, Lq=40)
    assert size(C.byref(few)) > 0 and size(C.byref(_bias(B=1024))) == 0 and size(C.byref(_bias(dh=96))) == 0 and size(None) == 0
    assert _attend(lib, few, ws=P16, ws_bytes=size(C.byref(few)) - 1) == B.E_WORKSPACE and _attend(lib, few) == B.E_WORKSPACE


STEPS = dict(do_row=256, do_batch=10240, dq_row=256, dq_batch=10240, dk_row=128, dk_batch=6400, dv_row=128, dv_batch=6400)


def _attend_back(lib, a, steps=None, Q=P16, K=P16, V=P16, O=P16, rest=P16, lse=P16, dO=P16, table=P16, bucket=P16, lens=NULL, first=NULL, dQ=P16, dK=P16,
                 dV=P16, dtable=P16, ws=P16, ws_bytes=1 << 40):
    st = B.BiasAttentionSteps(**{**STEPS, **(steps or {})})
    return lib.chorus_attention_bias_backward(C.byref(a), C.byref(st), Q, K, V, O, rest, lse, dO, table, bucket, lens, first, dQ, dK, dV, dtable, ws,
                                              ws_bytes, NULL)


@pytest.mark.parametrize("change,want", SHAPES + [(dict(B=0), B.E_SHAPE), (dict(Lq=0), B.E_SHAPE), (dict(Lk=0), B.E_SHAPE)])
def test_attention_bias_backward_refuses_shapes(change, want):
    assert _attend_back(P.load(), _bias(**change)) == want


@pytest.mark.parametrize("change,want", [(dict([(n, v)]), B.E_ARG) for n in ("Q", "K", "V", "O", "rest", "lse", "dO", "table", "bucket", "dQ", "dK", "dV",
                                                                              "dtable") for v in (NULL, P8)] +
                         [(dict(lens=P8), B.E_ARG), (dict(first=P8), B.E_ARG), (dict(ws=P8), B.E_ARG), (dict(ws=NULL), B.E_WORKSPACE),
                          (dict(ws_bytes=1000), B.E_WORKSPACE), (dict(steps=dict(do_row=248)), B.E_SHAPE), (dict(steps=dict(dq_batch=4)), B.E_SHAPE),
                          (dict(steps=dict(dk_row=1 << 24)), B.E_SHAPE), (dict(steps=dict(dv_batch=-8)), B.E_SHAPE)])
def test_attention_bias_backward_refuses_pointers(change, want):
    assert _attend_back(P.load(), _bias(), **change) == want


@pytest.mark.parametrize("n,far,both", [(32, 128, 1), (32, 128, 0), (8, 8, 0), (64, 512, 1), (16, 500, 1), (12, 100, 1), (2, 7, 0), (4, 3, 1), (20, 11, 1)])
def test_bias_buckets(n, far, both):
    out = (C.c_int32 * (2 * far + 1))()
    assert P.load().chorus_bias_buckets(n, far, both, out) == B.OK
    assert list(out) == OE.bias_buckets(n, far, bool(both)).tolist()


def test_bias_buckets_refuses():
    lib, out = P.load(), (C.c_int32 * 4096)()
    for n, far, both, to, want in ((1, 8, 0, out, B.E_ARG), (2, 8, 1, out, B.E_ARG), (33, 128, 1, out, B.E_ARG), (0, 8, 0, out, B.E_ARG),
                                   (32, 128, 1, None, B.E_ARG), (32, 513, 1, out, B.E_SHAPE), (32, 8, 1, out, B.E_SHAPE), (32, -1, 0, out, B.E_SHAPE)):
        assert lib.chorus_bias_buckets(n, far, both, to) == want, (n, far, both)


def test_gated_backward_workspace():
    size = P.load().chorus_gated_ffn_backward_workspace_bytes
    M, F, K = 100, 128, 64
    assert size(M, F, K) >= 2 * (M * 2 * F + 128 * 2 * F + 128 * K + 2 * F * K)
    assert size(0, F, K) == 0 and size(M, 96, K) == 0 and size(M, F, 1 << 21) == 0
    lib = P.load()
    assert _gated_back(lib, ws_bytes=size(4, 128, 64) - 1) == B.E_WORKSPACE


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_plain_gated_gradients_against_differences(act):
    rng = np.random.default_rng(1)
    x, w, dh = rng.standard_normal((3, 5)), rng.standard_normal((8, 5)), rng.standard_normal((3, 4))
    dx, dw, _ = OE.gated_backward(x, w, x @ w.T, dh, act)
    loss = lambda: float((OE.gated(x, w, act)[0] * dh).sum())  # noqa: E731
    for t, d in ((x, dx), (w, dw)):
        for i in np.ndindex(t.shape):
            keep = t[i]
            t[i] = keep + 1e-6
            up = loss()
            t[i] = keep - 1e-6
            down = loss()
            t[i] = keep
            assert abs((up - down) / 2e-6 - d[i]) < 1e-7 * (1 + abs(d[i])) * 10


def test_plain_attention_gradients_against_differences():
    rng = np.random.default_rng(2)
    B_, Lq, Lk, H, Hk, dh = 2, 4, 5, 2, 1, 3
    q, k, v, do = (rng.standard_normal(s) for s in ((B_, Lq, H, dh), (B_, Lk, Hk, dh), (B_, Lk, Hk, dh), (B_, Lq, H, dh)))
    table, bucket = rng.standard_normal((4, H)), OE.bias_buckets(4, 3, True)
    for causal, lens, first in ((False, [5, 3], [0, 0]), (True, [5, 4], [1, -2]), (False, [0, 2], [0, 1])):
        grads, _ = OE.attention_bias_backward(q, k, v, table, bucket, lens, first, causal, 0.7, do)
        loss = lambda: float((OE.attention_bias(q, k, v, table, bucket, lens, first, causal, 0.7)[0] * do).sum())  # noqa: E731
        for t, d in zip((q, k, v, table), grads):
            for i in np.ndindex(t.shape):
                keep = t[i]
                t[i] = keep + 1e-6
                up = loss()
                t[i] = keep - 1e-6
                down = loss()
                t[i] = keep
                assert abs((up - down) / 2e-6 - d[i]) < 1e-7 * (1 + abs(d[i]))


def test_plain_codes():
    codes, scale = OE.quant_rows_i8([[1.0, -0.5, 0.25, 2.0], [0.0, 0.0, 0.0, 0.0], [np.inf, 1.0, 0.0, 0.0]])
    assert codes.tolist() == [[64, -32, 16, 127], [0, 0, 0, 0], [0, 0, 0, 0]]  # 63.5 and 31.75, 15.875
    assert scale[0] == 2.0 / 127 and scale[1] == 0 and np.isnan(scale[2])
