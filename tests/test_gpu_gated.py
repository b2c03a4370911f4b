"""The gated half of a feed-forward block and its gradients on the GPU through the C ABI, against plain fp64 forms. A sum of K products of
bf16 in fp32: products are exact, blocks of 32 are added one behind the other, so at most (K / 32 + 32) 2^-24 sum|x w| =: E; activations
2^-17 of themselves (an exponent of up to 30 rounded to 24 bits) with a slope of at most 1.13; each rounding to bf16 2^-8, to the
16-bit words for the backward pass (9 bits behind the point) 2^-10."""
import numpy as np
import pytest
import torch

from oracle import encoder as OE
import paper_2604_04451_amd as P
from paper_2604_04451_amd import binding as B
from gpu_util import DEV, dev_bf16, dev_f32, host_bf16, host
import synth

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
U, V = 2.0 ** -8, 2.0 ** -17
ACT = {"gelu": B.ACT_GELU, "silu": B.ACT_SILU}


def _bf(a):
    return synth.round_bf16(np.ascontiguousarray(a, dtype=np.float32))


def _sum_error(a, b, n):
    return (n / 32 + 32) * 2.0 ** -24 * (np.abs(a).astype(np.float64) @ np.abs(b).astype(np.float64).T)


def _kept(words):
    """The values of the forward pass's 16-bit words: sign, 6 bits of exponent, 9 behind the point; 0 from 2^-40 down."""
    w = words.view(torch.int16).cpu().numpy().astype(np.int64) & 0xffff
    c = w & 0x7fff
    v = np.ldexp(1.0 + (c & 511) / 512.0, (c >> 9) - 40)
    return np.where(w >> 15, -1.0, 1.0) * np.where(c == 0, 0.0, np.where(c == 0x7fff, np.nan, v))


def _words(values):
    """As the forward pass writes them, halves away from zero."""
    m, e = np.frexp(np.abs(np.asarray(values, np.float64)))
    c = (e - 1 + 40) * 512 + np.floor((2 * m - 1) * 512 + 0.5).astype(np.int64)
    c = np.where((np.abs(values) > 0) & (c > 0), c, 0)
    assert c.max() < 0x7fff
    return torch.from_numpy((c | np.where(np.asarray(values) < 0, 0x8000, 0)).astype(np.uint16).view(np.int16)).to(DEV)


def _inputs(M, F, K):
    rng = np.random.default_rng(M * 3 + F + K)
    return _bf(rng.standard_normal((M, K))), _bf(rng.standard_normal((2 * F, K)) * 1.5 / np.sqrt(K)), _bf(rng.standard_normal((M, F)) * 0.1)


SIZES = [(1, 64, 64), (1, 640, 1024), (3, 64, 128), (16, 128, 4096), (17, 64, 64), (60, 192, 320), (77, 1024, 256), (130, 64, 512), (512, 2048, 256),
         (700, 4160, 128), (1100, 1024, 192)]


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("save", [False, True])
@pytest.mark.parametrize("M,F,K", SIZES + [(4200, 2112, 256)])
def test_forward(M, F, K, act, save):
    x, w, _ = _inputs(M, F, K)
    H = torch.full((M + 1, F), 3.0, dtype=BF, device=DEV)
    pre = torch.full((M + 1, 2 * F), 5.0, dtype=BF, device=DEV)
    B.chorus_gated_ffn(dev_bf16(x), dev_bf16(w), ACT[act], H[:M], pre=pre[:M] if save else None)
    h, want = OE.gated(x, w, act)
    E = _sum_error(x, w, K)
    a = OE.ACT[act][0](want[:, :F])
    tol = (1.13 * E[:, :F] + V * np.abs(a)) * (np.abs(want[:, F:]) + E[:, F:]) + np.abs(a) * E[:, F:]
    got = host_bf16(H)
    assert (np.abs(got[:M] - h) <= tol * (1 + U) + U * np.abs(h)).all()
    assert (got[M] == 3.0).all()
    if save:
        assert (np.abs(_kept(pre[:M]) - want) <= E * (1 + U) + 2.0 ** -10 * np.abs(want) + 2.0 ** -40).all()
    assert (pre[M if save else 0:] == 5.0).all()


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("M,F,K", SIZES)
def test_backward(M, F, K, act):
    x, w, dh = _inputs(M, F, K)
    PRE = _words(x.astype(np.float64) @ w.T.astype(np.float64))
    pre = _kept(PRE)
    X, W, DH = (dev_bf16(t) for t in (x, w, dh))
    dX = torch.full((M, K), float("nan"), dtype=BF, device=DEV)
    dW = torch.full((2 * F, K), float("nan"), dtype=BF, device=DEV)
    B.chorus_gated_ffn_backward(X, W, PRE, DH, ACT[act], dX, dW)
    dx, dw, d = OE.gated_backward(x, w, pre, dh, act)
    # a gradient of a projection: one rounding to bf16; the slope is a sum of two terms below 1.2
    other = np.concatenate((np.abs(dh * pre[:, F:]), np.abs(dh)), 1).astype(np.float64)
    e = (U + V) * np.abs(d) + V * 1.2 * other
    tx = e @ np.abs(w).astype(np.float64) + _sum_error(d, w.T, 2 * F)
    tw = e.T @ np.abs(x).astype(np.float64) + _sum_error(d.T, x.T, M)
    assert (np.abs(host_bf16(dX) - dx) <= tx * (1 + U) + U * np.abs(dx)).all()
    assert (np.abs(host_bf16(dW) - dw) <= tw * (1 + U) + U * np.abs(dw)).all()
    # fp32 weights' gradients, written and added; either gradient alone
    full = torch.full((2 * F, K), float("nan"), device=DEV)
    B.chorus_gated_ffn_backward(X, W, PRE, DH, ACT[act], None, full)
    assert (np.abs(host(full) - dw) <= tw).all()
    before = full.clone()
    B.chorus_gated_ffn_backward(X, W, PRE, DH, ACT[act], None, full, accumulate=True)
    assert (np.abs(host(full).astype(np.float64) - host(before) - dw) <= tw + 2.0 ** -22 * np.abs(host(full))).all()
    alone = torch.full((M, K), float("nan"), dtype=BF, device=DEV)
    B.chorus_gated_ffn_backward(X, W, PRE, DH, ACT[act], alone, None)
    assert torch.equal(alone, dX)


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_far_arguments_of_the_activation(act):
    """Gates from -1e7 to 1e7: the activation is 0 or the gate, its slope 0 or 1, and nothing is NaN; forward alone from -1e30 to 1e30, whose
    projections come back as NaN."""
    K, F = 64, 64
    g = np.array([-1e30, -1e10, -1e7, -300.0, -100.0, -30.0, -16.5, -1e-30, 0.0, 1e-30, 16.5, 30.0, 100.0, 300.0, 1e7, 1e10, 1e30])
    M = len(g)
    x, w, dh = np.zeros((M, K)), np.zeros((2 * F, K)), np.ones((M, F))
    x[:, 0], x[:, 1] = g, 1.0
    w[:F, 0], w[F:, 1] = 1.0, 2.0
    x, w, dh = _bf(x), _bf(w), _bf(dh)
    for rows in (slice(0, M), np.repeat(np.arange(M), 3)):
        X, DH = dev_bf16(x[rows]), dev_bf16(dh[rows])
        m = X.shape[0]
        H, pre = torch.empty(m, F, dtype=BF, device=DEV), torch.empty(m, 2 * F, dtype=BF, device=DEV)
        B.chorus_gated_ffn(X, dev_bf16(w), ACT[act], H, pre=pre)
        with np.errstate(over="ignore"):
            want, p = OE.gated(x[rows], w, act)
            _, _, d = OE.gated_backward(x[rows], w, np.clip(p, -1e5, 1e5), dh[rows], act)
        assert (np.abs(host_bf16(H) - want) <= (U + 2 * V) * np.abs(want) + 1e-30).all()
        dX, dW = torch.empty(m, K, dtype=BF, device=DEV), torch.empty(2 * F, K, dtype=BF, device=DEV)
        B.chorus_gated_ffn_backward(X, dev_bf16(w), pre, DH, ACT[act], dX, None)
        dx = host_bf16(dX)
        inside = np.abs(x[rows][:, 0]) < 2.0 ** 24
        assert np.isfinite(dx[inside]).all() and np.isnan(dx[~inside]).all()
        slope = d[:, :F].sum(1)  # w of the gate is 1 in the first column
        assert (np.abs(dx[:, 0] - slope) <= 3 * U * np.abs(slope) + F * 2 * 1e-6)[inside].all()
        assert np.array_equal(np.isnan(_kept(pre)[:, :F]), np.repeat(~inside[:, None], F, 1))


def test_results_do_not_depend_on_the_call():
    """The same call twice, and in a captured graph replayed with eager calls between: equal bits. Two workspaces at once."""
    M, F, K = 200, 320, 256
    x, w, dh = (dev_bf16(t) for t in _inputs(M, F, K))

    def step(H, pre, dX, dW, ws):
        B.chorus_gated_ffn(x, w, B.ACT_GELU, H, pre=pre)
        B.chorus_gated_ffn_backward(x, w, pre, dh, B.ACT_GELU, dX, dW, ws=ws)

    def buffers():
        n = B.chorus_gated_ffn_backward_workspace_bytes(M, F, K)
        return (torch.zeros(M, F, dtype=BF, device=DEV), torch.zeros(M, 2 * F, dtype=BF, device=DEV), torch.zeros(M, K, dtype=BF, device=DEV),
                torch.zeros(2 * F, K, dtype=BF, device=DEV), torch.empty(n, dtype=torch.uint8, device=DEV))

    want, other, captured = buffers(), buffers(), buffers()
    step(*want)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(*captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(*captured)
    for _ in range(3):
        for t in captured[:4]:
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        step(*other)
        torch.cuda.synchronize()
        for a, b, c in zip(want[:4], other[:4], captured[:4]):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(a.view(torch.int16), c.view(torch.int16))
