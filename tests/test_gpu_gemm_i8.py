"""Quantisation of rows and products of 8-bit integers on the GPU through the C ABI, against plain fp64 forms. Codes and scales are
exact (one fp32 division a scale); sums of codes are whole numbers. Behind them: the sum's way to fp32, two scales and the bias, 2^-24
each of what they round, so 2^-22 (|product| + |bias|); bf16 results half a step, 2^-8 |y|; the GELU's exponential and reciprocal
2^-17 |y| (an exponent of up to 30 rounded to 24 bits), its slope at most 1.13."""
import numpy as np
import pytest
import torch

from oracle import encoder as OE
import paper_2604_04451_amd as P
from paper_2604_04451_amd import binding as B
from gpu_util import DEV, dev_bf16, dev_f32, host
import synth

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _bf(a):
    return synth.round_bf16(np.ascontiguousarray(a, dtype=np.float32))


def _quant(x, ld=None, Kp=None):
    M, K = x.shape
    rows = np.full((M, ld or K), 7.0, np.float32)
    rows[:, :K] = x
    X = dev_bf16(rows)[:, :K]
    codes = torch.full((M, Kp or -(-K // 128) * 128), 99, dtype=torch.int8, device=DEV)
    scale = torch.full((M,), 5.0, device=DEV)
    return B.chorus_quant_rows_i8(X, codes, scale)


@pytest.mark.parametrize("M,K,ld,Kp", [(1, 8, None, None), (1, 5120, None, None), (3, 1000, 1016, 1024), (77, 64, 72, 64), (2050, 4096, None, None),
                                       (2049, 1544, 1600, 1664), (5, 12296, None, None), (2, 20000, 20008, 20096), (2048, 4104, None, None)])
def test_quant_rows(M, K, ld, Kp):
    rng = np.random.default_rng(M * 7 + K)
    x = _bf(rng.standard_normal((M, K)) * np.exp(rng.uniform(-3, 3, (M, 1))))
    codes, scale = _quant(x, ld, Kp)
    want, unit = OE.quant_rows_i8(x)
    got = host(codes)
    assert np.array_equal(got[:, :K], want)
    assert not got[:, K:].any()
    assert np.array_equal(host(scale), np.abs(x).max(1) / np.float32(127))
    assert np.allclose(host(scale), unit, rtol=2.0 ** -23, atol=0)


def test_quant_halves_go_to_even():
    """Quotients that are exactly a half: max 127 and values of n + 1/2, and rows where the quotient's factor rounds."""
    halves = np.arange(-126.5, 127.0, 1.0)
    rows = [np.concatenate(([127.0], halves, [0.0] * (256 - 1 - len(halves))))]
    for top in (254.0, 127.0 / 4, 127.0 * 2.0 ** -40, 127.0 * 2.0 ** 60):
        rows.append(rows[0] * (top / 127.0))
    # 3 x 127 / 2 over 2 max: quotients n + 1/2 with a largest value that 127 does not divide
    odd = np.zeros(256)
    odd[0] = 129.0
    odd[1:65] = 129.0 * np.arange(1, 128, 2) / 254.0  # rounded to bf16 below: near halves, on both sides
    rows.append(odd)
    x = _bf(np.stack(rows))
    codes, _ = _quant(x)
    assert np.array_equal(host(codes), OE.quant_rows_i8(x)[0])


def test_quant_every_pair_of_a_value_and_a_largest_one():
    """All mantissas of the largest value against all values of the eight binades below it."""
    tops = 1.0 + np.arange(128) / 128.0
    values = np.concatenate([(1.0 + np.arange(128) / 128.0) * 2.0 ** -e for e in range(9)])
    x = np.zeros((128, 1160))
    for i, t in enumerate(tops):
        v = values[values <= t]
        x[i, :len(v)] = v * np.where(np.arange(len(v)) % 2, -1, 1)
        x[i, -1] = t
    x = _bf(x)
    codes, _ = _quant(x)
    assert np.array_equal(host(codes)[:, :1160], OE.quant_rows_i8(x)[0])


def test_quant_ends_of_the_range():
    rng = np.random.default_rng(3)
    n = rng.standard_normal((9, 128))
    x = _bf(n * np.array([1e38, 3e36, 1e-30, 1e-37, 1e-39, 1.0, 1.0, 1.0, 1.0])[:, None])
    x[5] = 0.0
    x[6, 3] = np.inf
    x[7, 100] = np.nan
    x[8, 0] = -np.inf
    codes, scale = _quant(x)
    want, _ = OE.quant_rows_i8(x)
    assert np.array_equal(host(codes), want)
    s = host(scale)
    assert s[5] == 0 and np.isnan(s[6:]).all() and np.array_equal(s[:5], np.abs(x[:5]).max(1) / np.float32(127))


def _product(rng, M, N, K):
    a = rng.integers(-127, 128, (M, K)).astype(np.int8)
    w = rng.integers(-127, 128, (N, K)).astype(np.int8)
    a[:, 0] = np.where(rng.random(M) < 0.1, -128, a[:, 0])
    return a, w, (rng.random(M) * 0.02).astype(np.float32), (rng.random(N) * 1e-3).astype(np.float32), rng.standard_normal(N).astype(np.float32)


def _check(a, w, sa, sw, bias, epilogue, gates=False):
    M, N = a.shape[0], w.shape[0]
    prod = (a.astype(np.float64) @ w.astype(np.float64).T) * sa[:, None].astype(np.float64) * sw.astype(np.float64)
    b = 0.0 if bias is None else bias.astype(np.float64)
    y = prod + b
    tol = 2.0 ** -22 * (np.abs(prod) + np.abs(b))
    rng = np.random.default_rng(5)
    kw = {}
    if epilogue == B.EPI_RESID:
        g0, g1 = (rng.standard_normal(N).astype(np.float32) for _ in range(2))
        r = rng.standard_normal((M, N)).astype(np.float32)
        out = dev_f32(r)
        gate = 1.0
        if gates:
            kw = dict(gate0=dev_f32(g0), gate1=dev_f32(g1))
            gate = g0.astype(np.float64) + g1
        y, tol = r + 0.5 * gate * y, np.abs(0.5 * gate) * tol + 2.0 ** -22 * (np.abs(r) + (np.abs(g0) + np.abs(g1) + 1.0) * np.abs(y))
    else:
        out = torch.full((M, N), float("nan"), dtype=torch.float32 if epilogue == B.EPI_F32 else BF, device=DEV)
        if epilogue == B.EPI_GELU_BF16:
            y, tol = OE.gelu(y), 1.13 * tol + 2.0 ** -17 * np.abs(OE.gelu(y)) + 1e-30
        if epilogue != B.EPI_F32:
            tol = tol * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(y)
    put = lambda t: torch.from_numpy(t).to(DEV)  # noqa: E731
    B.chorus_gemm_i8(put(a), put(sa), put(w), put(sw), epilogue, out, bias=None if bias is None else put(bias), scale=0.5, **kw)
    got = host(out.float()).astype(np.float64)
    assert (np.abs(got - y) <= tol).all(), float((np.abs(got - y) - tol).max())


@pytest.mark.parametrize("epilogue", [B.EPI_BF16, B.EPI_GELU_BF16, B.EPI_F32, B.EPI_RESID])
@pytest.mark.parametrize("M,N,K", [(1, 8, 128), (1, 1000, 5120), (2, 24, 256), (16, 512, 1024), (15, 4096, 128), (17, 136, 384), (33, 40, 8960),
                                   (64, 64, 128), (77, 1536, 1536), (300, 264, 640), (512, 1536, 4096), (1000, 4608, 256), (1300, 2304, 512)])
def test_product(M, N, K, epilogue):
    rng = np.random.default_rng(M + N + K)
    a, w, sa, sw, bias = _product(rng, M, N, K)
    _check(a, w, sa, sw, bias if M % 2 else None, epilogue, gates=M % 3 == 0)


@pytest.mark.parametrize("M,N", [(2100, 8960), (8200, 1536), (4000, 5120)])
def test_large_tiles_and_cut_rows(M, N):
    rng = np.random.default_rng(M)
    a, w, sa, sw, bias = _product(rng, M, N, 256)
    for epilogue in (B.EPI_GELU_BF16, B.EPI_F32):
        _check(a, w, sa, sw, bias, epilogue)


def test_largest_sums():
    """All codes -128 and 127 over the longest rows that the call takes: 128 * 128 * 131072 would be 2^31."""
    K = 131072 - 128
    for x, y in ((127, 127), (-127, 127), (-128, 127), (-128, -128)):
        for M in (3, 70):
            a, w = np.full((M, K), x, np.int8), np.full((16, K), y, np.int8)
            _check(a, w, np.full(M, 1e-4, np.float32), np.full(16, 1e-4, np.float32), None, B.EPI_F32)


def test_rows_that_are_not_finite_stay_rows():
    rng = np.random.default_rng(9)
    for M in (5, 40):
        x = _bf(rng.standard_normal((M, 128)))
        x[1, 5], x[3, 7] = np.inf, np.nan
        codes, scale = _quant(x)
        _, w, _, sw, _ = _product(rng, 1, 64, 128)
        out = torch.empty(M, 64, device=DEV)
        B.chorus_gemm_i8(codes, scale, torch.from_numpy(w).to(DEV), torch.from_numpy(sw).to(DEV), B.EPI_F32, out)
        bad = np.isnan(host(out))
        assert bad[[1, 3]].all() and not np.delete(bad, [1, 3], 0).any()


@pytest.mark.parametrize("M", [1, 200])
def test_captured_with_its_quantisation(M):
    """Replayed on new inputs, with eager work between the replays."""
    rng = np.random.default_rng(M)
    K, N = 512, 256
    _, w, _, sw, bias = _product(rng, 1, N, K)
    W, SW, bias = (torch.from_numpy(t).to(DEV) for t in (w, sw, bias))
    X = torch.zeros(M, K, dtype=BF, device=DEV)
    codes, scale = torch.empty(M, K, dtype=torch.int8, device=DEV), torch.empty(M, device=DEV)
    out = torch.empty(M, N, dtype=BF, device=DEV)

    def both(x, c, s, o):
        B.chorus_quant_rows_i8(x, c, s)
        return B.chorus_gemm_i8(c, s, W, SW, B.EPI_GELU_BF16, o, bias=bias)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        both(X, codes, scale, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        both(X, codes, scale, out)
    for i in range(3):
        x = dev_bf16(_bf(rng.standard_normal((M, K))))
        X.copy_(x)
        graph.replay()
        want = both(x, torch.empty_like(codes), torch.empty_like(scale), torch.empty_like(out))
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
