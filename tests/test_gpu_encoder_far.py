"""Operators of an encoder's layers, and 8-bit products, whose tensors reach beyond 2^31 values: each result has the bits that the same rows have in a small
call, or that the same tensors give when they lie together."""
import pytest
import torch

from paper_2604_04451_amd import binding as B
from gpu_util import DEV

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
BATCH = (1 << 31) + 64  # values from one sequence to the next


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def far(t, row):
    """A copy of t [2, L, heads, dh] in a buffer with `row` values from row to row and BATCH from sequence to sequence."""
    n, L, heads, dh = t.shape
    room = torch.empty(BATCH + row * L, dtype=BF, device=DEV)
    view = room.as_strided(t.shape, (BATCH, row, dh, 1))
    view.copy_(t)
    return view


@pytest.mark.parametrize("Lq,dh", [(1, 64), (40, 64), (40, 128)])
def test_attention_bias(Lq, dh):
    torch.manual_seed(Lq + dh)
    H, Hk, Lk, row = 4, 2, 300, 1 << 20
    q, do = (torch.randn(2, Lq, H, dh, device=DEV).to(BF) for _ in range(2))
    k, v = (torch.randn(2, Lk, Hk, dh, device=DEV).to(BF) for _ in range(2))
    table, bucket = torch.randn(32, H, device=DEV), B.chorus_bias_buckets(32, 128)
    first = torch.tensor([Lk - Lq, 17], dtype=torch.int32, device=DEV)

    def run(move):
        Q, K, V, DO = move(q), move(k), move(v), move(do)
        O, rest, dQ = move(torch.zeros_like(q)), move(torch.zeros_like(q)), move(torch.zeros_like(q))
        served = move(torch.zeros_like(q))
        dK, dV = move(torch.zeros_like(k)), move(torch.zeros_like(k))
        lse, dtable = torch.zeros(2, H, Lq, device=DEV), torch.zeros_like(table)
        how = dict(first=first, causal=True, scale=dh ** -0.5)
        B.chorus_attention_bias(Q, K, V, served, table, bucket, **how)
        B.chorus_attention_bias(Q, K, V, O, table, bucket, lse=lse, rest=rest, **how)
        B.chorus_attention_bias_backward(Q, K, V, O, rest, lse, DO, table, bucket, dQ, dK, dV, dtable, **how)
        return [t.contiguous() for t in (served, O, dQ, dK, dV)] + [lse, dtable]

    for a, b in zip(run(lambda t: far(t, row)), run(lambda t: t.clone())):
        assert torch.equal(a, b) and a.float().abs().sum() > 0


def test_gemm_i8():
    M, N, K = 66000, 33024, 128
    g = torch.Generator(device=DEV).manual_seed(1)
    a = torch.randint(-128, 128, (M, K), dtype=torch.int8, device=DEV, generator=g)
    w = torch.randint(-128, 128, (N, K), dtype=torch.int8, device=DEV, generator=g)
    sa, sw = torch.rand(M, device=DEV, generator=g), torch.rand(N, device=DEV, generator=g)
    out = B.chorus_gemm_i8(a, sa, w, sw, B.EPI_BF16, torch.empty(M, N, dtype=BF, device=DEV))
    assert M * N > 1 << 31
    few = torch.empty(256, N, dtype=BF, device=DEV)
    for at in (0, M // 2 // 4 * 4, M - 256):
        B.chorus_gemm_i8(a[at:at + 256].contiguous(), sa[at:at + 256].clone(), w, sw, B.EPI_BF16, few)
        assert torch.equal(out[at:at + 256], few)


def test_gated():
    """H and what is kept of the projections pass 2^31 values; the gradients of the tokens, which no other token's come into."""
    M, F, K = 66048, 33024, 64
    x, w = torch.randn(M, K, device=DEV).to(BF), (torch.randn(2 * F, K, device=DEV) / 8).to(BF)
    h, pre = torch.empty(M, F, dtype=BF, device=DEV), torch.empty(M, 2 * F, dtype=BF, device=DEV)
    B.chorus_gated_ffn(x, w, B.ACT_SILU, h, pre=pre)
    dh = torch.full((M, F), 0.5, dtype=BF, device=DEV)
    dx, _ = B.chorus_gated_ffn_backward(x, w, pre, dh, B.ACT_SILU, torch.empty_like(x), None)
    assert M * F > 1 << 31
    for at in (0, M // 2, M - 256):
        rows = slice(at, at + 256)
        few, kept = torch.empty(256, F, dtype=BF, device=DEV), torch.empty(256, 2 * F, dtype=BF, device=DEV)
        B.chorus_gated_ffn(x[rows].contiguous(), w, B.ACT_SILU, few, pre=kept)
        assert torch.equal(h[rows], few) and torch.equal(pre[rows].view(torch.int16), kept.view(torch.int16))
        want, _ = B.chorus_gated_ffn_backward(x[rows].contiguous(), w, kept, dh[rows], B.ACT_SILU, torch.empty(256, K, dtype=BF, device=DEV), None)
        assert (dx[rows].float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()  # sums over 66048 in the order of another tile
