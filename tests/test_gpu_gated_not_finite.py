"""The gated half of a feed-forward block with an infinity in its weights or tokens: it is one, or NaN, in its own column or row, as the definition has it, and
changes nothing of the others. K of an odd number of steps among them, whose last one a kernel of few rows has twice in hand."""
import numpy as np
import pytest
import torch

from paper_2604_04451_amd import binding as B
from gpu_util import DEV, dev_bf16, host_bf16
from test_gpu_gated import BF, _inputs

pytestmark = pytest.mark.gpu


def run(x, w, M, F):
    H = torch.empty(M, F, dtype=BF, device=DEV)
    B.chorus_gated_ffn(dev_bf16(x), dev_bf16(w), B.ACT_SILU, H)
    return host_bf16(H)


@pytest.mark.parametrize("M,F,K", [(1, 64, 64), (3, 640, 192), (16, 128, 1088), (30, 1024, 64), (40, 192, 192), (300, 640, 320)])
def test_forward(M, F, K):
    x, w, _ = _inputs(M, F, K)
    x[:, K - 1] = np.where(x[:, K - 1] == 0, 1.0, x[:, K - 1])
    clean = run(x, w, M, F)
    w[F + 5, K - 1] = np.inf  # the other factor of column 5
    got = run(x, w, M, F)
    others = np.delete(np.arange(F), 5)
    assert np.array_equal(got[:, others], clean[:, others])
    gate = x.astype(np.float64) @ w[5].astype(np.float64)
    assert np.array_equal(got[:, 5], np.where(gate * x[:, K - 1] > 0, np.inf, -np.inf))  # silu has the sign of the gate
    w[F + 5, K - 1] = 0.5
    x[M // 2, 3] = np.nan
    rows = np.delete(np.arange(M), M // 2)
    clean[:, 5] = run(np.where(np.isnan(x), 0.0, x).astype(np.float32), w, M, F)[:, 5]
    got = run(x, w, M, F)
    assert np.isnan(got[M // 2]).all() and np.array_equal(got[rows], clean[rows])
