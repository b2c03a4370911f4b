"""Products of 8-bit integers on each of their tiles, whole and with the last rows in a launch of their own, with rows and columns that do not fill the tiles. Bounds
and references of test_gpu_gemm_i8.py; which tiles a size takes is held by test_encoder_routes_cpu.py."""
import numpy as np
import pytest

from test_encoder_routes_cpu import I8
from test_gpu_gemm_i8 import _check, _product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,epilogue", [size for size, _ in I8])
def test_product(M, N, K, epilogue):
    rng = np.random.default_rng(M + N + K)
    a, w, sa, sw, bias = _product(rng, M, N, K)
    _check(a, w, sa, sw, bias, epilogue, gates=True)
