"""The gated half of a feed-forward block on each of its tiles, with rows and columns that do not fill them, with and without the projections kept; and a
backward pass behind the large ones. Bounds and references of test_gpu_gated.py; which tile a size takes is held by test_encoder_routes_cpu.py."""
import pytest

import test_gpu_gated as G
from test_encoder_routes_cpu import GATED

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("save", [False, True])
@pytest.mark.parametrize("M,F,K", [size for size, _ in GATED])
def test_forward(M, F, K, act, save):
    G.test_forward(M, F, K, act, save)


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("M,F,K", [(1300, 1088, 512), (385, 2624, 1024)])
def test_backward(M, F, K, act):
    G.test_backward(M, F, K, act)
