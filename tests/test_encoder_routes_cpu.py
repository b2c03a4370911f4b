"""Which kernels the gated half of a feed-forward block and the products of 8-bit integers take, from the host's plan: every one of them has sizes in the
GPU tests, and those sizes keep taking it."""
import ctypes as C

import pytest

import paper_2604_04451_amd as P
from paper_2604_04451_amd import binding as B

P.load()
FEW, T64, T128X256, T256, T128, DEEP, T256X192 = range(7)

# (M, F, K): (rows of the first launch on 256 x 256 tiles, kernel of the others)
GATED = [((3, 640, 128), (0, FEW)), ((33, 192, 320), (0, T64)), ((132, 8256, 128), (0, T128)), ((77, 13376, 64), (0, DEEP)), ((385, 5184, 1024), (0, T128X256)),
         ((139, 9152, 1024), (0, T128X256)), ((1300, 3136, 512), (0, T256X192)), ((65, 6848, 64), (0, T256X192)), ((1300, 4160, 512), (0, T256)),
         ((263, 12608, 448), (0, T256)), ((4200, 2112, 512), (3840, T64)), ((824, 9408, 384), (768, T64)), ((609, 13184, 576), (512, DEEP))]

# (M, N, K, epilogue): the same
I8 = [((5, 1000, 1024, B.EPI_RESID), (0, FEW)), ((33, 8, 512, B.EPI_BF16), (0, T64)), ((77, 1544, 640, B.EPI_RESID), (0, T64)),
      ((18224, 136, 256, B.EPI_GELU_BF16), (0, T128)), ((16147, 72, 128, B.EPI_RESID), (0, T128)), ((14967, 72, 128, B.EPI_F32), (0, T128)),
      ((15063, 72, 256, B.EPI_GELU_BF16), (0, DEEP)), ((16322, 80, 256, B.EPI_RESID), (0, DEEP)), ((15949, 72, 256, B.EPI_F32), (0, DEEP)),
      ((12196, 424, 1920, B.EPI_BF16), (0, T128X256)), ((17840, 136, 2176, B.EPI_GELU_BF16), (0, T128X256)), ((10627, 656, 3456, B.EPI_RESID), (0, T128X256)),
      ((13086, 392, 4736, B.EPI_F32), (0, T128X256)),
      ((16746, 392, 256, B.EPI_BF16), (0, T256)), ((13103, 520, 1024, B.EPI_GELU_BF16), (0, T256)), ((8201, 1544, 256, B.EPI_RESID), (0, T256)),
      ((13149, 520, 128, B.EPI_F32), (0, T256)),
      ((1448, 13144, 640, B.EPI_BF16), (1024, T128)), ((2321, 6952, 768, B.EPI_GELU_BF16), (2304, T64)), ((2064, 8296, 1152, B.EPI_GELU_BF16), (1792, DEEP)),
      ((8200, 2312, 512, B.EPI_F32), (6400, T128)), ((8200, 2312, 512, B.EPI_RESID), (6400, T128)), ((2050, 8968, 512, B.EPI_F32), (1792, DEEP)),
      ((2050, 8968, 512, B.EPI_RESID), (1792, DEEP)), ((16639, 912, 512, B.EPI_RESID), (16384, T64))]


@pytest.mark.parametrize("size,want", GATED)
def test_gated(size, want):
    assert B.chorus_gated_ffn_plan(*size) == want


@pytest.mark.parametrize("size,want", I8)
def test_gemm_i8(size, want):
    assert B.chorus_gemm_i8_plan(*size) == want


@pytest.mark.parametrize("size,want", [((512, 10240, 4096), (0, T256X192)), ((4096, 10240, 4096), (0, T256)), ((1, 10240, 4096), (0, FEW))])
def test_gated_of_an_encoder(size, want):
    assert B.chorus_gated_ffn_plan(*size) == want


@pytest.mark.parametrize("size,want", [((13103, 1536, 8960, B.EPI_F32), (10752, None)), ((32760, 8960, 1536, B.EPI_GELU_BF16), (None, T256))])
def test_gemm_i8_of_a_block(size, want):
    got = B.chorus_gemm_i8_plan(*size)
    assert all(w is None or g == w for g, w in zip(got, want))


def test_every_kernel_has_a_size():
    assert {w[1] for _, w in GATED} == {FEW, T64, T128X256, T256, T128, DEEP, T256X192} and any(w[0] for _, w in GATED)
    assert {(s[3], w[1]) for s, w in I8} >= {(e, t) for e in (B.EPI_GELU_BF16, B.EPI_RESID) for t in (T64, T128, T256, T128X256, DEEP)}
    assert {(s[3], bool(w[0])) for s, w in I8} >= {(e, True) for e in range(4)}


def test_refusals():
    lib, out = P.load(), B.GemmPlan()
    to = C.byref(out)
    for call, want in ((lambda: lib.chorus_gated_ffn_plan(4, 128, 64, None), B.E_ARG), (lambda: lib.chorus_gated_ffn_plan(0, 128, 64, to), B.E_ARG),
                       (lambda: lib.chorus_gated_ffn_plan(4, 96, 64, to), B.E_SHAPE), (lambda: lib.chorus_gemm_i8_plan(4, 64, 128, 0, None), B.E_ARG),
                       (lambda: lib.chorus_gemm_i8_plan(0, 64, 128, 0, to), B.E_ARG), (lambda: lib.chorus_gemm_i8_plan(4, 64, 128, 4, to), B.E_ARG),
                       (lambda: lib.chorus_gemm_i8_plan(4, 64, 64, 0, to), B.E_SHAPE), (lambda: lib.chorus_gemm_i8_plan(4, 60, 128, 0, to), B.E_SHAPE),
                       (lambda: lib.chorus_gemm_i8_plan(4, 64, 131072, 0, to), B.E_SHAPE)):
        assert call() == want
