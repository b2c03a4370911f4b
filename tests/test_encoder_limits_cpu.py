"""Limits of the 8-bit products and of attention with a bias by distance, refused before any device work: sums of -128 by -128 that pass 32 bits, counts that
pass a grid, and outputs whose sequences would lie on top of one another."""
import pytest

import paper_2604_04451_amd as P
from paper_2604_04451_amd import binding as B
from test_encoder_cpu import P16, _attend, _attend_back, _bias, _i8


@pytest.mark.parametrize("change,want", [(dict(K=131072), B.E_SHAPE), (dict(K=131072 - 128, M=0), B.OK), (dict(N=(1 << 24) + 8), B.E_SHAPE),
                                         (dict(N=(1 << 31) - 8), B.E_SHAPE), (dict(N=1 << 24, M=0), B.OK)])
def test_gemm_i8(change, want):
    assert _i8(P.load(), **change) == want


@pytest.mark.parametrize("change,want", [(dict(n_buckets=(1 << 16) + 1), B.E_SHAPE), (dict(n_buckets=(1 << 31) - 1), B.E_SHAPE), (dict(o_batch=0), B.E_SHAPE)])
def test_attention_bias(change, want):
    assert _attend(P.load(), _bias(**change)) == want
    assert _attend_back(P.load(), _bias(**change), ws=P16) == want


@pytest.mark.parametrize("name", ["dq_batch", "dk_batch", "dv_batch"])
def test_gradients_on_top_of_one_another(name):
    assert _attend_back(P.load(), _bias(), steps={name: 0}) == B.E_SHAPE


@pytest.mark.parametrize("change", [dict(q_batch=0), dict(k_batch=0, v_batch=0)])
def test_one_input_for_all_sequences(change):
    assert _attend(P.load(), _bias(Lq=0, **change)) == B.OK
