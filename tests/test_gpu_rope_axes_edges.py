"""Axis rotations at the ends of the number range, on the GPU through the C ABI: what does not turn passes through whatever stands beside it.
Tolerance of values that turn: one rounding of the result, 2^-8 |y|, and 2^-19 of the largest magnitude of the pair for the fp32 sine and products."""
import numpy as np
import pytest
import torch

from oracle import blocks as OB
from paper_2604_04451_amd import binding as B
from gpu_util import DEV, dev_bf16, dev_f32, host_bf16
import synth

pytestmark = pytest.mark.gpu

U = 2.0 ** -8
ODD = np.array([np.inf, -np.inf, np.nan, 3e38, -3e38, -0.0, 0.0, 1e-40, -2.0, 1.5], np.float32)


def _rotate(x, H, dh, pos, freq, axis, halves, scale, pad=3):
    L = x.shape[0]
    out = torch.full((H, L + pad, dh), 3.0, dtype=torch.bfloat16, device=DEV)
    B.chorus_rope_axes(dev_bf16(x), 0, None, B.ROPE_NORM_NONE, out, L, H, dh, dev_f32(pos), torch.from_numpy(freq).to(DEV),
                       torch.from_numpy(axis).to(DEV), B.ROPE_HALVES if halves else B.ROPE_PAIRS, scale)
    return out


@pytest.mark.parametrize("H,dh", [(1, 64), (9, 64), (12, 128), (40, 128), (41, 128)])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("n_pairs", [0, 16, 32])
def test_what_does_not_turn_passes_through(H, dh, halves, n_pairs):
    """Infinities, NaN, zeros of both signs, the largest and subnormal values in pairs of no axis and behind the pairs: the same bits out."""
    print(f"[case] rope_axes passes H={H} dh={dh} halves={halves} n_pairs={n_pairs}", flush=True)
    rng = np.random.default_rng(H + n_pairs)
    L = 7
    pos = rng.uniform(-50, 50, (L, 2)).astype(np.float32)
    freq, axis = rng.uniform(0.01, 1.0, n_pairs), rng.integers(0, 2, n_pairs).astype(np.int32)
    axis[::3] = rng.choice([-1, 2, 2 ** 31 - 1, -2 ** 31], axis[::3].size)
    turns = np.zeros(dh, bool)
    for p in range(n_pairs):
        if 0 <= axis[p] < 2:
            turns[[p, n_pairs + p] if halves else [2 * p, 2 * p + 1]] = True
    x = synth.round_bf16(rng.standard_normal((L, H, dh)).astype(np.float32))
    stays = synth.round_bf16(rng.choice(ODD, (L, H, dh)))
    x = np.where(turns, x, stays)
    got = _rotate(x.reshape(L, H * dh), H, dh, pos, freq, axis, halves, 1.0)
    assert not got[:, L:].view(torch.int16).any()
    want = dev_bf16(x.transpose(1, 0, 2)).view(torch.int16)[:, :, torch.from_numpy(~turns)]
    have = got[:, :L].view(torch.int16)[:, :, torch.from_numpy(~turns)]
    nan = torch.from_numpy(np.isnan(x.transpose(1, 0, 2)[:, :, ~turns])).to(DEV)
    assert torch.equal(have[~nan], want[~nan])
    assert torch.isnan(got[:, :L][:, :, torch.from_numpy(~turns)][nan]).all()
    ref = OB.rope_axes(np.where(turns, x, 0.0).reshape(L, H * dh), None, "none", H, dh, pos, freq, axis, halves)
    off = np.abs(host_bf16(got[:, :L]) - ref)[:, :, turns]
    assert (off <= (U * np.abs(ref) + 2.0 ** -19 * np.abs(x).transpose(1, 0, 2).max(2, keepdims=True, where=turns, initial=0.0))[:, :, turns]).all()


@pytest.mark.parametrize("H,L,pad", [(2, 0, 5), (41, 0, 1)])
def test_no_rows_but_padding(H, L, pad):
    print(f"[case] rope_axes H={H} L=0 with {pad} rows of padding", flush=True)
    out = _rotate(np.zeros((0, H * 64), np.float32), H, 64, np.zeros((0, 2), np.float32), np.ones(32), np.zeros(32, np.int32), False, 1.0, pad)
    assert not out.view(torch.int16).any()


@pytest.mark.parametrize("H,dh", [(3, 64), (12, 128), (41, 128)])
@pytest.mark.parametrize("halves", [False, True])
def test_largest_values_scaled_down(H, dh, halves):
    """Pairs whose turned values fp32 does not hold until they are multiplied by out_scale, which the results hold again."""
    print(f"[case] rope_axes largest H={H} dh={dh} halves={halves}", flush=True)
    rng = np.random.default_rng(dh)
    L = 50
    pos = rng.uniform(-50, 50, (L, 2)).astype(np.float32)
    freq, axis = (t.numpy() for t in B.chorus_rope_axes_table((16, 32), device="cpu"))
    x = synth.round_bf16((rng.choice([-1.0, 1.0], (L, H * dh)) * rng.uniform(1.5, 1.9, (L, H * dh)) * 2.0 ** 127).astype(np.float32))
    got = host_bf16(_rotate(x, H, dh, pos, freq, axis, halves, 0.25))[:, :L]
    ref = OB.rope_axes(x, None, "none", H, dh, pos, freq, axis, halves, 0.25)
    assert np.abs(ref).max() > 2.0 ** 126  # turned values beyond 2^128
    assert (np.abs(got - ref) <= U * np.abs(ref) + 2.0 ** -19 * np.abs(ref).max(2, keepdims=True)).all()
