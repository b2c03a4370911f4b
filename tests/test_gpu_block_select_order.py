"""Scores of the choice of key blocks beyond what fp64 sums hold: terms that are more than 2^30 apart, where the order of the additions
decides. They have one order wherever a row's scores are made again in fp64, be it for a few blocks or for all: eight consecutive values one
after the other, then sums dh / 16, dh / 32, ..., 1 places apart. The choice is exact by that."""
import numpy as np
import pytest
import torch

from paper_2604_04451_amd import binding as B
from gpu_util import DEV, dev_bf16
import synth

pytestmark = pytest.mark.gpu


def scores(Qm, Km):
    """[nq, dh] x [nk, dh] -> [nq, nk]; products of bf16 are exact, so a fused multiply-add is an addition."""
    p = Qm.astype(np.float64)[:, None] * Km.astype(np.float64)[None]
    p = p.reshape(*p.shape[:2], -1, 8)
    s = np.zeros(p.shape[:3])
    for e in range(8):
        s = s + p[..., e]
    while s.shape[2] > 1:
        n = s.shape[2] // 2
        s = s[..., :n] + s[..., n:]
    return s[..., 0]


def choose(s, keep, rule):
    out = np.full((s.shape[0], keep), -1, np.int32)
    may = np.flatnonzero(rule != 2)
    for a in range(s.shape[0]):
        best = np.sort(may[np.lexsort((may, -s[a, may], rule[may] != 1))][:keep])
        out[a, :best.size] = best
    return out


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("nk,keep", [(20, 6), (32, 11), (33, 7), (400, 60), (1000, 301), (2000, 90), (3000, 500)])
def test_one_order_of_sums(dh, nk, keep):
    print(f"[case] block_select order of sums dh={dh} nk={nk} keep={keep}", flush=True)
    rng = np.random.default_rng(dh + nk)
    nq = 9
    Qm = synth.round_bf16(rng.choice([-1.0, 1.0, 0.5], (nq, dh)).astype(np.float32))
    Km = rng.integers(-3, 4, (nk, dh)).astype(np.float64)
    for b in range(nk):  # large terms that cancel, or nearly, with some of the others lost or kept by where they stand
        at = rng.permutation(dh)[:6]
        Km[b, at] = 2.0 ** rng.choice([52, 53, 54, 55], 6) * rng.choice([-1.0, 1.0], 6)
    Km = synth.round_bf16(Km.astype(np.float32))
    rule = np.zeros(nk, np.uint8)
    few = rule.copy()
    few[rng.permutation(nk)[20:]] = 2  # twenty blocks are left
    s = scores(Qm, Km)
    for r, k in ((rule, keep), (few, min(keep, 7))):
        out = torch.empty(1, nq, k, dtype=torch.int32, device=DEV)
        B.chorus_block_select(dev_bf16(Qm[None]), dev_bf16(Km[None]), out, torch.from_numpy(r).to(DEV))
        np.testing.assert_array_equal(out.cpu().numpy()[0], choose(s, k, r))


def test_blocks_alike_but_for_places():
    """The same products in the same order of sums, equal scores: by index, in rows with a few such blocks and with many."""
    print("[case] block_select alike", flush=True)
    rng = np.random.default_rng(4)
    dh, nk = 128, 300
    Qm = np.ones((2, dh), np.float32)
    row = np.zeros(dh, np.float32)
    row[[0, 1, 2, 9, 64]] = 2.0 ** 40, 1.0, -2.0 ** 40, 2.0 ** -14, 1.0
    Km = np.stack([row if b % 3 else row[::-1] for b in range(nk)])
    Km[5, 70] += 2.0 ** -20
    s = scores(Qm, Km)
    few = np.where(np.arange(nk) % 10 == 5, 0, 2).astype(np.uint8)
    for r, k in ((np.zeros(nk, np.uint8), 40), (few, 12)):
        out = torch.empty(1, 2, k, dtype=torch.int32, device=DEV)
        B.chorus_block_select(dev_bf16(Qm[None]), dev_bf16(Km[None]), out, torch.from_numpy(r).to(DEV))
        np.testing.assert_array_equal(out.cpu().numpy()[0], choose(s, k, r))
