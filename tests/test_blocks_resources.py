"""Scratch memory in the kernels of attention over selected blocks and what feeds it, from the compiler's report (no GPU): none, but for the
choice with 20 scores a lane, where up to nine values of a lane wait there while the scores are made."""
import pytest

from test_kernel_resources import _scratch


@pytest.mark.parametrize("source,count", [("block_attention.hip", 8), ("block_select.hip", 16), ("rope_axes.hip", 48)])
def test_scratch(source, count, tmp_path):
    got = _scratch(source, tmp_path)
    kernels = {n: v for n, v in got.items() if "_kernel" in n}
    assert len(kernels) >= count, sorted(got)
    twenty = {n for n in kernels if "block_select_kernel" in n and "ELi20E" in n}
    assert not {n: v for n, v in kernels.items() if v and n not in twenty}
    assert all(kernels[n] <= 48 for n in twenty)
