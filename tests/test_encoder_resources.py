"""Scratch memory in the kernels of the 8-bit products, the gated feed-forward block and attention with a bias, from the compiler's report (no GPU): none, but
for those whose loops use all registers of their share and that keep a few values of their ends there (up to 20 bytes a lane)."""
import pytest

from test_kernel_resources import _scratch


@pytest.mark.parametrize("source,count,full,most", [
    ("gemm_i8.hip", 28, (), 0), ("gated.hip", 26, ("gated_kernelILi0ELb1ELi8ELi8", "gated_kernelILi1ELb1ELi8ELi8"), 12),
    ("bias_attention.hip", 10, ("bias_few_kernelILi128E", "bias_attention_kernelILi64ELb1E"), 16),
    ("bias_attention_backward.hip", 7, ("bias_dkv_kernelILi64E",), 20),
])
def test_scratch(source, count, full, most, tmp_path):
    got = _scratch(source, tmp_path)
    kernels = {n: v for n, v in got.items() if "_kernel" in n}
    assert len(kernels) >= count, sorted(got)
    limit = {n: most if any(f in n for f in full) else 0 for n in kernels}
    assert not {n: v for n, v in kernels.items() if v > limit[n]}
