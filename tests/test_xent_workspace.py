"""Workspace of the linear cross entropy, and its pieces of the vocabulary."""
import pytest
import torch

from paper_2009_03816_b200 import binding
from paper_2009_03816_b200 import build as _build

MB = 1 << 20


@pytest.fixture(scope="module")
def bytes_of():
    _build.build_library()
    return lambda T, D, V, flags: binding.psops_xent_workspace_bytes(
        binding.psops_xent_config(T, D, V, binding.PSOPS_BF16, flags))


@pytest.mark.parametrize("T,D,V", [(1, 4097, 131_072), (1, 4096, 131_072), (300, 9000, 262_144), (4, 2001, 1 << 20)])
def test_rows_that_pass_through_the_workspace_are_no_second_copy_of_w(bytes_of, T, D, V):
    plain = bytes_of(T, (D + 7) // 8 * 8, V, binding.PSOPS_XENT_GRADS)
    staged = bytes_of(T, D, V, binding.PSOPS_XENT_GRADS | binding.PSOPS_XENT_STAGED)
    assert 2 * V * D > 600 * MB                     # more than a piece
    assert plain < staged <= plain + 2 * 512 * MB + MB


@pytest.mark.gpu
@pytest.mark.parametrize("T,D,V", [(3, 4097, 70_001), (200, 4097, 70_001)])
def test_several_pieces_of_rows_that_pass_through_the_workspace(T, D, V):
    from test_gpu_xent import _run
    _run(T, D, V, torch.bfloat16, seed=91, masked=0.2)
