"""Which form of the linear cross entropy a call takes, and that the forms on both sides
of each rule give the values of the definition."""
import pytest
import torch

from paper_2009_03816_b200 import training

import gpu_util
from test_gpu_xent import _run

pytestmark = pytest.mark.gpu


def _launches(T, D, V, shift=0):
    """Kernels of (the loss, the gradients)."""
    gpu_util.ensure_library()
    flat = torch.zeros(V * D + 8, device="cuda", dtype=torch.bfloat16)
    w = flat[shift:shift + V * D].view(V, D)
    h, y = torch.zeros(T, D, device="cuda", dtype=torch.bfloat16), torch.zeros(T, device="cuda", dtype=torch.int64)
    op = training.LinearXent(T, D, V)
    _, rows, lse = op.forward(h, w, y)
    first = op.launches
    op.backward(h, w, y, lse, torch.ones((), device="cuda"), rows=rows)
    second = op.launches - first
    op.close()
    return first, second


# gradients of few tokens in their own form: two launches; on the tensor cores: six, more where w is packed
@pytest.mark.parametrize("T,D,V,own", [(1, 4096, 32_768, True), (2, 4096, 32_768, True), (4, 4096, 16_384, True), (4, 4096, 32_768, False),
                                       (3, 1000, 32_003, True), (3, 1536, 32_768, False), (4, 512, 131_072, True),
                                       (1, 1100, 16_384, True), (2, 1100, 8000, True), (2, 1100, 65_536, False)])
def test_gradients_of_few_tokens_take_the_form_that_was_faster(T, D, V, own):
    assert (_launches(T, D, V)[1] == 2) == own


def test_gradients_of_few_tokens_by_alignment():
    assert _launches(3, 1000, 32_003)[1] == 2 and _launches(3, 1000, 32_003, 1)[1] > 2


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,V", [(4, 128, 30_000), (4, 128, 29_000), (3, 1536, 9000), (2, 61, 4000), (4, 1100, 9000)])
def test_values_of_few_tokens_on_both_sides(T, D, V, dtype):
    _run(T, D, V, dtype, seed=81)
    _run(T, D, V, dtype, seed=82, masked=0.4, reduction="sum")


# few classes: one launch for the loss and two for the gradients, where those are faster
@pytest.mark.parametrize("T,D,V,loss,grads", [(256, 84, 10, True, True), (1024, 84, 10, True, True), (4096, 84, 10, True, False),
                                              (9000, 84, 10, False, False), (1024, 512, 10, True, False), (4096, 512, 10, False, False),
                                              (256, 512, 64, False, False), (2048, 84, 64, True, False), (4096, 84, 64, False, False)])
def test_few_classes_take_the_form_that_was_faster(T, D, V, loss, grads):
    got = _launches(T, D, V)
    assert (got[0] == 1) == loss and (got[1] == 2) == grads, got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,V", [(1024, 84, 10), (1025, 84, 10), (8192, 84, 10), (8193, 84, 10), (700, 512, 10), (256, 193, 64), (256, 192, 64),
                                   (300, 12_000, 1), (6, 4000, 3), (2049, 512, 10)])
def test_values_of_few_classes_on_both_sides(T, D, V, dtype):
    _run(T, D, V, dtype, seed=83)
    _run(T, D, V, dtype, seed=84, masked=0.4, reduction="sum")


# the loss of few tokens in its own form: one launch
@pytest.mark.parametrize("T,D,V,own", [(1, 4096, 32_768, True), (4, 64, 32_768, True), (4, 64, 65_536, False), (1, 320, 40_000, False),
                                       (4, 512, 131_072, True)])
def test_the_loss_of_few_tokens_takes_the_form_that_was_faster(T, D, V, own):
    assert (_launches(T, D, V)[0] == 1) == own


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,V", [(1, 61, 32_768), (4, 61, 32_769), (2, 320, 33_000), (3, 321, 33_000)])
def test_values_of_the_loss_of_few_tokens_on_both_sides(T, D, V, dtype):
    _run(T, D, V, dtype, seed=85)
    _run(T, D, V, dtype, seed=86, masked=0.4, reduction="sum")
