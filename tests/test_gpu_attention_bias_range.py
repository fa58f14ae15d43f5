"""Attention under finite biases of any size."""
import pytest
import torch

from attention_util import inputs, lengths_to_offsets
from paper_2009_03816_b200 import training
from paper_2009_03816_b200 import build as _build

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _library():
    _build.build_library()


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("lowest,out", [(-1e31, True), (-1.0001e30, True), (-1e30, False), (-8e29, False), (-6.95e29, False), (-65504.0, False)])
def test_what_takes_pairs_out(lowest, out, dtype):
    """It is the bias itself that lies below -1e30; other numbers are biases, fp16's lowest among them."""
    op = training.Attention(40, 1, 2, 1, 16, dtype=dtype, buckets=[0, 1], gradients=False)
    x = inputs(40, 2, 1, 16, dtype, grad=False)
    bias = torch.tensor([[lowest, 0.0], [0.0, 0.0]], device="cuda")
    bias = bias.to(F16) if lowest == -65504.0 and dtype is F16 else bias
    o, lse = op.forward(x["q"], x["k"], x["v"], lengths_to_offsets([40]), bias)
    if out:                                              # the first token of head 0 is left with no pair
        assert not o[0, 0].any() and float(lse[0, 0]) == -torch.inf
    else:                                                # or has one
        assert torch.equal(o[0, 0], x["v"][0, 0])
        score = float(x["q"][0, 0].double() @ x["k"][0, 0].double()) / 4.0
        assert abs(float(lse[0, 0]) - (lowest + score)) <= 2.0 ** -22 * abs(lowest)
    assert torch.equal(o[0, 1], x["v"][0, 0]) and torch.isfinite(o).all() and torch.isfinite(lse[:, 1:]).all()
