"""Keep8.hooks() around the other operators, and what it holds on the GPU."""
import pytest
import torch

from attention_util import inputs, lengths_to_offsets
from paper_2009_03816_b200 import training
from paper_2009_03816_b200 import build as _build

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def keep():
    _build.build_library()
    return training.Keep8()


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("outlier", [1.0, 60.0, 300.0])
def test_attention_keeps_what_its_statistics_belong_to(keep, outlier, dtype):
    """Its backward pass takes lse for that of the scores: with q and k rounded to 8 bits probabilities would not sum to 1,
    and in fp16, beside a channel of large numbers, pass its range.  Gradients are those without the hooks, bit for bit."""
    T = 700
    x = inputs(T, 4, 2, 128, dtype, 3, buckets=[0, 1, 20])
    x["q"][:, :, 5] *= outlier
    op = training.Attention(T, 2, 4, 2, 128, dtype=dtype, buckets=[0, 1, 20])
    offsets = lengths_to_offsets([500, 200])
    leaves = [[x[n].clone().requires_grad_() for n in ("q", "k", "v", "bias")] for _ in range(2)]
    op(*leaves[0][:3], offsets, leaves[0][3]).backward(x["grad"])
    before = keep.launches
    with keep.hooks():
        q, k, v, bias = leaves[1]
        out = op(q * 1, k * 1, v * 1, offsets, bias)
        assert keep.launches == before
        h = torch.tanh(out)                                          # others are kept in 8 bits as before
        assert keep.launches == before + 1
    out.backward(x["grad"])
    for a, b in zip(*leaves):
        assert torch.equal(a.grad, b.grad) and torch.isfinite(a.grad).all()


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_linear_cross_entropy_keeps_what_its_statistics_belong_to(keep, dtype):
    gen = torch.Generator(device="cuda").manual_seed(4)
    h = torch.empty(300, 256, device="cuda").normal_(generator=gen)
    h[:, 7] *= 40.0
    h, w = h.to(dtype), (torch.empty(1000, 256, device="cuda").normal_(generator=gen) / 8).to(dtype)
    y = torch.randint(0, 1000, (300,), device="cuda", generator=gen)
    xent = training.LinearXent(300, 256, 1000, dtype=dtype)
    leaves = [[h.clone().requires_grad_(), w.clone().requires_grad_()] for _ in range(2)]
    xent(*leaves[0], y).backward()
    with keep.hooks():
        loss = xent(leaves[1][0] * 1, leaves[1][1], y)
    loss.backward()
    for a, b in zip(*leaves):
        assert torch.equal(a.grad, b.grad)


def test_a_weight_stepped_too_early_is_noticed(keep):
    master = torch.randn(128, 128, device="cuda")
    w = master.to(BF16).requires_grad_()
    grad = torch.zeros_like(w)
    opt = training.AdamW([master], [grad], copies=[w])
    x = torch.randn(64, 128, device="cuda").to(BF16).requires_grad_()
    with keep.hooks():
        y = ((x * 1.0) @ w).sum()
    opt.step(1e-3)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.backward()


def test_what_one_input_of_three_products_takes(keep):
    """1.03 bytes an element, not three times that."""
    rows, width = 4096, 1024
    x = torch.empty(rows, width, dtype=BF16, device="cuda").normal_().requires_grad_()
    ws = [(torch.randn(width, 16, device="cuda") / 32).to(BF16).requires_grad_() for _ in range(3)]
    sum((x * 1.0 @ w).float().sum() for w in ws).backward()          # the products' own workspaces
    with keep.hooks():
        h = x * 1.0
        before = torch.cuda.memory_allocated()
        y = sum((h @ w).float().sum() for w in ws)
        held = torch.cuda.memory_allocated() - before
    exact = rows * width + 4 * rows * width // 128
    assert exact <= held < 1.1 * exact + 3 * rows * 16 * 4 * 3, (held, exact)
    del h
    y.backward()
