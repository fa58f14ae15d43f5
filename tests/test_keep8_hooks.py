"""What Keep8.hooks() keeps and what it leaves alone, on the CPU: a stand-in takes the place of the kernels, which copies."""
import gc
import weakref

import pytest
import torch

from paper_2009_03816_b200 import training


class Stand(training.Keep8):
    """Keeps CPU tensors: codes are a copy, in 16 bits for want of a kernel."""

    def __init__(self):
        self.device = type("Device", (), {"index": -1})()            # what get_device() says of CPU tensors
        self.packed = []

    def _join(self):
        pass

    def pack(self, x):
        self.packed.append(tuple(x.shape))
        return x.clone(), torch.zeros(1)

    def unpack(self, codes, scales, shape, dtype, *, out=None):
        return codes.clone()


@pytest.fixture
def keep():
    return Stand()


def some(*shape, seed=0, dtype=torch.bfloat16):
    return torch.empty(*shape).normal_(generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("change", ["weight", "small", "fp32"])
def test_what_is_changed_after_it_was_saved_is_noticed(keep, change):
    """As without the hooks: a weight stepped before its backward pass raises an error."""
    dtype = torch.float32 if change == "fp32" else torch.bfloat16
    w = some(64, 128, dtype=dtype).requires_grad_()
    x = some(8 if change == "small" else 100, 64, seed=1, dtype=dtype)
    with keep.hooks():
        h = x.clone().requires_grad_() * 1.0
        y = (h @ w).sum()
    with torch.no_grad():
        (w if change == "weight" else h).mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.backward()


def test_what_is_kept_in_8_bits_may_change(keep):
    """Its codes are a copy."""
    w, x = some(64, 128).requires_grad_(), some(100, 64, seed=1)
    with keep.hooks():
        h = x.clone().requires_grad_() * 1.0
        y = (h @ w).sum()
    with torch.no_grad():
        h.zero_()
    y.backward()
    assert keep.packed == [(100, 64)]
    torch.testing.assert_close(w.grad, x.T @ torch.ones(100, 128, dtype=torch.bfloat16))


def test_second_derivatives_of_what_is_left_alone(keep):
    x, w = some(5, 6, dtype=torch.float64).requires_grad_(), some(6, 7, seed=1, dtype=torch.float64).requires_grad_()
    f = lambda: torch.tanh(x @ w).pow(3).sum()
    with keep.hooks():
        y = f()
        (dx,) = torch.autograd.grad(y, x, create_graph=True)
        got = torch.autograd.grad(dx.square().sum(), (x, w))
    (dx,) = torch.autograd.grad(f(), x, create_graph=True)
    for a, b in zip(got, torch.autograd.grad(dx.square().sum(), (x, w))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_results_that_are_left_alone_are_freed(keep, dtype):
    """What an operation saves of its own result must not keep the graph alive that holds it."""
    held = []
    for _ in range(3):
        x = some(20, 30, dtype=dtype).requires_grad_()
        with keep.hooks():
            y = torch.softmax(torch.exp(x), -1)
        held.append(weakref.ref(y))
        held.append(weakref.ref(x))
        del x, y
    gc.collect()
    assert all(ref() is None for ref in held)


def test_one_tensor_is_kept_once(keep):
    """However many operations save it; what has changed in between is another tensor, and so are other views."""
    x = some(100, 64).requires_grad_() * 1.0
    ws = [some(64, 64, seed=i).requires_grad_() for i in range(3)]
    with keep.hooks():
        y = sum((x @ w).float().sum() for w in ws)
        assert keep.packed == [(100, 64)]
        y.backward()
    want = x.detach().T @ torch.ones(100, 64, dtype=torch.bfloat16)
    for w in ws:
        torch.testing.assert_close(w.grad, want)
    keep.packed.clear()
    leaf = some(2, 50, 64).requires_grad_()
    with keep.hooks():
        t = leaf * 1.0
        y = sum((t @ w).float().sum() for w in ws)                   # a view of t each time
        assert len(keep.packed) == 1
        u = t * t                                                    # another shape
        assert len(keep.packed) == 2
        old = t @ ws[0]
        with torch.no_grad():
            t.mul_(2.0)
        new = t @ ws[0]
        assert len(keep.packed) == 3
    del u, y
    ws[0].grad = None
    (old + new).float().sum().backward()
    ones = torch.ones(100, 64, dtype=torch.bfloat16)
    kept = leaf.detach().reshape(100, 64)
    torch.testing.assert_close(ws[0].grad, (kept.T @ ones) + (2 * kept).T @ ones, rtol=2e-2, atol=1e-1)


def test_nothing_outlives_its_graph(keep):
    """Once the graphs that hold them are gone, the codes are; another tensor at the same place is another tensor."""
    w = some(64, 64).requires_grad_()
    context = keep.hooks()
    for i in range(20):
        x = some(100, 64, seed=i).requires_grad_() * 1.0
        with context:
            y = (x @ w).sum()
        w.grad = None
        y.backward()
        torch.testing.assert_close(w.grad, x.detach().T @ torch.ones(100, 64, dtype=torch.bfloat16))
        del x, y
    assert len(keep.packed) == 20


def test_casts_of_weights_are_left_alone(keep):
    """A master weight in fp32 that is cast for each product, as autocast does too."""
    w = some(64, 128, dtype=torch.float32).requires_grad_()
    x = some(100, 64, seed=1).requires_grad_()
    with keep.hooks():
        h = x * 1.0
        y = h @ w.bfloat16()
        z = y @ w.to(torch.bfloat16).t()
        assert keep.packed == [(100, 64), (100, 128)]
    z.sum().backward()
    keep.packed.clear()
    with keep.hooks(), torch.autocast("cpu", dtype=torch.bfloat16):
        h = torch.tanh(torch.nn.functional.linear(x * 1.0, w.t()))
        h = torch.nn.functional.linear(h, w)
    assert (128, 64) not in keep.packed and (64, 128) not in keep.packed and (100, 128) in keep.packed
    h.sum().backward()


def test_broadcast_tensors_are_left_alone(keep):
    """Their codes would take more room than they do."""
    row = some(1, 128, seed=2).requires_grad_() * 1.0
    x = some(100, 128).requires_grad_() * 1.0
    with keep.hooks():
        y = x * row.expand(100, 128)
        assert keep.packed == [(100, 128)]
    y.sum().backward()
