"""Kept activations: autograd, hooks, streams and graphs, large tensors, refusals of the entries."""
import math

import pytest
import torch

from paper_2009_03816_b200 import binding, training
from paper_2009_03816_b200 import build as _build

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def keep():
    _build.build_library()
    return training.Keep8()


def some(*shape, dtype=BF16, seed=0):
    return torch.empty(*shape, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def test_bounds_of_what_is_kept(keep):
    x = some(50, 1000)
    codes, scales = keep.pack(x)
    back = keep.unpack(codes, scales, x.shape, x.dtype)
    half = scales.repeat_interleave(128, 1)[:, :1000].double() / 2
    # half a step of the codes, and the result's rounding
    assert bool(((back.double() - x.double()).abs() <= half * (1 + 2.0 ** -20) + 2.0 ** -8 * x.double().abs()).all())


@pytest.mark.parametrize("kind", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
def test_autograd(keep, gated, kind):
    """Any strides, broadcast upstream gradients; what autograd gives is what the entries give."""
    a = some(3, 70, 40, seed=1).transpose(1, 2).detach().requires_grad_()
    b = some(3, 40, 70, seed=2).requires_grad_() if gated else None
    y = keep(a, b, kind)
    grad = some(3, 40, 70, seed=3)
    y.backward(grad)
    want, kept = keep.activate(a.detach().contiguous(), b.detach() if gated else None, kind)
    da, db = keep.activate_backward(kept, grad, kind)
    assert torch.equal(y, want) and torch.equal(a.grad, da)
    if gated:
        assert torch.equal(b.grad, db)
    c = a.detach().clone().requires_grad_()
    keep(c, b.detach() if gated else None, kind).sum().backward()
    ones, _ = keep.activate_backward(kept, torch.ones_like(grad), kind)
    assert torch.equal(c.grad, ones)
    out = torch.zeros(3, 40, 70, dtype=BF16, device="cuda")
    with torch.no_grad():
        assert keep.activate(a.detach().contiguous(), b.detach() if gated else None, kind, out=out)[0] is out
    assert torch.equal(out, want)


def test_gradient_against_differences(keep):
    """By differences of the formula in 64 bits at the kept values."""
    a, b, grad = some(20, 256, seed=4), some(20, 256, seed=5), some(20, 256, seed=6)
    _, kept = keep.activate(a, b, "gelu")
    da, db = keep.activate_backward(kept, grad, "gelu")
    A = keep.unpack(kept[0], kept[1], a.shape, BF16)              # rounded: the values themselves from codes and scales
    A = kept[0].double() * kept[1].double().repeat_interleave(128, 1)
    B = kept[2].double() * kept[3].double().repeat_interleave(128, 1)
    f = lambda t: t * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3))
    step = 1e-5
    slope = (f(A + step) - f(A - step)) / (2 * step)
    G = grad.double()
    u = 2.0 ** -8
    for got, want in ((da, G * B * slope), (db, G * f(A))):
        assert bool(((got.double() - want).abs() <= u * want.abs() + 2e-6 * (G * B).abs() + 2e-6 * (G * A).abs()).all())


def test_second_derivatives_raise(keep):
    a = some(4, 64).requires_grad_()
    (da,) = torch.autograd.grad(keep(a).float().pow(2).sum(), a, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        da.float().sum().backward()


def test_hooks(keep):
    """Saved activations take 1.03 bytes an element, weights and small tensors are left alone, gradients follow from the kept values."""
    x, w = some(256, 384, seed=7), (some(384, 512, seed=8) / 20).requires_grad_()
    with keep.hooks():
        h = x.clone().requires_grad_() * 1.0
        y = torch.tanh(h @ w)
        torch.cuda.synchronize()
    before = keep.launches
    y.sum().backward()
    assert keep.launches > before                                   # something was brought back
    codes, scales = keep.pack(x)
    held = keep.unpack(codes, scales, x.shape, x.dtype)
    ty = keep.unpack(*keep.pack(torch.tanh(x @ w.detach())), y.shape, y.dtype)
    d = torch.ones_like(y) * (1 - ty * ty)
    torch.testing.assert_close(w.grad.float(), (held.T @ d).float(), rtol=2e-2, atol=2e-1)
    leaf = some(100, 100, seed=9).requires_grad_()
    version = keep.launches
    with keep.hooks():
        z = (leaf.t() * leaf.t()).sum() + (some(10, 10).requires_grad_() ** 2).sum()      # views of leaves; small tensors
    assert keep.launches == version
    z.backward()
    with keep.hooks(least=50):
        t = some(10, 10, seed=3).requires_grad_() * 2.0
        z = (t ** 2).sum()
    assert keep.launches > version
    z.backward()


def test_streams_and_graphs(keep):
    a, b, grad = some(300, 640, seed=1), some(300, 640, seed=2), some(300, 640, seed=3)

    def run():
        y, kept = keep.activate(a, b, "silu")
        return (y, *keep.activate_backward(kept, grad, "silu", again=True), keep.unpack(*keep.pack(a), a.shape, BF16))

    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held = run()
    a.copy_(some(300, 640, seed=11))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(held, run()))
    own = training.Keep8(stream=side.cuda_stream)
    leaf = a.clone().requires_grad_()
    own(leaf, b, "silu").backward(grad)
    assert torch.equal(leaf.grad, run()[1])


def test_more_than_2_to_31_elements(keep):
    rows, cols = 70_000, 32_768
    x = torch.empty(rows, cols, dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    assert x.numel() > 2 ** 31
    codes, scales = keep.pack(x)
    y, kept = keep.activate(x, None, "silu")
    for r in (0, rows // 2, 65_600, rows - 1):
        c, s = keep.pack(x[r:r + 1])
        assert torch.equal(codes[r:r + 1], c) and torch.equal(scales[r:r + 1], s)
        assert torch.equal(y[r:r + 1], keep.activate(x[r:r + 1], None, "silu")[0]) and torch.equal(kept[0][r:r + 1], c)
    back = keep.unpack(codes, scales, x.shape, BF16, out=y)
    assert torch.equal(back[-1:], keep.unpack(codes[-1:], scales[-1:], (1, cols), BF16))
    da, _ = keep.activate_backward(kept, x, "silu", da=y)
    one, _ = keep.activate_backward(tuple(t[-1:] for t in kept), x[-1:], "silu")
    assert torch.equal(da[-1:], one)


def test_empty(keep):
    x = some(0, 40)
    codes, scales = keep.pack(x)
    assert codes.shape == (0, 48) and scales.shape == (0, 1) and keep.unpack(codes, scales, x.shape, BF16).shape == (0, 40)
    y, kept = keep.activate(x, x)
    assert y.shape == (0, 40) and keep.activate_backward(kept, y)[0].shape == (0, 40)


def test_refusals_of_the_entries(keep):
    lib, ctx = binding.load(), keep.ctx
    x, y = some(8, 64), torch.empty(8, 64, dtype=BF16, device="cuda")
    codes, scales = torch.zeros(8, 64, dtype=torch.int8, device="cuda"), torch.zeros(8, 1, device="cuda")
    p, c, s, o = x.data_ptr(), codes.data_ptr(), scales.data_ptr(), y.data_ptr()
    kind = binding.PSOPS_BF16
    OK, EINVAL, EALIGN = binding.PSOPS_OK, binding.PSOPS_EINVAL, binding.PSOPS_EALIGN
    assert lib.psops_keep_pack(ctx, kind, 8, 64, p, 64, c, s) == OK
    for code, a in ((EINVAL, (binding.PSOPS_F32, 8, 64, p, 64, c, s)), (EINVAL, (kind, -1, 64, p, 64, c, s)), (EINVAL, (kind, 8, 0, p, 64, c, s)),
                    (EINVAL, (kind, 8, 64, None, 64, c, s)), (EINVAL, (kind, 8, 64, p, 63, c, s)), (EINVAL, (kind, 8, 64, p, 64, None, s)),
                    (EINVAL, (kind, 8, 64, p, 64, c, None)), (EINVAL, (kind, 1 << 31, 64, p, 64, c, s)), (EINVAL, (kind, 1, 1 << 31, p, 1 << 31, c, s)),
                    (EALIGN, (kind, 8, 64, p + 1, 64, c, s)), (EALIGN, (kind, 8, 64, p, 64, c + 8, s)), (EALIGN, (kind, 8, 64, p, 64, c, s + 2))):
        assert lib.psops_keep_pack(ctx, *a) == code, a
    assert lib.psops_keep_unpack(ctx, kind, 8, 64, c, s, o, 64) == OK
    assert lib.psops_keep_unpack(ctx, kind, 8, 64, c, s, None, 64) == EINVAL
    assert lib.psops_keep_unpack(ctx, kind, 8, 64, c, s, o + 1, 64) == EALIGN
    act = lambda k=1, a=p, b=None, bc=None, bs=None, out=o: lib.psops_keep_activate(ctx, k, kind, 8, 64, a, 64, b, 64, out, 64, c, s, bc, bs)
    assert act() == OK
    for kw in (dict(k=3), dict(k=-1), dict(a=None), dict(b=p), dict(out=None)):
        assert act(**kw) == EINVAL, kw
    back = lambda k=1, bc=None, bs=None, dy=p, da=o, db=None, yy=None: lib.psops_keep_activate_backward(ctx, k, kind, 8, 64, c, s, bc, bs, dy, 64, da, 64, db, 64, yy, 64)
    assert back() == OK and back(da=None) == OK
    for code, kw in ((EINVAL, dict(k=5)), (EINVAL, dict(dy=None)), (EINVAL, dict(db=o)), (EINVAL, dict(bc=c)), (EALIGN, dict(yy=o + 1)),
                     (EALIGN, dict(bc=c + 4, bs=s))):
        assert back(**kw) == code, kw
    torch.cuda.synchronize()
