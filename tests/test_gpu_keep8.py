"""Activations kept in 8 bits: codes and scales exactly by their rule, results within a rounding of the formulas in 64 bits."""
import math

import pytest
import torch

from paper_2009_03816_b200 import binding
from paper_2009_03816_b200 import build as _build

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def keep():
    _build.build_library()
    from paper_2009_03816_b200 import training
    return training.Keep8()


def rule(x):
    """(codes, scales) in 64 bits; the scale's own rounding to fp32 is part of the rule."""
    cols = x.shape[-1]
    x = x.reshape(-1, cols).double()
    codes, scales = [], []
    for c in range(0, cols, 128):
        part = x[:, c:c + 128]
        top = part.abs().amax(1, keepdim=True)
        some = (top >= 2.0 ** -100) & (top < math.inf)
        quotient = (part * 127 / torch.where(some, top, 1.0)).abs()
        code = torch.sign(part) * torch.floor(quotient + 0.5)
        codes.append(torch.where(some, code, 0.0))
        scales.append(torch.where(some, (top.float() / torch.full_like(top, 127.0).float()).double(),
                                  torch.where(top < math.inf, 0.0, math.nan)))
    return torch.cat(codes, 1), torch.cat(scales, 1)


def values(codes, scales):
    return codes * scales.repeat_interleave(128, 1)[:, :codes.shape[1]]


def some(shape, dtype, seed=0, spread=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty(*shape, device="cuda").normal_(generator=gen)
    if spread:
        x *= torch.pow(10.0, torch.empty(*shape[:-1], 1, device="cuda").uniform_(-3, 2, generator=gen))
    return x.to(dtype)


def check_kept(codes, scales, x):
    want_codes, want_scales = rule(x)
    cols = x.shape[-1]
    got = codes.reshape(-1, codes.shape[-1])
    assert torch.equal(got[:, :cols].double(), want_codes)
    assert not got[:, cols:].any()
    got = scales.reshape(-1, scales.shape[-1]).double()
    assert bool(((got == want_scales) | (got.isnan() & want_scales.isnan())).all())


SHAPES = [(1, 1), (1, 16), (3, 7), (5, 127), (4, 128), (2, 129), (7, 255), (33, 1000), (2, 3, 257), (300, 683), (1, 100003), (70000, 8)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_there_and_back(keep, shape, dtype):
    x = some(shape, dtype, seed=sum(shape))
    codes, scales = keep.pack(x)
    check_kept(codes, scales, x)
    back = keep.unpack(codes, scales, x.shape, dtype)
    c, s = rule(x)
    assert torch.equal(back.reshape(c.shape), values(c.float(), s.float()).to(dtype))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("first,ld", [(0, 200), (1, 201), (2, 202), (8, 208), (3, 400)])
def test_rows_anywhere(keep, first, ld, dtype):
    flat = some((40 * ld + 64,), dtype, seed=ld, spread=False)
    x = flat[first:first + 40 * ld].view(40, ld)[:, :190]
    codes, scales = keep.pack(x)
    check_kept(codes, scales, x.contiguous())
    room = torch.full((40 * ld + 64,), 7.0, dtype=dtype, device="cuda")
    out = room[first:first + 40 * ld].view(40, ld)[:, :190]
    keep.unpack(codes, scales, x.shape, dtype, out=out)
    c, s = rule(x.contiguous())
    assert torch.equal(out, values(c.float(), s.float()).to(dtype))
    out.fill_(7.0)
    assert bool((room == 7.0).all())                      # nothing was written beside the rows


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_all_numbers_of_the_type(keep, dtype):
    """Every finite number against every largest number of a block in one octave: all ties are among them."""
    every = torch.arange(1 << 16, device="cuda", dtype=torch.int32).to(torch.uint16 if hasattr(torch, "uint16") else torch.int16)
    every = every.view(torch.int16).view(dtype)
    steps = 128 if dtype == torch.bfloat16 else 1024
    top = (1.0 + torch.arange(steps, device="cuda") / steps).to(dtype)[:: 1 if dtype == torch.bfloat16 else 7]
    small = every[(every.float().abs() <= 2.0) & (every.float().abs() > 2.0 ** -9)]
    for t in top.tolist():
        x = torch.where(small.float().abs() <= t, small, torch.zeros_like(small))
        pad = -x.numel() % 127
        x = torch.cat([x, torch.zeros(pad, dtype=dtype, device="cuda")]).view(-1, 127)
        x = torch.cat([x, torch.full((x.shape[0], 1), t, dtype=dtype, device="cuda")], 1)
        codes, scales = keep.pack(x)
        check_kept(codes, scales, x)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_extremes(keep, dtype):
    big = torch.finfo(dtype).max
    rows = torch.zeros(8, 256, dtype=dtype, device="cuda")
    rows[0, 3] = big
    rows[1, 200] = -big
    rows[2, 5] = torch.finfo(dtype).smallest_normal
    rows[3, 7] = math.inf
    rows[4, 130] = math.nan
    rows[5, 1], rows[5, 255] = -math.inf, 1.0
    rows[6, 9] = torch.finfo(dtype).smallest_normal / 4                    # fp16: kept; bf16: below 2^-100
    codes, scales = keep.pack(rows)
    check_kept(codes, scales, rows)
    back = keep.unpack(codes, scales, rows.shape, dtype)
    assert back[3, :128].isnan().all() and (back[3, 128:] == 0).all()
    assert back[4, 128:].isnan().all() and (back[4, :128] == 0).all()
    assert float(back[0, 3]) == big and float(back[1, 200]) == -big


def act(kind, t):
    if kind == "relu":
        return torch.relu(t)
    if kind == "silu":
        return t * torch.sigmoid(t)
    # (1 + tanh u) / 2 = sigmoid(2 u), which keeps its digits where tanh is close to -1
    return t * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("kind", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape,joint", [((1, 1), False), ((5, 683), True), ((64, 1024), True), ((3, 40, 129), False), ((700, 300), True)],
                         ids=str)
def test_activation(keep, shape, joint, gated, kind, dtype):
    W = shape[-1]
    if joint:
        x = some((*shape[:-1], 2 * W), dtype, seed=W)
        a, b = x[..., :W], x[..., W:]
    else:
        a, b = some(shape, dtype, seed=1), some(shape, dtype, seed=2)
    b = b if gated else None
    grad = some(shape, dtype, seed=3, spread=False)
    y, kept = keep.activate(a, b, kind)
    check_kept(kept[0], kept[1], a.contiguous())
    if gated:
        check_kept(kept[2], kept[3], b.contiguous())
    da, db, again = keep.activate_backward(kept, grad, kind, again=True)
    u = torch.finfo(dtype).eps / 2
    tiny = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134
    # fp32: the sigmoid's exponent is off by some 3 2^-24 of |z|, and a few more operations; where the derivative
    # is a difference of two terms, of the larger of them
    off = lambda t: 2.0 ** -24 * (16 + 6 * (t.abs() if kind == "silu" else 1.6 * t.abs() + 0.08 * t.abs() ** 3).clamp(max=150))

    def near(got, want, size, what):
        bad = ~((got.double() - want).abs() <= u * want.abs() + size + tiny)
        bad &= ~((got.double() == want))                                   # overflow to infinity on both sides
        bad &= ~((want.abs() >= torch.finfo(dtype).max) & got.isinf())
        assert not bool(bad.any()), (what, got[bad][:3], want[bad][:3])

    A, G = a.double(), grad.double()
    B = b.double() if gated else torch.ones_like(A)
    # a sigmoid below 2^-126 is zero (ex2 and rcp without subnormal numbers): off by 2^-126 of what it multiplies
    flush = 2.0 ** -125
    near(y, act(kind, A) * B, (act(kind, A) * B).abs() * off(A) * 2 + flush * (A * B).abs(), "y")
    c, s = rule(a.contiguous())
    A = values(c.float(), s.float()).double().view(shape).requires_grad_(True)
    if gated:
        c, s = rule(b.contiguous())
        B = values(c.float(), s.float()).double().view(shape)
    f = act(kind, A)
    (slope,) = torch.autograd.grad(f.sum(), A)
    A, f = A.detach(), f.detach()
    terms = torch.sigmoid(A if kind == "silu" else 1.5957691216057308 * (A + 0.044715 * A ** 3)) * (1 + (2 + 1.2 * A.abs() ** 3) * 1.0) \
        if kind != "relu" else torch.zeros_like(A)
    # beyond |z| = 20 the second term is below 2^-24 of the first or nothing at all
    terms = torch.where(A > 6, 2.0, terms)
    near(da, G * B * slope, (G * B).abs() * (terms * off(A) * 2 + flush * (1 + A.abs() + 0.3 * A.abs() ** 3)), "da")
    near(again, f * B, (f * B).abs() * off(A) * 2 + flush * (A * B).abs(), "again")
    if gated:
        near(db, G * f, (G * f).abs() * off(A) * 2 + flush * (G * A).abs(), "db")
    else:
        assert db is None
