"""Linear cross entropy against the definition in 64 bits.

Tolerances from counting roundings.  u16 is the unit roundoff of the 16-bit type
(half its epsilon: 2^-8 for bf16, 2^-11 for fp16), u = 2^-24.

* A logit is an fp32 sum of `dim` exact products: its error is at most
  2 dim u (sum of the products' magnitudes) =: e; tensor-core sums may drop the
  bits below the largest term's, which this bound covers for dim >= 4 and
  e >= 8 u times the largest product covers otherwise.
* lse and rows: e twice (label and maximum), plus the roundings of a sum of
  `vocab` exponentials in two stages and of base-2 logarithms: 64 u (1 + |lse|).
* dlogits: |d| (u16 + 2 e + 64 u) + 2^-24 of the largest |grad| (numbers below
  fp16's range); dh and dw: that summed against |w| or |h|, plus u16 of the
  result for the final rounding, plus 2^-25 absolute for fp16 results below its
  normal range, plus fp32 summation 2 n u of the magnitudes.
"""
import math

import pytest
import torch

from paper_2009_03816_b200 import binding, training

import gpu_util

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16)}


def _inputs(T, D, V, dtype, seed, scale=None, masked=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.empty(T, D, device="cuda").normal_(generator=g)
    w = (torch.empty(V, D, device="cuda").normal_(generator=g) * (scale or 2.0 / math.sqrt(D))).to(dtype)
    y = torch.randint(0, V, (T,), device="cuda", generator=g)
    if T:
        h = (h + torch.rand(T, 1, device="cuda", generator=g) * w[y].float()).to(dtype)
    else:
        h = h.to(dtype)
    y[torch.rand(T, device="cuda", generator=g) < masked] = -100
    return h, w, y


def _exact(h, w, y, grad_rows):
    """64-bit values and the magnitudes that the tolerances need."""
    T, V = h.shape[0], w.shape[0]
    keep = (y >= 0) & (y < V)
    h, w = h.double(), w.double()
    h = torch.where(keep[:, None], h, torch.zeros_like(h))
    at = torch.where(keep, y, torch.zeros_like(y))[:, None]
    s = h @ w.T
    e = (2 * h.shape[1] + 8) * U * (h.abs() @ w.T.abs())
    e_row = e.amax(1) if V else e.sum(1)
    lse = torch.where(keep, torch.logsumexp(s, 1), torch.zeros((), dtype=torch.float64, device="cuda"))
    rows = torch.where(keep, lse - s.gather(1, at)[:, 0], torch.zeros_like(lse))
    d = torch.exp(s - torch.logsumexp(s, 1, keepdim=True)) * keep[:, None]
    p = d.clone()
    d.scatter_add_(1, at, -keep.double()[:, None])
    g = torch.where(keep, grad_rows.double(), torch.zeros_like(lse))
    return dict(h=h, w=w, keep=keep, s=s, e_row=e_row, lse=lse, rows=rows, p=p, d=d * g[:, None], g=g,
                dh=(d * g[:, None]) @ w, dw=(d * g[:, None]).T @ h)


def _check_forward(x, loss, rows, lse, reduction="mean"):
    tol = 2 * x["e_row"] + 64 * U * (1 + x["lse"].abs())
    assert bool(((lse.double() - x["lse"]).abs() <= tol).all()), float((lse.double() - x["lse"]).abs().max())
    assert bool(((rows.double() - x["rows"]).abs() <= 2 * tol).all()), float((rows.double() - x["rows"]).abs().max())
    assert bool((rows[~x["keep"]] == 0).all()) and bool((lse[~x["keep"]] == 0).all())
    n = max(1, int(x["keep"].sum())) if reduction == "mean" else 1
    want = x["rows"].sum() / n
    assert abs(float(loss) - float(want)) <= float(2 * tol[x["keep"]].sum()) / n + 2 * U * abs(float(want))


def _check_grads(x, dh, dw, dtype):
    u16 = HALF[dtype]
    top = float(x["g"].abs().max()) if x["g"].numel() else 0.0
    err = x["d"].abs() * (u16 + 64 * U) + x["p"] * x["g"].abs()[:, None] * (2 * x["e_row"] + 128 * U)[:, None]
    if dtype == torch.float16:
        err = err + x["keep"].double()[:, None] * top * 2.0 ** -39       # fp16 holds them scaled by 2^15
    deep_v, deep_t = 2 * x["w"].shape[0] * U, 2 * x["h"].shape[0] * U
    tiny = 2.0 ** -24 if dtype == torch.float16 else 1e-38
    for got, want, spread, size in ((dh, x["dh"], err @ x["w"].abs(), x["d"].abs() @ x["w"].abs() * deep_v),
                                    (dw, x["dw"], err.T @ x["h"].abs(), x["d"].T.abs() @ x["h"].abs() * deep_t)):
        tol = spread + size + want.abs() * u16 * 1.01 + tiny
        off = (got.double() - want).abs()
        assert bool((off <= tol).all()), (float(off.max()), float((off / tol).max()))


def _run(T, D, V, dtype, seed=1, masked=0.0, reduction="mean"):
    gpu_util.ensure_library()
    h, w, y = _inputs(T, D, V, dtype, seed, masked=masked)
    grad = torch.tensor(1.7, device="cuda")
    n = max(1, int((y >= 0).sum()))
    x = _exact(h, w, y, torch.full((T,), 1.7 / (n if reduction == "mean" else 1), device="cuda", dtype=torch.float64))
    op = training.LinearXent(max(1, T), D, V, dtype=dtype)
    loss, rows, lse = op.forward(h, w, y, reduction)
    dh, dw = op.backward(h, w, y, lse, grad, reduction)
    _check_forward(x, loss, rows, lse, reduction)
    _check_grads(x, dh, dw, dtype)
    again = op.forward(h, w, y, reduction), op.backward(h, w, y, lse, grad, reduction)
    for a, b in zip((loss, rows, lse, dh, dw), (*again[0], *again[1])):
        assert torch.equal(a, b), "two runs differ"
    op.close()


SHAPES = [(1, 1, 1), (1, 8, 2), (2, 3, 5), (256, 84, 10), (3, 64, 257), (65, 72, 255), (255, 128, 256), (256, 64, 512),
          (257, 200, 1000), (31, 1000, 3001), (513, 264, 700), (1, 512, 4097), (129, 65, 129), (300, 520, 2049),
          (1024, 256, 8193), (64, 4096, 640), (5, 13_000, 300)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,V", SHAPES)
def test_sizes(T, D, V, dtype):
    _run(T, D, V, dtype)


@pytest.mark.parametrize("T,D,V", [(1600, 200, 700), (2500, 61, 130), (1536, 1024, 257), (9000, 72, 500)])
def test_many_tokens_and_a_small_vocabulary(T, D, V):
    # dw in shares of the tokens, and with most tokens left out fewer shares than there is room for
    _run(T, D, V, torch.bfloat16, seed=61)
    _run(T, D, V, torch.float16, seed=62, masked=0.97, reduction="sum")


@pytest.mark.parametrize("masked", [0.3, 0.9, 1.0])
@pytest.mark.parametrize("reduction", ["mean", "sum"])
def test_left_out_tokens(masked, reduction):
    _run(333, 136, 600, torch.bfloat16, seed=3, masked=masked, reduction=reduction)
    _run(333, 136, 600, torch.float16, seed=4, masked=masked, reduction=reduction)


HEADS = [(1, 2048, 8), (300, 100, 64), (77, 550, 50), (4096, 33, 17), (4097, 40, 17), (1000, 7, 33), (9, 1, 64), (130, 1600, 12)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,V", HEADS)
def test_few_classes(T, D, V, dtype):
    _run(T, D, V, dtype, seed=21, masked=0.2)
    _run(T, D, V, dtype, seed=22, reduction="sum")


FEW = [(1, 4096, 3000), (2, 1000, 70_001), (3, 61, 5000), (4, 256, 100), (4, 2048, 1001), (1, 600, 66), (2, 4100, 300),
       (1, 30_000, 70), (7, 3000, 777), (8, 2056, 4096), (9, 64, 500)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,V", FEW)
def test_few_tokens(T, D, V, dtype):
    _run(T, D, V, dtype, seed=23)
    _run(T, D, V, dtype, seed=24, masked=0.5, reduction="sum")


@pytest.mark.parametrize("T,D,V", [(50, 30, 20), (6, 200, 900), (4, 200, 900), (3, 1500, 333), (2, 3001, 100)])
def test_small_forms_leave_out_and_weigh_like_the_others(T, D, V):
    h, w, y = _inputs(T, D, V, torch.bfloat16, 31, masked=0.4)
    y[0], y[1] = V - 1, -7
    op = training.LinearXent(T, D, V)
    bad = h.clone()
    bad[y < 0] = float("nan")
    want, got = op.forward(h, w, y), op.forward(bad, w, y)
    grad = torch.randn(T, device="cuda")
    want_g, got_g = op.backward(h, w, y, want[2], grad, "none"), op.backward(bad, w, y, got[2], grad, "none")
    for a, b in zip((*want, *want_g), (*got, *got_g)):
        assert torch.equal(a, b)
    x = _exact(h, w, y, grad)
    _check_forward(x, *want)
    _check_grads(x, *want_g, torch.bfloat16)
    h[0] = float("nan")
    loss, rows, lse = op.forward(h, w, y)
    assert math.isnan(float(loss)) and math.isnan(float(rows[0])) and int(rows.isnan().sum()) == 1
    # the large form after the small one on one context, and the small one again: counters start anew
    if T == 6:
        big = training.LinearXent(40, D, V)
        h2, _, y2 = _inputs(40, D, V, torch.bfloat16, 32)
        for _ in range(2):
            first = big.forward(bad, w, y)
            assert all(torch.equal(a, b) for a, b in zip(first, want))
            _check_forward(_exact(h2, w, y2, grad.new_zeros(40)), *big.forward(h2, w, y2))
        big.close()
    op.close()


def test_several_pieces_of_the_vocabulary():
    # 32,768 rows of workspace make a piece 8,192 entries: three pieces, the last one short
    T, D, V = 700, 128, 20_011
    h, w, y = _inputs(T, D, V, torch.bfloat16, 8, masked=0.2)
    x = _exact(h, w, y, torch.full((T,), 0.5, device="cuda"))
    op = training.LinearXent(32_768, D, V)
    loss, rows, lse = op.forward(h, w, y, "sum")
    dh, dw = op.backward(h, w, y, lse, torch.tensor([0.5], device="cuda"), "sum")
    _check_forward(x, loss, rows, lse, "sum")
    _check_grads(x, dh, dw, torch.bfloat16)
    op.close()


@pytest.mark.parametrize("D", [64, 61])
def test_a_small_vocabulary_in_several_pieces(D):
    # 200,192 rows of workspace make a piece 2,048 entries; dw is summed in shares, piece by piece
    T, V = 2000, 2300
    h, w, y = _inputs(T, D, V, torch.bfloat16, 71, masked=0.1)
    x = _exact(h, w, y, torch.ones(T, device="cuda"))
    op = training.LinearXent(200_000, D, V)
    loss, rows, lse = op.forward(h, w, y, "sum")
    dh, dw = op.backward(h, w, y, lse, torch.ones(1, device="cuda"), "sum")
    _check_forward(x, loss, rows, lse, "sum")
    _check_grads(x, dh, dw, torch.bfloat16)
    op.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_per_token_gradients(dtype):
    T, D, V = 150, 96, 777
    h, w, y = _inputs(T, D, V, dtype, 5, masked=0.2)
    grad = torch.randn(T, device="cuda") * 10.0 ** torch.randint(-3, 3, (T,), device="cuda").float()
    grad[7] = 0.0
    x = _exact(h, w, y, grad)
    op = training.LinearXent(T, D, V, dtype=dtype)
    _, _, lse = op.forward(h, w, y)
    dh, dw = op.backward(h, w, y, lse, grad, "none")
    _check_grads(x, dh, dw, dtype)
    assert bool((dh[7] == 0).all())
    op.close()


def test_nothing_leaks_from_tokens_that_are_left_out():
    T, D, V = 290, 72, 500
    h, w, y = _inputs(T, D, V, torch.bfloat16, 6, masked=0.5)
    op = training.LinearXent(T, D, V)
    want = op.forward(h, w, y)
    want_g = op.backward(h, w, y, want[2], torch.tensor(1.0, device="cuda"))
    bad = h.clone()
    out = torch.nonzero(y < 0)[:, 0]
    bad[out[0::3]] = float("nan")
    bad[out[1::3]] = float("inf")
    bad[out[2::3]] = torch.finfo(torch.bfloat16).min
    y2 = y.clone()
    y2[out[0]], y2[out[1]], y2[out[2]] = V, -1, 2 ** 40      # any label outside the vocabulary
    got = op.forward(bad, w, y2)
    got_g = op.backward(bad, w, y2, got[2], torch.tensor(1.0, device="cuda"))
    for a, b in zip((*want, *want_g), (*got, *got_g)):
        assert torch.equal(a, b)
    assert bool((got_g[0][out] == 0).all())
    op.close()


def test_extreme_logits_and_nan_rows():
    T, D, V = 40, 64, 300
    h, w, y = _inputs(T, D, V, torch.bfloat16, 7)
    h[3] *= 1000                                             # logits in the thousands: one probability is 1
    h[5] = 0                                                 # all logits equal
    op = training.LinearXent(T, D, V)
    x = _exact(h, w, y, torch.full((T,), 1.0 / T, device="cuda"))
    loss, rows, lse = op.forward(h, w, y)
    _check_forward(x, loss, rows, lse)
    _check_grads(x, *op.backward(h, w, y, lse, torch.tensor(1.0, device="cuda")), torch.bfloat16)
    assert float(lse[5]) == pytest.approx(math.log(V), rel=4 * U)
    h[9] = float("nan")
    loss, rows, lse = op.forward(h, w, y)
    assert math.isnan(float(loss)) and math.isnan(float(rows[9])) and math.isnan(float(lse[9]))
    ok = torch.arange(T, device="cuda") != 9
    assert bool(rows[ok].isfinite().all())
    dh, _ = op.backward(h, w, y, lse, torch.tensor(1.0, device="cuda"))
    assert bool(dh[9].isnan().all()) and bool(dh[ok].isfinite().all())
    op.close()


@pytest.mark.parametrize("D", [64, 61])
def test_strides_offsets_and_untouched_gaps(D):
    T, V = 70, 333
    h, w, y = _inputs(T, D, V, torch.float16, 9)
    x = _exact(h, w, y, torch.full((T,), 1.0, device="cuda"))
    op = training.LinearXent(T, D, V, dtype=torch.float16)
    loss, rows, lse = op.forward(h, w, y, "sum")
    grad = torch.tensor(1.0, device="cuda")
    dh, dw = op.backward(h, w, y, lse, grad, "sum")
    _check_grads(x, dh, dw, torch.float16)
    for pad, shift in ((8, 0), (8, 8), (3, 0), (5, 1), (0, 1), (7, 3)):
        def strided(t):
            flat = torch.full((t.shape[0] * (D + pad) + shift + 16,), 3.25, device="cuda", dtype=t.dtype)
            view = flat[shift:shift + t.shape[0] * (D + pad)].view(t.shape[0], D + pad)[:, :D]
            view.copy_(t)
            return flat, view
        (_, h2), (_, w2) = strided(h), strided(w)
        (fh, dh2), (fw, dw2) = strided(dh * 0), strided(dw * 0)
        got = op.forward(h2, w2, y, "sum")
        op.backward(h2, w2, y, got[2], grad, "sum", dh=dh2, dw=dw2)
        for a, b in zip((loss, rows, lse, dh, dw), (*got, dh2, dw2)):
            assert torch.equal(a, b), (pad, shift)
        for flat, view in ((fh, dh2), (fw, dw2)):
            view.fill_(3.25)
            assert bool((flat == 3.25).all()), "wrote beside the rows"
    op.close()


@pytest.mark.parametrize("T,D,V", [(7, 64, 300), (40, 64, 300), (20, 32, 30)])
def test_confident_tokens_keep_their_digits_with_rows(T, D, V):
    # every token is all but certain: its loss, and with it its gradient, is about 1e-5 to 1e-3.  The loss itself is
    # good to the fp32 error of a logit of about 20 (2e-6 and less); the gradient may add 16-bit roundings to that.
    h, w, y = _inputs(T, D, V, torch.bfloat16, 51)
    g = torch.Generator(device="cuda").manual_seed(52)
    lean = 14 + 4 * torch.rand(T, 1, device="cuda", generator=g)
    h = (h.float() * 0.1 + lean * w[y].float() / (w[y].float() ** 2).sum(1, keepdim=True)).to(torch.bfloat16)
    op = training.LinearXent(T, D, V)
    loss, rows, lse = op.forward(h, w, y)
    x = _exact(h, w, y, torch.ones(T, device="cuda"))
    assert float(x["rows"].median()) < 1e-3
    dh, dw = op.backward(h, w, y, lse, torch.tensor(1.0, device="cuda"), "sum", rows=rows)
    off = (rows.double() - x["rows"]).abs()                       # what the forward pass is off by
    assert bool((off <= 4 * x["e_row"] + 64 * U * (1 + x["lse"].abs())).all())
    spread = (HALF[torch.bfloat16] * x["d"].abs() + 2e-5 * x["p"])
    spread.scatter_add_(1, y[:, None], (off + 4 * U * x["rows"])[:, None])
    spread.scatter_add_(1, y[:, None], -2e-5 * x["p"].gather(1, y[:, None]))
    tol = spread @ x["w"].abs() + x["dh"].abs() * HALF[torch.bfloat16] * 1.02 + 1e-9
    assert bool(((dh.double() - x["dh"]).abs() <= tol).all())
    tol = spread.T @ x["h"].abs() + x["dw"].abs() * HALF[torch.bfloat16] * 1.02 + 1e-9
    assert bool(((dw.double() - x["dw"]).abs() <= tol).all())
    op.close()


def test_gradients_against_differences():
    T, D, V = 24, 32, 50
    h, w, y = _inputs(T, D, V, torch.bfloat16, 11, masked=0.2)
    op = training.LinearXent(T, D, V)
    loss, rows, lse = op.forward(h, w, y)
    dh, dw = op.backward(h, w, y, lse, torch.tensor(1.0, device="cuda"))
    # a step of 2^-4 of an element's own power of two moves it exactly; the loss has curvature below 1 in these units
    for t, grad in ((h, dh), (w, dw)):
        for i, j in ((0, 0), (3, 7), (11, 31), (23, 16)):
            keep = t[i, j].clone()
            eps = max(2.0 ** math.floor(math.log2(max(abs(float(keep)), 2.0 ** -6))), 2.0 ** -6) / 16
            t[i, j] = keep + eps
            up, a = float(t[i, j]), float(op.forward(h, w, y)[0])
            t[i, j] = keep - eps
            down, b = float(t[i, j]), float(op.forward(h, w, y)[0])
            t[i, j] = keep
            # central difference: third derivative <= 1, losses good to 1e-6, gradient good to 2^-7
            slope = (a - b) / (up - down)
            assert abs(slope - float(grad[i, j])) <= eps ** 2 + 4e-6 / (up - down) + abs(slope) * 2.0 ** -7 + 1e-5


def test_autograd_matches_and_batched_shapes():
    T, D, V = 6 * 20, 64, 200
    h, w, y = _inputs(T, D, V, torch.bfloat16, 12, masked=0.3)
    op = training.LinearXent(T, D, V)
    loss, rows, lse = op.forward(h, w, y)
    dh, dw = op.backward(h, w, y, lse, torch.tensor(2.0, device="cuda"), rows=rows)
    h3 = h.view(6, 20, D).clone().requires_grad_()
    w3 = w.clone().requires_grad_()
    out = op(h3, w3, y.view(6, 20))
    (2.0 * out).backward()
    assert torch.equal(out, loss) and torch.equal(h3.grad.view(T, D), dh) and torch.equal(w3.grad, dw)
    each = op(h3, w3.detach(), y.view(6, 20), "none")
    assert torch.equal(each.view(-1), rows)
    h3.grad = None
    each.sum().backward()
    assert h3.grad.shape == h3.shape
    op.close()


def test_autograd_of_slices_and_broadcast_inputs():
    B, S, D, V = 5, 21, 64, 130
    h, w, y = _inputs(B * S, D, V, torch.bfloat16, 41)
    h, y = h.view(B, S, D), y.view(B, S)
    op = training.LinearXent(B * S, D, V)
    # next-token slices: neither h nor the labels can be seen as one run of rows
    h1, w1 = h.clone().requires_grad_(), w.clone().requires_grad_()
    op(h1[:, :-1], w1, y[:, 1:]).backward()
    flat, labels = h[:, :-1].reshape(-1, D), y[:, 1:].reshape(-1)
    loss, rows, lse = op.forward(flat, w, labels)
    dh, dw = op.backward(flat, w, labels, lse, torch.tensor(1.0, device="cuda"), rows=rows)
    assert torch.equal(h1.grad[:, :-1].reshape(-1, D), dh) and torch.equal(w1.grad, dw)
    assert bool((h1.grad[:, -1] == 0).all())
    # one hidden state shared by all tokens, and weights that are a transposed view
    one = h[0, 0].clone().requires_grad_()
    wt = w.t().contiguous().requires_grad_()
    op(one.expand(B * S, D), wt.t(), y.reshape(-1), "sum").backward()
    full = h[0, 0].expand(B * S, D).contiguous()
    _, rows, lse = op.forward(full, w, y.reshape(-1), "sum")
    dh, dw = op.backward(full, w, y.reshape(-1), lse, torch.tensor(1.0, device="cuda"), "sum", rows=rows)
    assert torch.equal(wt.grad, dw.t())
    want = dh.double().sum(0)
    assert bool(((one.grad.double() - want).abs() <= HALF[torch.bfloat16] * (want.abs() + dh.double().abs().sum(0))).all())
    op.close()


def test_follows_the_current_stream():
    T, D, V = 400, 64, 3000
    h, w, y = _inputs(T, D, V, torch.bfloat16, 42)
    grad = torch.tensor(1.0, device="cuda")
    op = training.LinearXent(T, D, V)
    want = op.forward(h, w, y)
    want_g = op.backward(h, w, y, want[2], grad)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for k in range(9):
        with torch.cuda.stream(streams[k % 3]):
            got = op.forward(h, w, y)
            got_g = op.backward(h, w, y, got[2], grad)
            same = [torch.equal(a, b) for a, b in zip((*want, *want_g), (*got, *got_g))]
        assert all(same), k
    fixed = training.LinearXent(T, D, V, stream=streams[0].cuda_stream)
    got = fixed.forward(h, w, y)
    assert fixed.stream == streams[0].cuda_stream
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    op.close(), fixed.close()


def test_weights_past_32_bit_offsets():
    # 2.4e9 elements of w: both the offset in elements and in bytes pass 32 bits
    T, D, V = 6, 4096, 590_000
    g = torch.Generator(device="cuda").manual_seed(5)
    w = torch.empty(V, D, device="cuda", dtype=torch.bfloat16).normal_(0.0, 0.02, generator=g)
    h = torch.empty(T, D, device="cuda", dtype=torch.bfloat16).normal_(generator=g)
    y = torch.tensor([V - 1, 0, V // 2, V - 300, 2 ** 19 + 1, -5], device="cuda")
    op = training.LinearXent(T, D, V)
    for n in (T, 2):                                  # on the tensor cores, and as few tokens
        loss, rows, lse = op.forward(h[:n], w, y[:n])
        keep = y[:n] >= 0
        s = torch.cat([h[:n].double() @ w[i:i + 100_000].double().T for i in range(0, V, 100_000)], 1)
        want = torch.logsumexp(s, 1)
        e = (2 * D + 8) * U * (h[:n].double().abs() @ w[:1000].double().abs().T).amax(1) * 1.5
        assert bool(((lse.double() - want).abs()[keep] <= (2 * e + 64 * U * (1 + want))[keep]).all())
        right = s.gather(1, y[:n].clamp(min=0)[:, None])[:, 0]
        assert bool(((rows.double() - (want - right)).abs()[keep] <= (4 * e + 128 * U * (1 + want))[keep]).all())
        dh, dw = op.backward(h[:n], w, y[:n], lse, torch.tensor(1.0, device="cuda"), "sum")
        for v in (0, V - 1, V - 300, 2 ** 19 + 1, 2 ** 19):
            d = torch.exp(s[:, v] - want) - (y[:n] == v).double()
            d = torch.where(keep, d, torch.zeros_like(d))
            exact = d @ h[:n].double()
            tol = (d.abs() * (HALF[torch.bfloat16] + 1e-4)) @ h[:n].double().abs() + exact.abs() * HALF[torch.bfloat16] * 1.01 + 1e-9
            assert bool(((dw[v].double() - exact).abs() <= tol).all()), v
        assert bool(dh.isfinite().all()) and (n == 2 or bool((dh[5] == 0).all()))
        del s, dw
    op.close()


def test_no_tokens_and_fewer_tokens_than_made_for():
    D, V = 40, 90
    h, w, y = _inputs(700, D, V, torch.bfloat16, 13)
    op = training.LinearXent(700, D, V)
    op.backward(h, w, y, op.forward(h, w, y)[2], torch.tensor(1.0, device="cuda"))   # fills the workspace
    loss, rows, lse = op.forward(h[:0], w, y[:0])
    dh, dw = op.backward(h[:0], w, y[:0], lse, torch.tensor(1.0, device="cuda"))
    assert float(loss) == 0.0 and rows.numel() == 0 and dh.shape == (0, D) and bool((dw == 0).all())
    x = _exact(h[:37], w, y[:37], torch.full((37,), 1.0 / 37, device="cuda"))
    loss, rows, lse = op.forward(h[:37], w, y[:37])
    _check_forward(x, loss, rows, lse)
    _check_grads(x, *op.backward(h[:37], w, y[:37], lse, torch.tensor(1.0, device="cuda")), torch.bfloat16)
    none, dw = op.backward(h[:37], w, y[:37], lse, torch.tensor(1.0, device="cuda"), want=(False, True))
    assert none is None
    dh, none = op.backward(h[:37], w, y[:37], lse, torch.tensor(1.0, device="cuda"), want=(True, False))
    assert none is None
    _check_grads(x, dh, dw, torch.bfloat16)
    op.close()


def test_other_stream_and_graph_replay():
    T, D, V = 100, 64, 600
    h, w, y = _inputs(T, D, V, torch.bfloat16, 14)
    op = training.LinearXent(T, D, V)
    want = op.forward(h, w, y)
    want_g = op.backward(h, w, y, want[2], torch.tensor(1.0, device="cuda"))
    grad = torch.tensor(1.0, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        op2 = training.LinearXent(T, D, V)
        graph = torch.cuda.CUDAGraph()
        hs = torch.zeros_like(h)
        with torch.cuda.graph(graph, stream=side):
            got = op2.forward(hs, w, y)
            got_g = op2.backward(hs, w, y, got[2], grad)
        hs.copy_(h)
        graph.replay()
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip((*want, *want_g), (*got, *got_g)):
        assert torch.equal(a, b)
    del graph
    op.close(), op2.close()


def test_refusals():
    T, D, V = 10, 64, 30
    h, w, y = _inputs(T, D, V, torch.bfloat16, 15)
    op = training.LinearXent(T, D, V)
    _, _, lse = op.forward(h, w, y)
    one = torch.tensor(1.0, device="cuda")
    bad = [
        lambda: training.LinearXent(0, D, V), lambda: training.LinearXent(T, 0, V), lambda: training.LinearXent(T, D, 0),
        lambda: training.LinearXent(T, D, V, dtype=torch.float32), lambda: training.LinearXent(T, D, V, device="cpu"),
        lambda: training.LinearXent(1 << 25, D, V), lambda: training.LinearXent(T, D, 2 ** 31),
        lambda: op.forward(h.half(), w, y), lambda: op.forward(h, w.half(), y), lambda: op.forward(h.cpu(), w, y),
        lambda: op.forward(h, w[:29], y), lambda: op.forward(h[:, :60], w, y), lambda: op.forward(h, w, y[:9]),
        lambda: op.forward(h, w, y.int()), lambda: op.forward(h, w, y, "none"), lambda: op.forward(h.t().contiguous().t(), w, y),
        lambda: op.forward(torch.cat([h, h]), w, torch.cat([y, y])),
        lambda: op.backward(h, w, y, lse[:9], one), lambda: op.backward(h, w, y, lse, one, "none"),
        lambda: op.backward(h, w, y, lse, 1.0), lambda: op.backward(h, w, y, lse, one.double()),
        lambda: op.backward(h, w, y, lse, one, dh=h[:9]), lambda: op.backward(h, w, y, lse, one, dw=w.float()),
        lambda: op.backward(h, w, y, lse, one, "max"),
    ]
    for k, f in enumerate(bad):
        with pytest.raises(binding.PsopsError) as e:
            f()
        assert e.value.code == binding.PSOPS_EINVAL, k
    alone = training.LinearXent(T, D, V, gradients=False)
    alone.forward(h, w, y)
    with pytest.raises(binding.PsopsError) as e:
        alone.backward(h, w, y, lse, one)
    assert e.value.code == binding.PSOPS_ESTATE
    odd = torch.zeros(V * D + 1, device="cuda", dtype=torch.bfloat16)[1:].view(V, D)
    with pytest.raises(binding.PsopsError) as e:
        binding.psops_xent_forward(op.ctx, h, D, odd, D, y, T, binding.PSOPS_MEAN, lse, None, None)
    assert e.value.code == binding.PSOPS_EALIGN
    op.close(), alone.close()


def test_loss_as_the_fitness_of_a_swarm():
    """The device loss of every worker goes straight into the synchronisation."""
    K, D, V, T = 4, 16, 12, 64
    torch.manual_seed(2)
    n = V * D
    x = torch.randn(K, n, device="cuda")
    h = torch.randn(T, D, device="cuda", dtype=torch.bfloat16)
    y = torch.randint(0, V, (T,), device="cuda")
    op = training.LinearXent(T, D, V, gradients=False)
    losses = torch.stack([op.forward(h, x[k].view(V, D).bfloat16(), y)[0] for k in range(K)])
    swarm = binding.Swarm(x, torch.zeros_like(x), x.clone(), m_max=0.7, m_min=0.7, c1=1.5, c2=1.5, seed=3)
    swarm.set_losses(losses)
    swarm.sync()
    g, improved, _ = swarm.info()
    assert g == int(losses.argmin()) and improved.all()
    swarm.close(), op.close()
