"""How exact the linear cross entropy is, in norms and in signed bias against 64 bits.

The tolerances come from the sums.  u = 2^-24.

* The tensor cores cut a running sum off after every 16 products: a chain of n such
  blocks ends c n u of its value nearer to zero, c measured as 0.17 to 0.49 for bf16
  and 0.35 to 1.5 for fp16.  A logit's chains have at most 48 blocks and 0.3 (bf16)
  or 0.6 (fp16) of that is put back; inputs that lean to their label have c of 0.26
  to 0.38 and 0.35 to 0.97, which leaves 0.08 and 0.37 of 48 u; the fp32 sums of up
  to six chains and the base-2 softmax add some 4 u of rounding: 8 u and 22 u of the
  logit.  Where all products have one sign, 0.19 and 0.9 of 48 u stay: 14 u and 48 u.
  Where nothing is cut off, what is put back is the error: 0.3 and 0.6 of 48 u, and
  rounding: 19 u and 33 u.
* dh and dw: a chain has at most 512 blocks, each of which cuts off at most a unit in
  the last place, 2 u: a bias of at most 1024 u = 6.1e-5, and nothing is put back.
  The rounding of the logits' gradients to 16 bits has a bias of its own (a token's
  label has one gradient near -1, whose rounding all of dh's row shares), so that this
  bias is taken against exact sums of logits' gradients that are rounded.  The
  rounding of the N > 250,000 results averages out to some unit roundoff over
  sqrt(N), below 1e-5.  The error as a whole: the logits' gradients are rounded once
  and the results once more, each with the same relative spread at most, so that its
  norm is at most sqrt(2) of that of exact products rounded once.
"""
import math

import pytest
import torch

from paper_2009_03816_b200 import training

import gpu_util

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float16]
SUM_BIAS = 1024 * U + 1e-5
HEADROOM = {torch.bfloat16: 1.0, torch.float16: 32768.0}     # of the logits' gradients in their 16 bits


def _projection(got, want):
    """(signed relative bias, relative error in the 2-norm)."""
    off = got.double() - want
    size = (want * want).sum()
    return float((off * want).sum() / size), float(off.norm() / size.sqrt())


def _leaning(T, D, V, dtype, seed):
    gpu_util.ensure_library()
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.empty(V, D, device="cuda").normal_(0.0, 0.02, generator=g).to(dtype)
    y = torch.randint(0, V, (T,), device="cuda", generator=g)
    lean = torch.empty(T, 1, device="cuda").uniform_(4.0, 16.0, generator=g) / (D * 0.02)
    h = (torch.empty(T, D, device="cuda").normal_(generator=g) + lean * w[y].float() / 0.02).to(dtype)
    return h, w, y


def _rounded(d, dtype):
    return (d * HEADROOM[dtype]).to(dtype).double() / HEADROOM[dtype]


def _exact(h, w, y, grad):
    logits = h.double() @ w.double().T
    lse = torch.logsumexp(logits, 1)
    at = torch.arange(len(y), device="cuda")
    right = logits[at, y]
    d = torch.exp(logits - lse[:, None])
    d[at, y] -= 1.0
    d16 = _rounded(d, h.dtype)
    return lse, lse - right, right, [(x @ w.double() * grad, x.T @ h.double() * grad) for x in (d, d16)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D,V", [(512, 1000, 3000), (256, 1536, 8192), (384, 2048, 5001), (256, 4096, 4096), (100, 4096, 2000)])
def test_leaning_inputs(T, D, V, dtype):
    h, w, y = _leaning(T, D, V, dtype, 5)
    lse, rows, right, (exact, summed) = _exact(h, w, y, 1.0 / T)
    op = training.LinearXent(T, D, V, dtype=dtype)
    loss, rows1, lse1 = op.forward(h, w, y)
    dh1, dw1 = op.backward(h, w, y, lse1, torch.tensor(1.0, device="cuda"), rows=rows1)
    op.close()
    tol = (8 if dtype == torch.bfloat16 else 22) * U
    logit = lse1.double() - rows1.double()                 # what the label's logit came out as
    size = float(right.norm())
    assert abs(float(((logit - right) * right.sign()).sum() / right.abs().sum())) <= tol        # bias
    assert float((logit - right).norm()) <= 2 * tol * size                                      # spread
    assert abs(float((lse1.double() - lse).mean() / lse.mean())) <= tol
    assert float((lse1.double() - lse).norm() / lse.norm()) <= 2 * tol
    assert abs(float(loss) - float(rows.mean())) <= 2 * tol * float(lse.mean())
    for got, want, sums in zip((dh1, dw1), exact, summed):
        error, rounded = _projection(got, want)[1], _projection(want.to(dtype), want)[1]
        bias = _projection(got, sums)[0]
        assert error <= 1.5 * rounded and abs(bias) <= SUM_BIAS, (error / rounded, bias)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [768, 2048])
def test_logits_of_one_sign_and_logits_that_need_no_rounding(D, dtype):
    T = V = 256
    gpu_util.ensure_library()
    g = torch.Generator(device="cuda").manual_seed(6)
    y = torch.arange(T, device="cuda")
    op = training.LinearXent(T, D, V, dtype=dtype, gradients=False)
    w = torch.empty(V, D, device="cuda").normal_(0.0, 0.02, generator=g).to(dtype)
    h = (w.float().sign() * torch.rand(T, D, device="cuda", generator=g)).to(dtype)
    right = (h.double() * w.double()).sum(1)
    _, rows, lse = op.forward(h, w, y)
    bias = float((lse.double() - rows.double() - right).sum() / right.sum())
    assert abs(bias) <= (14 if dtype == torch.bfloat16 else 48) * U, bias
    # one feature in each: the logit 16 at the label and zeros elsewhere, exactly
    h = torch.zeros(T, D, device="cuda")
    h[y, y] = 16.0
    w = torch.eye(V, D, device="cuda").to(dtype)
    _, rows, lse = op.forward(h.to(dtype), w, y)
    want = math.log(math.exp(16.0) + V - 1)
    assert float((lse.double() - want).abs().max()) <= (19 if dtype == torch.bfloat16 else 33) * U * 16.0
    op.close()


@pytest.mark.parametrize("dtype", TYPES)
def test_dh_summed_over_a_long_vocabulary(dtype):
    # 72 tiles of dh on 74 pairs of CTAs: one share, a sum of 131,072 terms
    T, D, V = 2048, 2304, 131_072
    h, w, y = _leaning(T, D, V, dtype, 7)
    op = training.LinearXent(T, D, V, dtype=dtype)
    _, rows, lse = op.forward(h, w, y)
    dh, _ = op.backward(h, w, y, lse, torch.tensor(1024.0, device="cuda"), rows=rows, want=(True, False))
    op.close()
    want, sums = (torch.empty(T, D, device="cuda", dtype=torch.float64) for _ in range(2))
    for a in range(0, T, 512):
        s = h[a:a + 512].double() @ w.double().T
        d = torch.exp(s - torch.logsumexp(s, 1, keepdim=True))
        d[torch.arange(512, device="cuda"), y[a:a + 512]] -= 1.0
        want[a:a + 512] = d @ w.double() * (1024.0 / T)
        sums[a:a + 512] = _rounded(d, dtype) @ w.double() * (1024.0 / T)
    bias, error = _projection(dh, sums)[0], _projection(dh, want)[1]
    rounded = _projection(want.to(dtype), want)[1]
    assert abs(bias) <= SUM_BIAS and error <= 1.5 * rounded, (bias, error / rounded)


@pytest.mark.parametrize("dtype", TYPES)
def test_dw_summed_over_many_tokens_of_one_sign(dtype):
    # labels among the first classes: for the others all 300,000 terms of dw are positive
    T, D, V, first = 300_000, 256, 9728, 100
    gpu_util.ensure_library()
    g = torch.Generator(device="cuda").manual_seed(8)
    w = (0.02 * torch.rand(V, D, device="cuda", generator=g)).to(dtype)
    h = torch.rand(T, D, device="cuda", generator=g).to(dtype)
    y = torch.randint(0, first, (T,), device="cuda", generator=g)
    op = training.LinearXent(T, D, V, dtype=dtype)
    _, rows, lse = op.forward(h, w, y)
    _, dw = op.backward(h, w, y, lse, torch.tensor(1024.0, device="cuda"), rows=rows, want=(False, True))
    op.close()
    want, sums = (torch.zeros(V - first, D, device="cuda", dtype=torch.float64) for _ in range(2))
    for a in range(0, T, 20_000):
        s = h[a:a + 20_000].double() @ w.double().T
        p = torch.exp(s - torch.logsumexp(s, 1, keepdim=True))[:, first:]
        want += p.T @ h[a:a + 20_000].double() * (1024.0 / T)
        sums += _rounded(p, dtype).T @ h[a:a + 20_000].double() * (1024.0 / T)
    bias, error = _projection(dw[first:], sums)[0], _projection(dw[first:], want)[1]
    own, rounded = _projection(sums.to(dtype), sums)      # here the results are much alike: their rounding has a bias too
    assert abs(bias) <= SUM_BIAS + 2 * abs(own) and error <= 1.5 * rounded, (bias, own, error / rounded)
