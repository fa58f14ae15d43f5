"""How exact the linear cross entropy is, in norms and in signed bias against 64 bits.

The tolerances come from the sums.  u = 2^-24.

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
