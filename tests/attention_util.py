"""Attention in 64 bits from the formulas, with a bound for each element of what a
correct computation may be off by, counted in roundings:

  u    half a step of the 16-bit type, relative: p and ds once each in their
       products, every result once
  f    fp32 arithmetic: a score is a sum of dim products and a few more operations
"""
import math

import torch

F = 2.0 ** -24


def lengths_to_offsets(lengths, first=0, device="cuda"):
    at = [first]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device=device)


def reference(q, k, v, lengths, first=0, grad=None, bias=None, buckets=None, scale=None):
    """Dict name -> (exact, bound); rows of no sequence are zero in both."""
    T, H, D = q.shape
    G = k.shape[1]
    g = H // G
    dev = q.device
    scale = scale if scale is not None else D ** -0.5
    u = torch.finfo(q.dtype).eps / 2
    tiny = 2.0 ** -25 if q.dtype == torch.float16 else 2.0 ** -134       # half the smallest number's step
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64, device=dev)
    R = {"out": [zero(T, H, D), zero(T, H, D)], "lse": [zero(H, T), zero(H, T)]}
    if grad is not None:
        R.update(dq=[zero(T, H, D), zero(T, H, D)], dk=[zero(T, G, D), zero(T, G, D)], dv=[zero(T, G, D), zero(T, G, D)])
        if bias is not None:
            R["dbias"] = [zero(len(buckets), H), zero(len(buckets), H)]
    # fp16: what is smaller than this in ds is lost in the scaled range (2^14 down to 2^-25)
    lost = 0.0
    if grad is not None and q.dtype == torch.float16 and T:
        lost = 2.0 ** -37 * float(grad.double().norm(dim=-1).max() * v.double().norm(dim=-1).max())
    at = first
    for n in lengths:
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        d = torch.arange(n, device=dev)[:, None] - torch.arange(n, device=dev)
        for h in range(H):
            Q, K, V = q[rows, h].double(), k[rows, h // g].double(), v[rows, h // g].double()
            x = scale * (Q @ K.T)
            size = scale * (Q.abs() @ K.abs().T)
            if bias is not None:
                of = torch.bucketize(d.clamp(min=0), torch.tensor(buckets, device=dev), right=True) - 1
                b = bias[:, h].double()[of]
                x = x + b
                size = size + b.abs().nan_to_num(posinf=0.0)
            x = torch.where(d >= 0, x, -math.inf)
            size = torch.where(d >= 0, size, 0.0)
            lse = torch.logsumexp(x, -1)
            R["lse"][0][h, rows] = lse
            # a score: D / 16 cut sums (a step each, 2 F) and its products' sum, scaling, bias, the conversion to base 2
            score = size * F * (D / 8 + 8) + F * (8 + 4 * lse.abs().nan_to_num(posinf=0.0)[:, None])
            most = score.amax(-1)
            R["lse"][1][h, rows] = most + F * (8 + 2 * lse.abs()) + n * F / 16
            p = torch.exp(x - lse.nan_to_num(neginf=0.0)[:, None])
            # relative: two scores' errors (its own and the sum's), exp2 and sums in fp32
            rel = score + most[:, None] + F * (16 + n / 16)
            o = p @ V
            e_out = (p * (u + rel)) @ V.abs() * (1 + 2 * u) + u * o.abs() + tiny
            R["out"][0][rows, h], R["out"][1][rows, h] = o, e_out
            if grad is None:
                continue
            dO = grad[rows, h].double()
            dp = dO @ V.T
            delta = (dO * o).sum(-1, keepdim=True)
            ds = torch.where(d >= 0, p * (dp - delta), 0.0)
            e_delta = (dO.abs() * e_out).sum(-1, keepdim=True) + F * D * (dO * o).abs().sum(-1, keepdim=True)
            e_dp = (dO.abs() @ V.abs().T) * F * (D / 8 + 8)
            e_ds = torch.where(d >= 0, p * (e_delta + e_dp) + rel * ds.abs() * (1 + u), 0.0)
            in_product = e_ds + u * (ds.abs() + e_ds) + torch.where(d >= 0, lost, 0.0)
            sums = 2 * F * (n / 16 + 8)                                   # cut sums of up to n terms
            dq = scale * (ds @ K)
            R["dq"][0][rows, h] = dq
            R["dq"][1][rows, h] = (scale * (in_product + sums * ds.abs()) @ K.abs()) * (1 + 2 * u) + u * dq.abs() + tiny
            R["dk"][0][rows, h // g] += scale * (ds.T @ Q)
            R["dk"][1][rows, h // g] += (scale * (in_product + sums * g * ds.abs()).T @ Q.abs()) * (1 + 2 * u)
            R["dv"][0][rows, h // g] += p.T @ dO
            R["dv"][1][rows, h // g] += ((p * (u + rel + sums * g)).T @ dO.abs()) * (1 + 2 * u) + n * 2.0 ** -38 * dO.abs().amax()
            if bias is not None:
                keep = d >= 0
                R["dbias"][0][:, h].index_add_(0, of[keep], ds[keep])
                R["dbias"][1][:, h].index_add_(0, of[keep], e_ds[keep] + F * (n + 64) * ds[keep].abs())
    for name in ("dk", "dv"):
        if name in R:
            R[name][1] += u * (R[name][0].abs() + R[name][1]) + tiny
    if "dbias" in R:
        w = 2.0 ** -24 if bias.dtype == torch.float32 else u
        R["dbias"][1] += w * (R["dbias"][0].abs() + R["dbias"][1]) + tiny
    return R


def compare(got, want, what=""):
    """`got`: name -> tensor; every element within its bound."""
    for name, t in got.items():
        exact, bound = want[name]
        off = (t.double() - exact).abs()
        bad = ~(off <= bound) & ~((t.double() == exact) | (t.double().isnan() & exact.isnan()))
        if bool(bad.any()):
            i = tuple(int(x) for x in torch.nonzero(bad)[0])
            raise AssertionError(f"{what} {name}: {int(bad.sum())} of {bad.numel()} outside; first at {i}: got {float(t[i])!r}, "
                                 f"exact {float(exact[i])!r}, bound {float(bound[i]):.3g}")


def inputs(tokens, heads, kv_heads, dim, dtype, seed=0, grad=True, buckets=None, bias_dtype=None, spread=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.empty(*s, device="cuda").normal_(generator=gen)
    x = normal(tokens, heads + 2 * kv_heads, dim)
    x[:, :heads] *= spread
    x = x.to(dtype)
    out = {"q": x[:, :heads], "k": x[:, heads:heads + kv_heads], "v": x[:, heads + kv_heads:]}
    if buckets is not None:
        out["bias"] = normal(len(buckets), heads).to(bias_dtype or dtype)
    if grad:
        out["grad"] = normal(tokens, heads, dim).to(dtype)
    return out
