"""AdamW over many tensors and the gradient norm, against plain implementations.

Two references.  (1) The documented fp32 sequence with every operation rounded
by itself, computed on the CPU: the library has to give the same
bits.  (2) The formula in 64 bits, with a tolerance from counting roundings:
u = 2^-24; m' and v' each take at most 4 roundings of same-signed or bounded
terms; p' takes 1 for the decay product, 1 for the final difference and at most
4 + 4 + 3 in the step (m', its product, the denominator, the quotient; the
constants are rounded once each).
"""
import math

import numpy as np
import pytest
import torch

from paper_2009_03816_b200 import binding, training

import gpu_util

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
B1, B2, EPS = 0.9, 0.999, 1e-8
SIZES = [1, 0, 7, 8, 9, 31, 255, 256, 257, 4096, 4103, 5, 20011]
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
GAP = 77.0


def _quantise(x, root):
    """Blocks of 256 from the tensor's start: (e4m3 numbers as floats, scales)."""
    n = x.numel()
    pad = torch.zeros(-(-n // 256) * 256)
    pad[:n] = x
    rows = pad.view(-1, 256)
    top = rows.abs().amax(1, keepdim=True)
    some = top >= 2.0 ** -100
    scale = torch.where(some, top / torch.tensor(448.0), torch.zeros(()))
    inv = torch.where(some, torch.tensor(448.0) / top, torch.zeros(()))
    t = rows * inv
    if root:
        t = torch.where(rows > 0, t.clamp(min=2.0 ** -9), t)
    return t.to(torch.float8_e4m3fn).float().view(-1)[:n], scale.view(-1)


def _values(q, scale):
    return q * scale.repeat_interleave(256)[:q.numel()]


def _step_fp32(p, g, m, v, t, lr, wd, scale):
    """The documented sequence; torch's fp32 operations on the CPU round each by itself."""
    f = lambda x: torch.tensor(float(np.float32(x)))
    pow1, pow2 = B1 ** (t - 1) * B1, B2 ** (t - 1) * B2
    g = g.float() * scale
    m = m * f(B1) + g * f(1 - B1)
    v = v * f(B2) + (g * g) * f(1 - B2)
    root = torch.from_numpy(np.sqrt(v.numpy()))         # correctly rounded, which torch does not promise on the CPU
    rate, spread = f(lr * (1.0 / (1.0 - pow1))), f(1.0 / math.sqrt(1.0 - pow2))
    p = p * f(1.0 - lr * wd) - (m * rate) / (root * spread + f(EPS))
    return p, m, v, root


class Tensors:
    """Lists of tensors laid out in flat buffers with gaps that must not change."""

    def __init__(self, sizes, bits, grad, copy, shifts, seed):
        rng = np.random.default_rng(seed)
        dev = "cuda"
        self.sizes, self.flats = sizes, []

        def lay(dtype, make, shift, per=1):
            first, at = [], 32 + shift
            for s in sizes:
                first.append(at)
                c = -(-s // per)
                at += c + (1 if per == 1 and shifts == "packed" else 32 - c % 32 + 32)
            flat = torch.full((at + 64,), GAP, dtype=torch.float32).to(dtype)
            for f, s in zip(first, sizes):
                if s:
                    flat[f:f + -(-s // per)] = make(s)
            flat = flat.to(dev)
            self.flats.append((flat, [(f, f + -(-s // per)) for f, s in zip(first, sizes)]))
            return [flat[f:f + -(-s // per)] for f, s in zip(first, sizes)]

        normal = lambda scale: lambda s: torch.from_numpy(rng.standard_normal(s).astype(np.float32) * scale
                                                          * 10.0 ** rng.uniform(-3, 0.5, s).astype(np.float32))
        off = {"same": (0, 0, 0, 0, 0), "packed": (0,) * 5, "apart": (1, 3, 2, 5, 7)}[shifts]
        self.p = lay(torch.float32, normal(1.0), off[0])
        self.g = lay(TYPES[grad], lambda s: normal(0.1)(s).to(TYPES[grad]), off[1])
        self.copies = None
        if copy:
            self.copies = [c if i % 4 != 3 else None
                           for i, c in enumerate(lay(TYPES[copy], lambda s: torch.zeros(s), off[4]))]
        m = [normal(0.01)(s) for s in sizes]
        v = [normal(0.02)(s) ** 2 for s in sizes]
        if bits == 32:
            self.ref = [(a.clone(), b.clone()) for a, b in zip(m, v)]
            it = iter(m), iter(v)
            live = [x for x in m if x.numel()], [x for x in v if x.numel()]
            it = iter(live[0]), iter(live[1])
            self.moments = (lay(torch.float32, lambda s: next(it[0]), off[2]),
                            lay(torch.float32, lambda s: next(it[1]), off[3]))
        else:
            qm = [_quantise(a, False) for a in m]
            qr = [_quantise(b.sqrt(), True) for b in v]
            self.ref = list(zip(qm, qr))
            four = []
            for pairs, k, o in ((qm, 0, off[2]), (qm, 1, 0), (qr, 0, off[3]), (qr, 1, 0)):
                it = iter([x[k] for x in pairs if x[k].numel()])
                four.append(lay(torch.float8_e4m3fn if k == 0 else torch.float32,
                                lambda s, it=it, k=k: next(it).to(torch.float8_e4m3fn) if k == 0 else next(it),
                                o, 1 if k == 0 else 256))
            self.moments = tuple(four)

    def check_gaps(self):
        for flat, spans in self.flats:
            keep = torch.ones(flat.numel(), dtype=torch.bool)
            for a, b in spans:
                keep[a:b] = False
            gap = torch.tensor(GAP).to(flat.dtype).float()
            assert bool((flat.float().cpu()[keep] == gap).all()), "wrote between the tensors"


def _same(got, want, what):
    got, want = got.detach().float().cpu(), want.float()
    ok = (got == want) | (got.isnan() & want.isnan())
    assert bool(ok.all()), (what, int((~ok).sum()), got[~ok][:4], want[~ok][:4])


@pytest.mark.parametrize("shifts", ["same", "packed", "apart"])
@pytest.mark.parametrize("bits,grad,copy", [(32, "f32", None), (32, "bf16", "bf16"), (32, "f16", "bf16"),
                                            (32, "f32", "f16"), (8, "f32", None), (8, "bf16", "bf16"),
                                            (8, "f16", "f16"), (8, "f32", "bf16"), (8, "bf16", None)])
def test_adamw_same_bits_as_the_documented_sequence(bits, grad, copy, shifts):
    gpu_util.ensure_library()
    x = Tensors(SIZES, bits, grad, copy, shifts, seed=len(shifts) + bits)
    wd = [0.1 if i % 3 else 0.0 for i in range(len(SIZES))]
    opt = training.AdamW(x.p, x.g, bits=bits, moments=x.moments, copies=x.copies, betas=(B1, B2), eps=EPS,
                         weight_decay=wd, steps_done=6)
    scale = torch.tensor(0.37, device="cuda")
    p = [t.cpu() for t in x.p]
    g = [t.cpu() for t in x.g]
    for t, lr in ((7, 1e-3), (8, 3e-3), (9, 0.0)):
        opt.step(lr, scale)
        for i in range(len(SIZES)):
            if SIZES[i] == 0:
                continue
            if bits == 32:
                m, v = x.ref[i]
            else:
                m = _values(*x.ref[i][0])
                v = _values(*x.ref[i][1])
                v = v * v
            p[i], m, v, root = _step_fp32(p[i], g[i], m, v, t, lr, wd[i], scale.cpu())
            x.ref[i] = (m, v) if bits == 32 else (_quantise(m, False), _quantise(root, True))
            _same(x.p[i], p[i], ("p", i, t))
            if bits == 32:
                _same(x.moments[0][i], m, ("m", i, t))
                _same(x.moments[1][i], v, ("v", i, t))
            else:
                for k, want in enumerate((*x.ref[i][0], *x.ref[i][1])):
                    _same(x.moments[k][i], want, ("moment", k, i, t))
            if x.copies is not None and x.copies[i] is not None:
                _same(x.copies[i], p[i].to(TYPES[copy]), ("copy", i, t))
    if copy is not None:                           # an element without a copy keeps its gap
        for flat, spans in x.flats:
            if flat.dtype == TYPES[copy] and copy != grad:
                assert bool((flat[spans[3][0]:spans[3][1]] == 0).all())
    x.check_gaps()
    assert opt.steps == 9 and opt.launches == 3
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_against_the_formula_in_64_bits(bits):
    n, t, lr, wd = 50_021, 4, 2e-3, 0.05
    x = Tensors([n], bits, "f32", None, "same", seed=3)
    if bits == 32:
        m, v = (a.double() for a in x.ref[0])
    else:
        m = x.ref[0][0][0].double() * x.ref[0][0][1].double().repeat_interleave(256)[:n]
        v = (x.ref[0][1][0].double() * x.ref[0][1][1].double().repeat_interleave(256)[:n]) ** 2
    p, g = x.p[0].cpu().double(), x.g[0].cpu().double()
    opt = training.AdamW(x.p, x.g, bits=bits, moments=x.moments, betas=(B1, B2), eps=EPS, weight_decay=wd, steps_done=t - 1)
    opt.step(lr)
    opt.close()
    m1, v1 = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
    step = lr * (m1 / (1 - B1 ** t)) / ((v1 / (1 - B2 ** t)).sqrt() + EPS)
    p1 = p * (1 - lr * wd) - step
    m_terms = B1 * m.abs() + (1 - B1) * g.abs()
    deeper = 2 if bits == 8 else 0                 # value = number * scale, v = r * r: further roundings
    at_m = (4 + deeper) * U * m_terms
    step_err = step.abs() * (8 + 3 * deeper) * U + lr / (1 - B1 ** t) * at_m / ((v1 / (1 - B2 ** t)).sqrt() + EPS)
    got = x.p[0].double().cpu()
    assert bool(((got - p1).abs() <= 3 * U * p.abs() + step_err + 1e-30).all())
    if bits == 32:
        assert bool(((x.moments[0][0].double().cpu() - m1).abs() <= at_m + 1e-38).all())
        assert bool(((x.moments[1][0].double().cpu() - v1).abs() <= 6 * U * v1 + 1e-37).all())
    else:
        for k, want in ((0, m1), (2, v1.sqrt())):
            q, s = x.moments[k][0].double().cpu(), x.moments[k + 1][0].double().cpu().repeat_interleave(256)[:n]
            # three fraction bits: half a step is 2^-4 of the value, at the least half of 2^-9; a root may be lifted by one
            tol = torch.maximum(want.abs() * 2.0 ** -4, s * 2.0 ** (-10 if k == 0 else -9)) * (1 + 1e-4)
            assert bool(((q * s - want).abs() <= tol).all()), k
        assert bool((x.moments[2][0].float().cpu()[v1 > 0] > 0).all())


def test_adamw8_blocks_of_nothing_and_spoilt_blocks():
    n = 1024
    p, g = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda")
    g[256:512] = 1e-35                              # m is below 2^-100: kept as nothing
    g[512 + 9] = float("nan")
    g[768 + 3] = float("inf")
    opt = training.AdamW([p], [g], bits=8, weight_decay=0.0)
    opt.step(1e-3)
    m, ms, r, rs = (x[0].float().cpu() for x in opt.moments)
    assert ms[0] == 0 and rs[0] == 0 and bool((m[:256] == 0).all()) and bool((r[:256] == 0).all())
    assert ms[1] == 0 and bool((m[256:512] == 0).all())
    pc = p.cpu()
    assert bool((pc[:256] == 1).all())
    assert math.isnan(pc[512 + 9]) and bool((pc[512:521] == 1).all()) and bool((pc[522:768] == 1).all())
    assert math.isnan(m[512 + 9]) or ms[2] != ms[2] or ms[2] == 0
    opt.close()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_adamw_skips_on_a_scale_that_is_not_finite(bad):
    x = Tensors(SIZES, 8, "bf16", "bf16", "same", seed=5)
    before = [flat.clone() for flat, _ in x.flats]
    opt = training.AdamW(x.p, x.g, bits=8, moments=x.moments, copies=x.copies, steps_done=11)
    opt.step(1e-3, torch.tensor(bad, device="cuda"))
    assert opt.steps == 11
    for b, (flat, _) in zip(before, x.flats):
        assert torch.equal(b.view(torch.uint8), flat.view(torch.uint8))
    opt.step(1e-3, torch.tensor(1.0, device="cuda"))
    assert opt.steps == 12
    opt.close()


def test_adamw_graph_replay_other_stream_and_new_gradients():
    torch.manual_seed(0)
    n = 70_001
    p0, ga, gb = torch.randn(n, device="cuda"), torch.randn(n, device="cuda"), torch.randn(n + 1, device="cuda")[1:]
    want = p0.clone()
    opt = training.AdamW([want], [ga])
    for k in range(6):
        opt.set_grads([ga if k < 3 else gb])
        opt.step(1e-2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = p0.clone()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        opt2 = training.AdamW([got], [ga])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            opt2.step(1e-2)
        for _ in range(3):
            graph.replay()
        opt2.set_grads([gb])
        for _ in range(3):
            graph.replay()
    torch.cuda.synchronize()
    assert opt2.steps == 6
    assert torch.equal(got, want) and torch.equal(opt.moments[1][0], opt2.moments[1][0])
    del graph
    opt.close(), opt2.close()


def test_adamw_and_norm_follow_the_current_stream():
    torch.manual_seed(1)
    n = 300_007
    p0, g = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    want, got = p0.clone(), p0.clone()
    a, b, gn = training.AdamW([want], [g]), training.AdamW([got], [g]), training.GradNorm([g])
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for k in range(9):
        a.step(1e-2, gn.norm(1.0)[1])
    torch.cuda.synchronize()
    norms = []
    for k in range(9):
        with torch.cuda.stream(streams[k % 3]):
            norm, factor = gn.norm(1.0)
            norms.append(norm)
            b.step(1e-2, factor)
    torch.cuda.synchronize()
    assert torch.equal(want, got) and len({float(x) for x in norms}) == 1
    a.close(), b.close(), gn.close()


def test_adamw_many_tensors_and_past_32_bits():
    # 3,000 tensors of odd sizes, then one whose byte offsets pass 2^32
    sizes = [1 + (i * 37) % 301 for i in range(3000)]
    flat = torch.zeros(sum(sizes), device="cuda")
    grads = torch.randn(sum(sizes), device="cuda")
    at = np.concatenate([[0], np.cumsum(sizes)])
    cut = lambda f: [f[a:b] for a, b in zip(at[:-1], at[1:])]
    whole = torch.zeros_like(flat)
    one, many = training.AdamW([whole], [grads]), training.AdamW(cut(flat), cut(grads))
    for _ in range(2):
        one.step(1e-2), many.step(1e-2)
    assert torch.equal(flat, whole)
    one.close(), many.close()
    n = 2 ** 30 + 4099
    p = torch.zeros(n, device="cuda")
    g = torch.zeros(n, device="cuda", dtype=torch.float16)
    g[-5000:] = 0.25
    opt = training.AdamW([p], [g], bits=8, weight_decay=0.0)
    opt.step(1e-2)
    assert bool((p[-5000:] < -0.0099).all()) and int((p != 0).sum()) == 5000
    opt.close()


def test_adamw_refusals():
    p, g = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    bad = [
        lambda: training.AdamW([], []),
        lambda: training.AdamW([p.cpu()], [g]),
        lambda: training.AdamW([p.half()], [g]),
        lambda: training.AdamW([p], [g[:63]]),
        lambda: training.AdamW([p], [g, g]),
        lambda: training.AdamW([p, p], [g, g.half()]),
        lambda: training.AdamW([p.view(8, 8).t()], [g]),
        lambda: training.AdamW([p], [g], bits=16),
        lambda: training.AdamW([p], [g], betas=(1.0, 0.9)),
        lambda: training.AdamW([p], [g], betas=(0.9, -0.1)),
        lambda: training.AdamW([p], [g], eps=-1.0),
        lambda: training.AdamW([p], [g], eps=float("nan")),
        lambda: training.AdamW([p], [g], steps_done=-1),
        lambda: training.AdamW([p], [g], weight_decay=float("inf")),
        lambda: training.AdamW([p], [g], weight_decay=[0.1, 0.1]),
        lambda: training.AdamW([p], [g], moments=([p],)),
        lambda: training.AdamW([p], [g], copies=[torch.zeros(64, device="cuda")]),
        lambda: training.AdamW([p], [g], bits=8, moments=([p], [p], [p], [p])),
    ]
    for k, f in enumerate(bad):
        with pytest.raises(binding.PsopsError) as e:
            f()
        assert e.value.code == binding.PSOPS_EINVAL, k
    opt = training.AdamW([p], [g])
    for f in (lambda: opt.step(float("nan")), lambda: opt.step(1e-3, 2.0), lambda: opt.step(1e-3, torch.tensor(1.0)),
              lambda: opt.set_grads([g.half()]), lambda: opt.set_grads([g[1:]])):
        with pytest.raises(binding.PsopsError) as e:
            f()
        assert e.value.code == binding.PSOPS_EINVAL
    opt.close()
    cfg = binding.psops_adamw_config(0.9, 0.999, 1e-8, 0, 32, binding.PSOPS_F32, binding.PSOPS_NONE, 1)
    t = (binding.psops_adamw_tensor * 1)()
    t[0] = binding.psops_adamw_tensor(p.data_ptr() + 2, g.data_ptr(), None, p.data_ptr(), p.data_ptr(), None, None, 60, 0.0)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    with pytest.raises(binding.PsopsError) as e:
        binding.psops_adamw_create(cfg, t, ws)
    assert e.value.code == binding.PSOPS_EALIGN
    t[0].p = p.data_ptr()
    with pytest.raises(binding.PsopsError) as e:
        binding.psops_adamw_create(cfg, t, ws, 16)
    assert e.value.code == binding.PSOPS_EWORKSPACE


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("packed", [True, False])
def test_gradnorm(kind, packed):
    rng = np.random.default_rng(9)
    sizes = SIZES + [70_003]
    at, first = 3, []
    for s in sizes:
        first.append(at)
        at += s + (0 if packed else 64 - s % 64)
    host = torch.from_numpy(rng.standard_normal(at + 9).astype(np.float32) * 10.0 ** rng.uniform(-4, 1, at + 9)).to(TYPES[kind])
    flat = host.cuda()
    grads = [flat[f:f + s] for f, s in zip(first, sizes)]
    want = math.sqrt(sum(float((host[f:f + s].double() ** 2).sum()) for f, s in zip(first, sizes)))
    gn = training.GradNorm(grads)
    norm, factor = gn.norm(1.0)
    # 16 squares in fp32 (one rounding each with fma), the rest in double, the root rounded: < 16 u of the sum
    assert abs(float(norm) - want) <= (8 + 2) * U * want
    assert float(factor) == float(np.float32(1.0) / (np.float32(float(norm)) + np.float32(1e-6))) and float(factor) < 1
    again, free = gn.norm(math.inf)
    assert float(again) == float(norm) and float(free) == 1.0
    assert float(gn.norm(2 * want)[1]) == 1.0 and float(gn.norm(0.0)[1]) == 0.0
    gn.set_grads([g.clone() for g in grads])
    assert float(gn.norm(1.0)[0]) == pytest.approx(want, rel=20 * U)
    for bad in (float("nan"), float("inf")):
        grads2 = [g.clone() for g in grads]
        grads2[-1][12_345] = bad
        gn.set_grads(grads2)
        norm, factor = gn.norm(1.0)
        assert not math.isfinite(float(norm)) and math.isnan(float(factor))
    gn.set_grads([torch.zeros_like(g) for g in grads])
    norm, factor = gn.norm(1.0)
    assert float(norm) == 0.0 and float(factor) == 1.0
    gn.close()


def test_gradnorm_empty_one_and_refusals():
    e = torch.zeros(0, device="cuda")
    gn = training.GradNorm([e, e])
    assert float(gn.norm(1.0)[0]) == 0.0
    gn.close()
    gn = training.GradNorm([torch.tensor([-3.0], device="cuda")])
    assert float(gn.norm(1.0)[0]) == 3.0
    for f in (lambda: gn.norm(-1.0), lambda: gn.norm(float("nan")), lambda: gn.norm(1.0, torch.zeros(2)),
              lambda: gn.set_grads([e]), lambda: training.GradNorm([]), lambda: training.GradNorm([torch.zeros(3)]),
              lambda: training.GradNorm([torch.zeros(3, device="cuda", dtype=torch.int32)])):
        with pytest.raises(binding.PsopsError) as err:
            f()
        assert err.value.code == binding.PSOPS_EINVAL
    gn.close()


def test_clipped_step_is_skipped_when_a_gradient_is_not_finite():
    p = torch.ones(5000, device="cuda")
    g = torch.full((5000,), 0.1, device="cuda")
    opt, gn = training.AdamW([p], [g]), training.GradNorm([g])
    opt.step(1e-3, gn.norm(1.0)[1])
    after = p.clone()
    g[77] = float("inf")
    opt.step(1e-3, gn.norm(1.0)[1])
    assert torch.equal(p, after) and opt.steps == 1
    g[77] = 0.1
    opt.step(1e-3, gn.norm(1.0)[1])
    assert not torch.equal(p, after) and opt.steps == 2
    opt.close(), gn.close()
