"""Attention where it can go wrong: what lies in masked places, biases that mask, strides, given results, streams and
graphs, large offsets, long sums; refusals of the C entries; the differentiable form."""
import math

import pytest
import torch

from attention_util import compare, inputs, lengths_to_offsets, reference
from paper_2009_03816_b200 import binding, training
from paper_2009_03816_b200 import build as _build

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
NAMES = ("out", "lse", "dq", "dk", "dv")


@pytest.fixture(scope="module", autouse=True)
def _library():
    _build.build_library()


def both(op, x, offsets, **kw):
    """Results of both passes by name."""
    bias = x.get("bias")
    out, lse = op.forward(x["q"], x["k"], x["v"], offsets, bias)
    dq, dk, dv, dbias = op.backward(x["q"], x["k"], x["v"], offsets, out, lse, x["grad"], bias)
    return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv, **({"dbias": dbias} if bias is not None else {}))


def make(lengths, heads=2, kv_heads=1, dim=64, dtype=BF16, first=0, rest=0, buckets=None, seed=0, **kw):
    T = first + sum(lengths) + rest
    x = inputs(T, heads, kv_heads, dim, dtype, seed, True, buckets)
    op = training.Attention(T, max(1, len(lengths)), heads, kv_heads, dim, dtype=dtype, buckets=buckets, **kw)
    return op, x, lengths_to_offsets(lengths, first)


def same(a, b, rows=slice(None)):
    for name in a:
        p, q = (a[name][:, rows], b[name][:, rows]) if name == "lse" else (a[name][rows], b[name][rows])
        if name != "dbias":
            assert torch.equal(p, q), name


# ---- masked places -----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("dim", [64, 80])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_other_sequences_and_rows_of_none_reach_nothing(what, dim, dtype):
    lengths, first, rest = [70, 130, 200], 20, 60
    op, x, offsets = make(lengths, 2, 1, dim, dtype, first, rest, buckets=[0, 1, 2, 8])
    clean = both(op, x, offsets)
    for lo, hi in ((0, 20), (420, 480), (90, 220)):          # in front, behind, the middle sequence
        y = {k: v.clone() if k != "bias" else v for k, v in x.items()}
        for name in ("q", "k", "v", "grad"):
            y[name][lo:hi] = what
        got = both(op, y, offsets)
        for a, b in ((20, 90), (90, 220), (220, 420)):
            if (a, b) != (lo, hi):
                # ds of fp16 is scaled by what is finite of do and v: other rows' norms may move it by a power of two
                same(got, clean, slice(a, b)) if dtype == BF16 else [
                    torch.testing.assert_close(got[n][a:b], clean[n][a:b], rtol=2e-2, atol=2e-3) for n in ("out", "dq", "dk", "dv")]
        if (lo, hi) == (90, 220):
            assert not torch.isfinite(got["out"][90:220]).any()
        else:
            assert torch.isfinite(got["dbias"]).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("at", [0, 37, 127, 128, 200, 299])
@pytest.mark.parametrize("name", ["k", "v"])
def test_later_tokens_reach_nothing(name, at, dim):
    op, x, offsets = make([300], 2, 1, dim, BF16)
    clean = both(op, x, offsets)
    y = {k: v.clone() for k, v in x.items()}
    y[name][at, 0, 3] = math.inf if name == "v" else math.nan
    got = both(op, y, offsets)
    # rows before `at` see none of it, forward and in dq; rows from `at` on do
    assert torch.equal(got["out"][:at], clean["out"][:at]) and torch.equal(got["lse"][:, :at], clean["lse"][:, :at])
    assert torch.equal(got["dq"][:at], clean["dq"][:at])
    if name == "v":
        assert (got["out"][at:, :, 3] == math.inf).all() and torch.equal(got["out"][at:, :, :3], clean["out"][at:, :, :3])
    else:
        assert got["out"][at:].isnan().all() and got["lse"][:, at:].isnan().all()
    assert not torch.isfinite(got["dq"][at:]).all(-1).any()


@pytest.mark.parametrize("at", [0, 64, 128, 255, 299])
def test_earlier_keys_see_none_of_an_earlier_gradient(at):
    """do of token `at` reaches dk and dv of keys up to it, none behind it."""
    op, x, offsets = make([300], 2, 1, 64, BF16)
    clean = both(op, x, offsets)
    y = {k: v.clone() for k, v in x.items()}
    y["grad"][at, 1, 7] = math.inf
    got = both(op, y, offsets)
    for name in ("dk", "dv"):
        assert torch.equal(got[name][at + 1:], clean[name][at + 1:]), name
    assert not torch.isfinite(got["dv"][:at + 1, :, 7]).any()
    assert torch.equal(got["dq"][:at], clean["dq"][:at]) and torch.equal(got["dq"][at + 1:], clean["dq"][at + 1:])


@pytest.mark.parametrize("lowest", [-math.inf, torch.finfo(torch.float32).min, -1e31])
def test_biases_that_mask(lowest):
    """Distances of a masked bucket count for nothing; a row with none left is zeros with lse -inf."""
    buckets = [0, 1, 40, 200]
    op, x, offsets = make([500, 30], 2, 2, 64, BF16, buckets=buckets)
    x["bias"] = x["bias"].float()
    op2 = training.Attention(530, 2, 2, 2, 64, buckets=buckets)
    x["bias"][2] = lowest                                          # distances 40 to 199
    y = dict(x, bias=x["bias"].clone())
    y["bias"][2] = -math.inf
    got = both(op2, x, offsets)
    compare(got, reference(x["q"], x["k"], x["v"], [500, 30], 0, x["grad"], y["bias"], buckets))
    assert not got["dbias"][2].any()
    y["bias"][:, 0] = lowest                                       # all of one head
    got = both(op, y, offsets)
    assert not got["out"][:, 0].any() and (got["lse"][0] == -math.inf).all()
    assert not got["dq"][:, 0].any() and not got["dk"][:, 0].any() and not got["dv"][:, 0].any() and not got["dbias"][:, 0].any()
    assert torch.isfinite(got["out"]).all() and torch.isfinite(got["dk"]).all()
    y["bias"][1:, 1] = lowest                                      # the token itself alone
    got = both(op, y, offsets)
    assert torch.equal(got["out"][:, 1], x["v"][:, 1])


def test_empty_calls():
    op = training.Attention(50, 4, 2, 1, 16, buckets=[0, 3])
    x = inputs(40, 2, 1, 16, BF16, buckets=[0, 3])
    for offsets in (torch.tensor([0], dtype=torch.int32, device="cuda"), lengths_to_offsets([0, 0, 0], 7)):
        got = both(op, x, offsets)
        for name, t in got.items():
            assert not t.any(), name
    y = {k: v[:0] if k != "bias" else v for k, v in x.items()}
    got = both(op, y, lengths_to_offsets([0, 0]))
    assert got["out"].shape == (0, 2, 16) and got["lse"].shape == (2, 0) and not got["dbias"].any()


def test_offsets_out_of_order_stay_in_bounds():
    """Whatever the offsets hold, nothing outside the tensors is touched and the call ends."""
    room = torch.full((300 * 64 + 200,), 7.0, dtype=BF16, device="cuda")
    op = training.Attention(100, 6, 3, 3, 64)
    x = inputs(100, 3, 3, 64, BF16)
    out = room[104:104 + 300 * 64].view(100, 3, 64)
    for bad in ([5, 90, 10, 100, 0, 100, 100], [-50, 30, 1000, 2 ** 31 - 1, -2 ** 31, 60, 80], [100, 0, 100, 0, 100, 0, 100]):
        offsets = torch.tensor(bad, dtype=torch.int32, device="cuda")
        _, lse = op.forward(x["q"], x["k"], x["v"], offsets, out=out)
        op.backward(x["q"], x["k"], x["v"], offsets, out, lse, x["grad"])
        torch.cuda.synchronize()
        assert (room[:104] == 7.0).all() and (room[104 + 300 * 64:] == 7.0).all()
    # and the holder still works
    offsets = lengths_to_offsets([60, 40])
    compare(both(op, x, offsets), reference(x["q"], x["k"], x["v"], [60, 40], 0, x["grad"]))


# ---- layouts ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_layouts(dtype):
    """Head-major tensors, gaps between rows, given results in views of one buffer; the same bits each time."""
    lengths, H, G, D = [150, 90], 4, 2, 40
    op, x, offsets = make(lengths, H, G, D, dtype, first=5, rest=9)
    want = both(op, x, offsets)
    T = 254
    head_major = {n: t.transpose(0, 1).contiguous().transpose(0, 1) for n, t in x.items()}
    assert head_major["q"].stride() == (D, T * D, 1)
    for name, t in both(op, head_major, offsets).items():
        assert torch.equal(t, want[name]), name
    wide = {}
    for n, t in x.items():
        room = torch.full((T, t.shape[1] + 1, D + 8), math.nan, dtype=dtype, device="cuda")
        room[:, :t.shape[1], :D] = t
        wide[n] = room[:, :t.shape[1], :D]
    for name, t in both(op, wide, offsets).items():
        assert torch.equal(t, want[name]), name
    joint = torch.full((T, H + 2 * G, D), 3.0, dtype=dtype, device="cuda")
    dq, dk, dv = joint[:, :H], joint[:, H:H + G], joint[:, H + G:]
    op.backward(x["q"], x["k"], x["v"], offsets, want["out"], want["lse"], x["grad"], dq=dq, dk=dk, dv=dv)
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        assert torch.equal(t[5:245], want[name][5:245])
    assert (joint[:5] == 3.0).all() and (joint[245:] == 3.0).all()                # rows of no sequence as they were
    out = torch.full((H, T, D), 3.0, dtype=dtype, device="cuda").transpose(0, 1)
    op.forward(x["q"], x["k"], x["v"], offsets, out=out)
    assert torch.equal(out[5:245], want["out"][5:245]) and (out[:5] == 3.0).all() and (out[245:] == 3.0).all()


def test_what_is_wanted():
    op, x, offsets = make([200], 2, 2, 64, BF16, buckets=[0, 2, 50])
    want = both(op, x, offsets)
    for wanted in ((True, False, False, False), (False, True, False, False), (False, False, True, False), (False, False, False, True),
                   (True, False, True, False), (False, False, False, False)):
        got = op.backward(x["q"], x["k"], x["v"], offsets, want["out"], want["lse"], x["grad"], x["bias"], want=wanted)
        for name, t, w in zip(("dq", "dk", "dv", "dbias"), got, wanted):
            assert torch.equal(t, want[name]) if w else t is None


def test_the_same_bits_again():
    lengths = [300, 5, 128, 77, 600, 1, 1, 250]
    op, x, offsets = make(lengths, 4, 2, 128, BF16, buckets=training.distance_buckets(16, 100))
    want = both(op, x, offsets)
    for _ in range(5):
        for name, t in both(op, x, offsets).items():
            assert torch.equal(t, want[name]), name
    # nor does it matter what else is in the batch: the sequence of 600 alone
    at = sum(lengths[:4])
    rows = slice(at, at + 600)
    alone = training.Attention(600, 1, 4, 2, 128, buckets=training.distance_buckets(16, 100))
    y = {n: t[rows] if n != "bias" else t for n, t in x.items()}
    got = both(alone, y, lengths_to_offsets([600]))
    for name in ("out", "dq", "dk", "dv"):
        assert torch.equal(got[name], want[name][rows]), name


@pytest.mark.parametrize("case", ["many short", "one long", "few sums", "many sums"])
def test_lists_of_tiles(case):
    """The list's kernel and the search without it; dbias joined within and by a kernel of its own."""
    buckets = [0, 1, 2, 30]
    lengths = {"many short": [1 + i % 5 for i in range(1500)], "one long": [5000], "few sums": [100, 40], "many sums": [129] * 60}[case]
    op, x, offsets = make(lengths, 1 if case != "few sums" else 2, 1, 32, BF16, buckets=buckets)
    compare(both(op, x, offsets), reference(x["q"], x["k"], x["v"], lengths, 0, x["grad"], x["bias"], buckets), case)


@pytest.mark.parametrize("kv_heads", [1, 2])
def test_sums_of_more_terms_than_go_at_a_time(kv_heads):
    """A row of 17,000 keys and keys of 34,000 queries, all numbers of one sign: cut-off sums must not add up."""
    T = 17000
    x = inputs(T, 2, kv_heads, 32, F16)
    x = {n: (t.abs() + 0.5).contiguous() if n in ("v", "grad") else (t * 0.1).contiguous() for n, t in x.items()}
    op = training.Attention(T, 1, 2, kv_heads, 32, dtype=F16)
    got = both(op, x, lengths_to_offsets([T]))
    want = reference(x["q"], x["k"], x["v"], [T], 0, x["grad"])
    compare(got, want)
    # 16,384 terms are 1,024 cut sums, each off by 2^-23 of the sum at most; half of that on average, and results are rounded
    for name in ("out", "dv"):
        exact = want[name][0]
        bias = float(((got[name].double() - exact) * exact).sum() / (exact * exact).sum())
        assert abs(bias) < 1024 * 2.0 ** -23 + 2.0 ** -13, (name, bias)


def test_offsets_beyond_32_bits():
    """More than 2^31 elements of q: the last sequences of a large batch."""
    T, H = 140_000, 128
    lengths = [100] * 1400
    q = torch.empty(T, H, 128, dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    assert q.numel() > 2 ** 31
    k, v = q[:, :1].clone(), q[:, 1:2].clone()
    grad = torch.empty_like(q).normal_()
    op = training.Attention(T, 1400, H, 1, 128)
    offsets = lengths_to_offsets(lengths)
    out, lse = op.forward(q, k, v, offsets)
    dq, dk, dv, _ = op.backward(q, k, v, offsets, out, lse, grad)
    rows = slice(T - 200, T)
    want = reference(q[rows], k[rows], v[rows], [100, 100], 0, grad[rows])
    compare(dict(out=out[rows], lse=lse[:, rows], dq=dq[rows], dk=dk[rows], dv=dv[rows]), want)


# ---- streams, graphs, the context ------------------------------------------------------------------------

def test_streams_and_graphs():
    lengths = [300, 40, 128]
    op, x, offsets = make(lengths, 2, 1, 64, BF16, buckets=[0, 1, 60])
    want = both(op, x, offsets)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, torch.cuda.current_stream(), side):
        with torch.cuda.stream(stream):
            got = both(op, x, offsets)
        stream.synchronize()
        for name, t in got.items():
            assert torch.equal(t, want[name]), name
    y = {n: t.clone() for n, t in x.items()}
    lengths_held = offsets.clone()
    with torch.cuda.stream(side):
        both(op, y, lengths_held)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held = both(op, y, lengths_held)
    for seed, other in ((1, [300, 40, 128]), (2, [1, 467, 0]), (3, [200, 200, 60])):
        z = inputs(468, 2, 1, 64, BF16, seed, True, [0, 1, 60])
        for n in y:
            y[n].copy_(z[n])
        lengths_held.copy_(lengths_to_offsets(other))
        graph.replay()
        torch.cuda.synchronize()
        eager = training.Attention(468, 3, 2, 1, 64, buckets=[0, 1, 60])
        for name, t in both(eager, z, lengths_to_offsets(other)).items():
            rows = slice(0, sum(other))
            assert torch.equal(t, held[name]), (seed, name)
    # a captured backward pass while an eager graph of the same leaves lives
    leaves = [t.clone().requires_grad_() for t in (x["q"], x["k"], x["v"])]
    alive = op(*leaves, offsets, x["bias"])
    with torch.cuda.stream(side):
        op(*leaves, offsets, x["bias"]).backward(x["grad"])
    side.synchronize()
    graph2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph2, stream=side):
        captured = both(op, x, offsets)
    graph2.replay()
    torch.cuda.synchronize()
    for name, t in captured.items():
        assert torch.equal(t, want[name]), name
    alive.backward(x["grad"])
    torch.cuda.synchronize()


def test_a_stream_of_its_own():
    side = torch.cuda.Stream()
    op, x, offsets = make([300, 40], 2, 1, 64, BF16, stream=side.cuda_stream)
    plain, _, _ = make([300, 40], 2, 1, 64, BF16)
    want = both(plain, x, offsets)
    leaves = [t.clone().requires_grad_() for t in (x["q"], x["k"], x["v"])]
    out = op(*leaves, offsets)                           # the differentiable call's results are the current stream's
    out.backward(x["grad"])
    for name, t in (("out", out), ("dq", leaves[0].grad), ("dk", leaves[1].grad), ("dv", leaves[2].grad)):
        assert torch.equal(t, want[name]), name


def test_creation_inside_a_capture_is_refused():
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        for make_one in (lambda: training.Attention(10, 1, 1, 1, 8), lambda: training.Keep8()):
            with pytest.raises(binding.PsopsError) as e:
                make_one()
            assert e.value.code == binding.PSOPS_ESTATE


def test_refusals_of_the_entries():
    lib = binding.load()
    op = training.Attention(64, 2, 4, 2, 16, buckets=[0, 5])
    plain = training.Attention(64, 2, 4, 2, 16, gradients=False)
    x = inputs(64, 4, 2, 16, BF16, buckets=[0, 5])
    offsets = lengths_to_offsets([60, 4])
    h = lambda t, a=None, b=None, off=0: binding.psops_heads(t.data_ptr() + off, t.stride(0) if a is None else a, t.stride(1) if b is None else b)
    q, k, v, out = h(x["q"]), h(x["k"]), h(x["v"]), h(torch.empty(64, 4, 16, dtype=BF16, device="cuda"))
    lse = torch.zeros(4, 64, device="cuda")
    bias, kind = x["bias"].data_ptr(), binding.PSOPS_BF16
    at = offsets.data_ptr()

    def forward(q=q, k=k, v=v, at=at, n=2, T=64, bias=bias, kind=kind, out=out, lse=lse.data_ptr(), ctx=op.ctx):
        return lib.psops_attention_forward(ctx, q, k, v, at, n, T, bias, kind, out, lse, 0)

    assert forward() == binding.PSOPS_OK
    for kw in (dict(T=65), dict(T=-1), dict(n=3), dict(n=-1), dict(q=None), dict(out=None), dict(at=None), dict(bias=None), dict(kind=F16),
               dict(kind=binding.PSOPS_F16), dict(lse=None), dict(q=h(x["q"], a=8)), dict(q=h(x["q"], b=8)), dict(k=binding.psops_heads(None, 32, 16)),
               dict(out=h(x["q"], a=40, b=16)), dict(v=h(x["v"], a=1 << 39)), dict(ctx=plain.ctx)):
        if kw.get("kind") is F16:
            kw = dict(kind=7)
        assert forward(**kw) == binding.PSOPS_EINVAL, kw
    for kw in (dict(q=h(x["q"], off=2)), dict(q=h(x["q"], a=132)), dict(k=h(x["k"], b=20)), dict(at=at + 2), dict(bias=bias + 1),
               dict(lse=lse.data_ptr() + 2), dict(out=h(x["q"], off=8))):
        assert forward(**kw) == binding.PSOPS_EALIGN, kw
    back = lambda ctx=op.ctx, dq=out, db=None, grad=out: lib.psops_attention_backward(ctx, q, k, v, at, 2, 64, bias if ctx is op.ctx else None, kind, out,
                                                                                      lse.data_ptr(), grad, dq, None, None, db, 0)
    assert back(ctx=plain.ctx) == binding.PSOPS_ESTATE
    assert back(grad=None) == binding.PSOPS_EINVAL
    assert back(dq=h(x["q"], a=40, b=16)) == binding.PSOPS_EINVAL
    assert back(db=lse.data_ptr() + 1) == binding.PSOPS_EALIGN
    torch.cuda.synchronize()
    with pytest.raises(binding.PsopsError) as e:
        training.Attention(64, 2, 4, 2, 12)
    assert e.value.code == binding.PSOPS_EINVAL


# ---- the differentiable form --------------------------------------------------------------------------------

def test_autograd_with_any_strides_and_shared_inputs():
    T, H, D = 200, 4, 24
    gen = torch.Generator(device="cuda").manual_seed(5)
    base = torch.empty(H, D, T, device="cuda").normal_(generator=gen).to(BF16)
    q = base.permute(2, 0, 1).detach().requires_grad_()                       # elements of a head T apart
    kv = torch.empty(T, 1, D, device="cuda").normal_(generator=gen).to(BF16).requires_grad_()
    k = kv.expand(T, 2, D)                                                    # one head broadcast to two: its gradient is their sum
    table = torch.empty(8, 3, device="cuda").normal_(generator=gen).requires_grad_()
    bias = table.T[:, :H]                                                     # a slice of a transposed table
    op = training.Attention(T, 2, H, 2, D, buckets=[0, 4, 20])
    offsets = lengths_to_offsets([120, 80])
    out = op(q, k, kv.expand(T, 2, D), offsets, bias)
    grad = torch.empty(T, H, D, device="cuda").normal_(generator=gen).to(BF16)
    out.backward(grad)
    full = k.detach().contiguous()
    want = reference(q.detach().contiguous(), full, full, [120, 80], 0, grad, bias.detach().contiguous(), [0, 4, 20])
    compare({"out": out.detach(), "dq": q.grad}, want)
    exact = (want["dk"][0] + want["dv"][0]).sum(1, keepdim=True)
    size = (want["dk"][0].abs() + want["dv"][0].abs()).sum(1, keepdim=True)
    bound = (want["dk"][1] + want["dv"][1]).sum(1, keepdim=True)
    # torch adds the heads and the two uses in bf16: three more roundings of sums no larger than `size`
    assert bool(((kv.grad.double() - exact).abs() <= bound + 3 * 2.0 ** -8 * (size + bound)).all())
    assert bool(((table.grad.double()[:4].T - want["dbias"][0]).abs() <= want["dbias"][1] + 2.0 ** -23 * want["dbias"][0].abs()).all())
    assert not table.grad[4:].any()
    # an upstream gradient that is broadcast
    q2 = q.detach().clone().requires_grad_()
    op(q2, full, full, offsets, bias.detach()).sum().backward()
    ones = reference(q2.detach().contiguous(), full, full, [120, 80], 0, torch.ones_like(grad), bias.detach().contiguous(), [0, 4, 20])
    compare({"dq": q2.grad}, ones)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_gradients_against_differences(dtype):
    """d/dt of sum(grad out) along a direction, by differences of the formula in 64 bits, against the kernel's gradients."""
    lengths, buckets = [90, 170], [0, 1, 3, 10, 40]
    op, x, offsets = make(lengths, 4, 2, 40, dtype, buckets=buckets, seed=9)
    got = both(op, x, offsets)
    want = reference(x["q"], x["k"], x["v"], lengths, 0, x["grad"], x["bias"], buckets)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for name, of in (("dq", "q"), ("dk", "k"), ("dv", "v"), ("dbias", "bias")):
        direction = torch.empty(x[of].shape, dtype=torch.float64, device="cuda").normal_(generator=gen)
        def value(t):
            y = {n: v.double() for n, v in x.items()}
            y[of] = y[of] + t * direction
            out = reference64(y, lengths, buckets)
            return float((out * x["grad"].double()).sum())
        step = 1e-4
        slope = (value(step) - value(-step)) / (2 * step)
        mine = float((got[name].double() * direction).sum())
        bound = float((want[name][1] * direction.abs()).sum())
        assert abs(mine - slope) <= bound + 1e-5 * (1 + abs(slope)), (name, mine, slope, bound)


def reference64(y, lengths, buckets):
    out = torch.zeros_like(y["q"])
    at, g = 0, y["q"].shape[1] // y["k"].shape[1]
    for n in lengths:
        r = slice(at, at + n)
        at += n
        d = torch.arange(n, device="cuda")[:, None] - torch.arange(n, device="cuda")
        of = torch.bucketize(d.clamp(min=0), torch.tensor(buckets, device="cuda"), right=True) - 1
        for h in range(out.shape[1]):
            s = y["q"][r, h] @ y["k"][r, h // g].T / y["q"].shape[2] ** 0.5 + y["bias"][:, h][of]
            out[r, h] = torch.softmax(torch.where(d >= 0, s, -math.inf), -1) @ y["v"][r, h // g]
    return out


def test_second_derivatives_raise():
    op, x, offsets = make([20], 1, 1, 16, BF16)
    q = x["q"].detach().contiguous().requires_grad_()
    (dq,) = torch.autograd.grad(op(q, x["k"], x["v"], offsets).float().pow(2).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        dq.float().sum().backward()


def test_given_results_count_as_changes():
    op, x, offsets = make([20], 1, 1, 16, BF16)
    out = torch.zeros(20, 1, 16, dtype=BF16, device="cuda")
    leaf = torch.ones(1, device="cuda", dtype=BF16, requires_grad=True)
    loss = (leaf * out).sum()
    op.forward(x["q"], x["k"], x["v"], offsets, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        loss.backward()


def test_launches_are_counted():
    op, x, offsets = make([100], 1, 1, 16, BF16)
    both(op, x, offsets)
    assert op.launches == 1 + 3                            # a short batch: no list forward; list, queries and keys backward


@pytest.mark.parametrize("heads,kv_heads", [(4, 1), (6, 2), (2, 1)])
@pytest.mark.parametrize("lengths", [[60], [300, 90], [1200]], ids=str)
def test_heads_that_share_keys_alone_or_in_one_work(heads, kv_heads, lengths):
    """Few tiles give each query head a CTA, many one for all that share a key head: the same within their bounds."""
    buckets = training.distance_buckets(8, 40)
    for copies in (1, 40):
        many = lengths * copies
        op, x, offsets = make(many, heads, kv_heads, 64, F16, buckets=buckets, seed=copies)
        got = both(op, x, offsets)
        rows = slice(sum(many) - sum(lengths), sum(many))
        y = {n: t[rows] if n != "bias" else t for n, t in x.items()}
        want = reference(y["q"], y["k"], y["v"], lengths, 0, y["grad"], y["bias"], buckets)
        compare({n: (t[:, rows] if n == "lse" else t[rows]) for n, t in got.items() if n != "dbias"}, want)
        again = both(op, x, offsets)
        for n in got:
            assert torch.equal(got[n], again[n]), n


def test_two_holders_at_once():
    """Two contexts on two streams do not meet."""
    lengths = [200, 500, 33]
    a, x, offsets = make(lengths, 4, 2, 64, BF16, buckets=[0, 3, 50])
    b, y, _ = make(lengths, 4, 2, 64, BF16, buckets=[0, 3, 50], seed=5)
    want_x, want_y = both(a, x, offsets), both(b, y, offsets)
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(s):
            got_x = both(a, x, offsets)
        with torch.cuda.stream(t):
            got_y = both(b, y, offsets)
        torch.cuda.synchronize()
        for n in want_x:
            assert torch.equal(got_x[n], want_x[n]) and torch.equal(got_y[n], want_y[n]), n


def test_a_whole_training_step_in_a_graph():
    """Attention, kept activations, head, clipping and AdamW recorded once and replayed on other batches."""
    T, V, H, D = 96, 200, 2, 16
    gen = torch.Generator(device="cuda").manual_seed(7)
    masters = [torch.empty(*s, device="cuda").normal_(0.0, 0.2, generator=gen) for s in ((V, 32), (32, 96), (4, H), (16, 32), (V, 32))]

    class Step:
        def __init__(self):
            self.p = [m.clone() for m in masters]
            self.copies = [p.to(BF16) for p in self.p]
            self.grads = [torch.zeros_like(c) for c in self.copies]
            self.attention = training.Attention(T, 3, H, 1, D, buckets=[0, 1, 2, 8])
            self.keep, self.xent = training.Keep8(), training.LinearXent(T, 32, V)
            self.opt, self.clip = training.AdamW(self.p, self.grads, copies=self.copies), training.GradNorm(self.grads)
            self.one = torch.ones((), device="cuda")

        def __call__(self, x, y, offsets):
            e, qkv, bias, down, w = self.copies
            de, dqkv, dbias, ddown, dw = self.grads
            h = e[x]
            u = h @ qkv
            p = u[:, :64].view(T, 4, D)
            q, k, v = p[:, :2], p[:, 2:3], p[:, 3:]
            o, lse = self.attention.forward(q, k, v, offsets, bias)
            act, kept = self.keep.activate(u[:, 64:80], u[:, 80:], "silu")
            top = h + o.reshape(T, 32) + act @ down
            _, rows, logs = self.xent.forward(top, w, y)
            dtop, _ = self.xent.backward(top, w, y, logs, self.one, rows=rows, dw=dw)
            du = torch.zeros_like(u)
            dp = du[:, :64].view(T, 4, D)
            self.attention.backward(q, k, v, offsets, o, lse, dtop.view(T, 2, D), bias, dq=dp[:, :2], dk=dp[:, 2:3], dv=dp[:, 3:], dbias=dbias)
            _, _, again = self.keep.activate_backward(kept, dtop @ down.T, "silu", again=True, da=du[:, 64:80], db=du[:, 80:])
            torch.mm(again.T, dtop, out=ddown)
            torch.mm(h.T, du, out=dqkv)
            de.copy_(torch.zeros(V, 32, device="cuda").index_add_(0, x, (dtop + du @ qkv.T).float()))
            _, factor = self.clip.norm(1.0)
            self.opt.step(1e-2, factor)

    def batch(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        return torch.randint(0, V, (T,), device="cuda", generator=g), torch.randint(0, V, (T,), device="cuda", generator=g)

    eager, recorded = Step(), Step()
    offsets = lengths_to_offsets([50, 1, 45])
    x, y = batch(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        recorded(x, y, offsets)
    side.synchronize()
    eager(x, y, offsets)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        recorded(x, y, offsets)
    for seed in (1, 2, 3):
        a, b = batch(seed)
        x.copy_(a), y.copy_(b)
        graph.replay()
        eager(a, b, offsets)
    torch.cuda.synchronize()
    # index_add_ adds in any order: what is not its gradient is the same to a rounding of bf16 and what follows from it
    for p, q, m in zip(eager.p, recorded.p, masters):
        assert float((p - q).norm()) < 0.05 * float((p - m).norm())
    assert recorded.opt.steps == eager.opt.steps == 4


@pytest.mark.parametrize("kv_heads", [1, 4])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
def test_large_numbers_in_rows_of_none_change_nothing(dtype, kv_heads):
    """What lies in front and behind has no part in the scale of ds either."""
    op, x, offsets = make([150, 40], 4, kv_heads, 64, dtype, 90, 110, buckets=[0, 1, 30])
    x["grad"] *= 2.0 ** -10
    clean = both(op, x, offsets)
    compare({n: t[:, 90:280] if n == "lse" else t[90:280] for n, t in clean.items() if n in ("dq", "dk", "dv")},
            reference(x["q"][90:280], x["k"][90:280], x["v"][90:280], [150, 40], 0, x["grad"][90:280], x["bias"], [0, 1, 30]))
    y = {n: t.clone() for n, t in x.items()}
    for n in ("q", "k", "v", "grad"):
        y[n][:90] = y[n][280:] = 65504.0
    got = both(op, y, offsets)
    same(got, clean)
    assert torch.equal(got["dbias"], clean["dbias"])


@pytest.mark.parametrize("order", [[0, 1024, 0, 1024], [1024, 0, 1024, 0], [0, 1024, 1000, 1024], [2000, -7, 1024, 3]], ids=str)
def test_offsets_out_of_order_with_a_cta_for_each_head(order):
    """More tiles than a batch in order could have: what is right is not said, but calls after it are."""
    op = training.Attention(1024, 3, 12, 1, 64, dtype=BF16, buckets=[0, 5])
    x = inputs(1024, 12, 1, 64, BF16, 0, True, [0, 5])
    good = lengths_to_offsets([500, 24, 500])
    want = both(op, x, good)
    both(op, x, torch.tensor(order, dtype=torch.int32, device="cuda"))
    got = both(op, x, good)
    for n in want:
        assert torch.equal(got[n], want[n]), n
