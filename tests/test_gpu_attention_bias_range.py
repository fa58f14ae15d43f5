"""Attention under finite biases beside which fp32 cannot hold a score: masks of -1e9 or of fp16's lowest number, levels
that a whole head shares.  A constant that all of a row's pairs have in common changes nothing but lse, so what such a bias
asks for follows from one that has the constant taken off."""
import pytest
import torch

from attention_util import F, compare, inputs, lengths_to_offsets, reference
from paper_2009_03816_b200 import training
from paper_2009_03816_b200 import build as _build

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
BUCKETS = [0, 4, 9, 30, 200]
# In the oracle's place of a level: pairs beside it have probabilities of e^-150 e^20 (scores differ by less than 20) at
# most, and thousands of them times numbers below 100 stay under 1e-50, less than half the smallest number of any type.
FAR = 150.0


@pytest.fixture(scope="module", autouse=True)
def _library():
    _build.build_library()


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("lowest,out", [(-1e31, True), (-1.0001e30, True), (-1e30, False), (-8e29, False), (-6.95e29, False), (-65504.0, False)])
def test_what_takes_pairs_out(lowest, out, dtype):
    """It is the bias itself that lies below -1e30; other numbers are biases, fp16's lowest among them."""
    op = training.Attention(40, 1, 2, 1, 16, dtype=dtype, buckets=[0, 1], gradients=False)
    x = inputs(40, 2, 1, 16, dtype, grad=False)
    bias = torch.tensor([[lowest, 0.0], [0.0, 0.0]], device="cuda")
    bias = bias.to(F16) if lowest == -65504.0 and dtype is F16 else bias
    o, lse = op.forward(x["q"], x["k"], x["v"], lengths_to_offsets([40]), bias)
    if out:                                              # the first token of head 0 is left with no pair
        assert not o[0, 0].any() and float(lse[0, 0]) == -torch.inf
    else:                                                # or has one
        assert torch.equal(o[0, 0], x["v"][0, 0])
        score = float(x["q"][0, 0].double() @ x["k"][0, 0].double()) / 4.0
        assert abs(float(lse[0, 0]) - (lowest + score)) <= 2.0 ** -22 * abs(lowest)
    assert torch.equal(o[0, 1], x["v"][0, 0]) and torch.isfinite(o).all() and torch.isfinite(lse[:, 1:]).all()


def check(lengths, dtype, dim, held, small, row_shift, heads=4, kv_heads=2, first=3, rest=5, grad=True):
    """held: the bias that is passed; small: one that asks for the same gradients; row_shift: what it takes off the lse
    of position i of a sequence, by head (heads x positions, 64 bits)."""
    T = first + sum(lengths) + rest
    x = inputs(T, heads, kv_heads, dim, dtype, 1)
    op = training.Attention(T, len(lengths), heads, kv_heads, dim, dtype=dtype, buckets=BUCKETS)
    offsets = lengths_to_offsets(lengths, first)
    out, lse = op.forward(x["q"], x["k"], x["v"], offsets, held)
    got = {"out": out}
    got["dq"], got["dk"], got["dv"], got["dbias"] = op.backward(x["q"], x["k"], x["v"], offsets, out, lse, x["grad"], held)
    want = reference(x["q"], x["k"], x["v"], lengths, first, x["grad"], small, BUCKETS)
    compare(got, want)
    exact, bound = want["lse"]
    at = first
    for n in lengths:
        rows = slice(at, at + n)
        at += n
        exact[:, rows] += row_shift[:, :n]
        bound[:, rows] += 2 * F * exact[:, rows].abs()
    compare({"lse": lse}, want)
    # each gradient by itself is the same
    for i, name in enumerate(("dq", "dk", "dv", "dbias")):
        alone = op.backward(x["q"], x["k"], x["v"], offsets, out, lse, x["grad"], held, want=[j == i for j in range(4)])[i]
        assert torch.equal(alone, got[name]), name
    op.close()


def table(dtype, heads=4, seed=2):
    return torch.empty(len(BUCKETS), heads, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


LEVELS = [(-1e4, F32), (-65504.0, F16), (-1e6, F32), (-1e9, F32), (-1e9, BF16), (-8e29, F32), (300.0, F16), (65504.0, F16), (1e9, F32)]
TYPES = [(level, kind, dtype) for level, kind in LEVELS for dtype in (BF16, F16) if kind in (F32, dtype)]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("level,kind,dtype", TYPES, ids=str)
def test_the_nearest_keys(level, kind, dtype, dim):
    """One bucket: the first tokens of each sequence have pairs of no other one."""
    held = table(kind)
    held[0] = level
    small = held.clone()
    small[0] = FAR if level > 0 else -FAR
    level = float(held[0, 0])
    shift = torch.zeros(4, 400, dtype=torch.float64, device="cuda")
    shift[:, :400 if level > 0 else BUCKETS[1]] = level - float(small[0, 0])
    check([1, 2, 200, 130, 5, 400], dtype, dim, held, small.float(), shift)


@pytest.mark.parametrize("copies", [1, 30])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("level,kind,dtype", TYPES, ids=str)
def test_a_whole_head(level, kind, dtype, dim, copies):
    """All buckets of one head, the other heads as usual; few tiles and many."""
    held = table(kind)
    held[:, 1] = level
    small = held.clone()
    small[:, 1] = 0.0
    shift = torch.zeros(4, 400, dtype=torch.float64, device="cuda")
    shift[1] = float(held[0, 1])
    check([1, 300, 2, 400, 64] * copies, dtype, dim, held, small.float(), shift)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("level", [-1e6, 1e6, -3000.0])
def test_differences_beside_a_level(level, dtype):
    """Buckets that differ by fractions beside the level they share; the softmax sees the fractions."""
    small = (table(F32) * 16).round() / 16
    held = small.clone()
    held[:, :3] += level
    assert torch.equal(held[:, :3].double() - level, small[:, :3].double())
    shift = torch.zeros(4, 400, dtype=torch.float64, device="cuda")
    shift[:3] = level
    check([300, 7, 400, 33], dtype, 64, held, small, shift)
    # levels that rise with the distance: each row's is the highest that it meets
    rise = held.clone()
    step = 1000.0 * torch.arange(len(BUCKETS), device="cuda")
    rise[:, 0] = level + step
    small[:, 0] = FAR * torch.arange(len(BUCKETS), device="cuda")
    of = torch.bucketize(torch.arange(400, device="cuda"), torch.tensor(BUCKETS, device="cuda"), right=True) - 1
    shift[0] = (rise[:, 0].double() - small[:, 0].double())[of]
    check([300, 7, 400, 33], dtype, 64, rise, small, shift)


def test_beside_infinities():
    """Buckets that are taken out beside a level, and rows that are left with none."""
    held = table(F32)
    held[0], held[2] = -1e9, -torch.inf
    small = held.clone()
    small[0] = -FAR
    shift = torch.zeros(4, 400, dtype=torch.float64, device="cuda")
    shift[:, :BUCKETS[1]] = -1e9 + FAR
    check([300, 9, 1], BF16, 64, held, small, shift)
    held[:, 0] = -torch.inf
    held[3, 0] = -1e9                # the first 30 tokens have nothing, those up to 199 this alone
    small[:, 0] = held[:, 0]
    small[3, 0] = -FAR
    shift[0] = 0.0
    shift[0, 30:] = -1e9 + FAR
    small[4, 0] = held[4, 0] = -torch.inf
    check([300, 9, 1], F16, 64, held, small, shift)


@pytest.mark.parametrize("lengths", [[100, 60], [700, 300, 2] * 20], ids=["few tiles", "many"])
def test_levels_that_come_and_go_in_a_graph(lengths):
    """What a table asks for is found on the device: a recorded pass is right for the tables of all its replays."""
    T = sum(lengths)
    x = inputs(T, 4, 2, 64, BF16, 1)
    bias, offsets = table(F32), lengths_to_offsets(lengths)
    op = training.Attention(T, len(lengths), 4, 2, 64, buckets=BUCKETS)

    def both(op):
        out, lse = op.forward(x["q"], x["k"], x["v"], offsets, bias)
        return (out, lse, *op.backward(x["q"], x["k"], x["v"], offsets, out, lse, x["grad"], bias))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(op)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held = both(op)
    for seed, level in ((1, None), (2, -1e9), (3, None), (4, 1e6)):
        bias.copy_(table(F32, seed=seed))
        if level is not None:
            bias[:2, 1:] = level
        graph.replay()
        torch.cuda.synchronize()
        fresh = training.Attention(T, len(lengths), 4, 2, 64, buckets=BUCKETS)
        for a, b in zip(held, both(fresh)):
            assert torch.equal(a, b), (seed, level)
        fresh.close()
