"""Attention against the formulas in 64 bits, within bounds counted in roundings."""
import pytest
import torch

from attention_util import compare, inputs, lengths_to_offsets, reference
from paper_2009_03816_b200 import build as _build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    _build.build_library()


def _run(lengths, heads, kv_heads, dim, dtype, buckets=None, first=0, rest=0, train=True, seed=0, spread=1.0, bias_dtype=None):
    from paper_2009_03816_b200 import training
    T = first + sum(lengths) + rest
    x = inputs(T, heads, kv_heads, dim, dtype, seed, train, buckets, bias_dtype, spread)
    op = training.Attention(max(T, 1), max(len(lengths), 1), heads, kv_heads, dim, dtype=dtype, buckets=buckets, gradients=train)
    offsets = lengths_to_offsets(lengths, first)
    bias = x.get("bias")
    out, lse = op.forward(x["q"], x["k"], x["v"], offsets, bias)
    got = {"out": out, "lse": lse}
    if train:
        dq, dk, dv, dbias = op.backward(x["q"], x["k"], x["v"], offsets, out, lse, x["grad"], bias)
        got.update(dq=dq, dk=dk, dv=dv)
        if bias is not None:
            got["dbias"] = dbias
    torch.cuda.synchronize()
    compare(got, reference(x["q"], x["k"], x["v"], lengths, first, x.get("grad"), bias, buckets), str((lengths, heads, kv_heads, dim)))
    op.close()
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("lengths", [[1], [2, 1], [17], [127], [128], [129], [300], [1000], [64, 0, 1, 190, 128, 0, 257]], ids=str)
def test_lengths(lengths, dtype):
    _run(lengths, 2, 1, 64, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("dim", [8, 16, 24, 40, 64, 72, 80, 120, 128])
def test_dims(dim, dtype):
    _run([70, 200, 5], 2, 2, dim, dtype, seed=dim)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (6, 2), (8, 1), (5, 5)])
def test_heads(heads, kv_heads):
    _run([150, 300], heads, kv_heads, 128, torch.bfloat16, seed=heads)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("count,far", [(8, 32), (32, 128), (48, 1000), (1, 1), (2, 2)])
def test_bias(count, far, dim, dtype):
    from paper_2009_03816_b200 import training
    buckets = training.distance_buckets(count, far)
    _run([1, 130, 700, 33], 4, 2, dim, dtype, buckets=buckets, seed=count)
    _run([1500], 1, 1, dim, dtype, buckets=buckets, seed=count, bias_dtype=torch.float32)


def test_rows_of_no_sequence():
    got = _run([100, 50], 2, 1, 64, torch.bfloat16, first=37, rest=90)
    for name in ("out", "dq", "dk", "dv"):
        assert not got[name][:37].any() and not got[name][187:].any()


def test_sharp_rows():
    _run([400], 2, 2, 128, torch.float16, spread=20.0)
    _run([400], 2, 2, 64, torch.bfloat16, spread=20.0)
