"""Argument checks of the attention's and the kept activations' C entries, and their holders, without a GPU."""
import ctypes

import pytest
import torch

from paper_2009_03816_b200 import binding, training
from paper_2009_03816_b200 import build as _build

BF16, F16, F32 = binding.PSOPS_BF16, binding.PSOPS_F16, binding.PSOPS_F32


@pytest.fixture(scope="module")
def lib():
    _build.build_library()
    return binding.load()


def _config(T=1000, S=7, H=4, G=2, D=64, kind=BF16, first=None, scale=0.125, flags=0, count=None):
    held = (ctypes.c_int32 * len(first))(*first) if first else None
    return binding.psops_attention_config(T, S, H, G, D, kind, len(first) if first and count is None else count or 0, held, scale,
                                          flags)


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(binding.psops_attention_config) == 48           # 8 + 6 x 4 + 8 + 2 x 4
    assert ctypes.sizeof(binding.psops_heads) == 24


def test_attention_config_and_workspace(lib):
    size = lambda **kw: binding.psops_attention_workspace_bytes(_config(**kw))
    assert size() > 0 and size() % 256 == 0
    assert size(flags=binding.PSOPS_ATTENTION_GRADS) > size()
    assert size(first=[0, 1, 5], flags=1) > size(flags=1)
    assert size(D=8) > 0 and size(D=128) > 0 and size(first=list(range(64))) > 0 and size(first=[0, 1024]) > 0
    # no score matrix: a long call's workspace is a small part of its tensors
    assert size(T=1 << 20, S=1, H=16, G=4, D=128, flags=1) < (1 << 20) * 16 * 128 * 2 // 20
    for kw in ({"T": 0}, {"T": (1 << 24) + 1}, {"S": 0}, {"H": 0}, {"H": 3}, {"G": 0}, {"G": 3}, {"D": 0}, {"D": 4}, {"D": 60}, {"D": 136},
               {"kind": F32}, {"kind": 0}, {"scale": 0.0}, {"scale": -1.0}, {"scale": float("inf")}, {"scale": float("nan")},
               {"flags": 2}, {"first": [1, 2]}, {"first": [0, 0]}, {"first": [0, 5, 4]}, {"first": [0, 1025]},
               {"first": list(range(65))}, {"count": 3}, {"count": -1}, {"H": 2048, "G": 1}):
        assert size(**kw) == 0, kw
    assert binding.load().psops_attention_workspace_bytes(None) == 0


def test_attention_refuses_before_touching_cuda(lib):
    out = ctypes.c_void_p(1)
    cfg = _config()
    for ws, size in ((None, 1 << 30), (0x101, 1 << 30), (0x100, 64)):
        assert lib.psops_attention_create(ctypes.byref(out), ctypes.byref(cfg), ws, size, None) == binding.PSOPS_EWORKSPACE
        assert not out.value
    assert lib.psops_attention_create(ctypes.byref(out), None, 0x100, 1 << 30, None) == binding.PSOPS_EINVAL
    assert lib.psops_attention_create(None, ctypes.byref(cfg), 0x100, 1 << 30, None) == binding.PSOPS_EINVAL
    assert lib.psops_attention_forward(None, None, None, None, None, 0, 0, None, 0, None, None, 0) == binding.PSOPS_EINVAL
    assert lib.psops_attention_backward(None, None, None, None, None, 0, 0, None, 0, None, None, None, None, None, None, None,
                                        0) == binding.PSOPS_EINVAL
    assert lib.psops_attention_set_stream(None, None) == binding.PSOPS_EINVAL
    assert lib.psops_attention_destroy(None) == binding.PSOPS_EINVAL
    assert lib.psops_attention_launch_count(None) == 0


def test_keep8_refuses_before_touching_cuda(lib):
    assert lib.psops_keep_create(None, None) == binding.PSOPS_EINVAL
    assert lib.psops_keep_pack(None, BF16, 1, 1, None, 1, None, None) == binding.PSOPS_EINVAL
    assert lib.psops_keep_unpack(None, BF16, 1, 1, None, None, None, 1) == binding.PSOPS_EINVAL
    assert lib.psops_keep_activate(None, 0, BF16, 1, 1, None, 1, None, 0, None, 1, None, None, None, None) == binding.PSOPS_EINVAL
    assert lib.psops_keep_activate_backward(None, 0, BF16, 1, 1, None, None, None, None, None, 1, None, 0, None, 0, None,
                                             0) == binding.PSOPS_EINVAL
    assert lib.psops_keep_set_stream(None, None) == binding.PSOPS_EINVAL
    assert lib.psops_keep_destroy(None) == binding.PSOPS_EINVAL


@pytest.mark.parametrize("count,far", [(1, 1), (2, 2), (3, 9), (8, 32), (16, 64), (32, 128), (32, 512), (48, 1000), (64, 64), (64, 1024)])
def test_distance_buckets(count, far):
    first = training.distance_buckets(count, far)
    near = count // 2
    assert len(first) == count and first[0] == 0 and first[:near] == list(range(near))
    assert all(a < b for a, b in zip(first, first[1:])) and first[-1] <= 1024
    for k, d in enumerate(first[near:]):
        # the smallest distance at or beyond near (far / near)^(k / n), or the next one that is free
        n = count - near
        if near and (near + k == 0 or d > first[near + k - 1] + 1):
            assert d ** n * near ** k >= far ** k * near ** n > (d - 1) ** n * near ** k
    for bad in ((0, 4), (65, 100), (8, 7), (8, 1025)):
        with pytest.raises(binding.PsopsError):
            training.distance_buckets(*bad)


# ---- the holders, on tensors in host memory, with stand-ins for the entries --------------------------------

@pytest.fixture
def attention(monkeypatch):
    calls = []
    monkeypatch.setattr(binding, "psops_attention_forward", lambda *a: calls.append(("forward", a)))
    monkeypatch.setattr(binding, "psops_attention_backward", lambda *a: calls.append(("backward", a)))
    monkeypatch.setattr(training.Attention, "_destroy", staticmethod(lambda ctx: calls.append(("destroy", ctx))))
    monkeypatch.setattr(training.Attention, "_launch_count", staticmethod(lambda ctx: 3))
    monkeypatch.setattr(training.Attention, "_follow", lambda op, *tensors: calls.append(("follow", tensors)))
    op = training.Attention.__new__(training.Attention)
    op.device = type("Cpu", (), {"index": -1})()          # get_device() of a tensor in host memory
    op.tokens, op.sequences, op.heads, op.kv_heads, op.dim, op.dtype = 20, 3, 4, 2, 8, torch.bfloat16
    op.buckets, op._follows, op.ctx = [0, 1, 4], True, 17
    yield op, calls
    op.ctx = None                                         # no context behind it


def _tensors(T=12):
    x = torch.zeros(T, 8, 8, dtype=torch.bfloat16)
    return x[:, :4], x[:, 4:6], x[:, 6:], torch.tensor([0, 5, T], dtype=torch.int32), torch.zeros(3, 4)


def test_attention_holder_passes_strides_and_zeroes_its_own_results(attention):
    op, calls = attention
    q, k, v, offsets, bias = _tensors()
    out, lse = op.forward(q, k, v, offsets, bias)
    assert out.shape == q.shape and out.is_contiguous() and lse.shape == (4, 12)
    name, a = calls[-1]
    assert name == "forward" and (a[1].token_stride, a[1].head_stride) == (64, 8) and a[2].p == k.data_ptr()
    assert a[5] == 2 and a[6] == 12 and a[8] == F32 and a[11] is True and a[9].token_stride == 32
    given = torch.ones_like(out)
    version = given._version
    got, lse = op.forward(q, k, v, offsets, bias, out=given)
    assert got is given and calls[-1][1][11] is False and not lse.any() and given._version > version
    grad = torch.zeros_like(out)
    dq, dk, dv, dbias = op.backward(q, k, v, offsets, out, lse, grad, bias, want=(True, False, True, True))
    a = calls[-1][1]
    assert dk is None and a[13] is None and a[12].p == dq.data_ptr() and a[16] is True and dbias.dtype == torch.float32
    # one given: what is made beside it starts as zeros, since rows of no sequence are left alone
    dq, dk, dv, dbias = op.backward(q, k, v, offsets, out, lse, grad, bias, dq=given)
    assert dq is given and calls[-1][1][16] is False and not dk.any() and not dv.any()
    assert [len(c[1]) for c in calls if c[0] == "follow"][-1] == 12        # all that the call touches
    op.close()
    op.close()
    assert [c for c in calls if c[0] == "destroy"] == [("destroy", 17)]


def test_attention_holder_refuses(attention):
    op, _ = attention
    q, k, v, offsets, bias = _tensors()
    out, lse = op.forward(q, k, v, offsets, bias)
    grad = torch.zeros_like(out)

    def refused(f, *a, **kw):
        with pytest.raises(binding.PsopsError) as e:
            f(*a, **kw)
        assert e.value.code == binding.PSOPS_EINVAL

    big = _tensors(21)
    for a in ((q.float(), k, v, offsets, bias), (q[:, :3], k, v, offsets, bias), (q, k[:5], v, offsets, bias), (q, k, q, offsets, bias),
              (q[..., :4], k, v, offsets, bias), (q.transpose(0, 2), k, v, offsets, bias), (None, k, v, offsets, bias),
              (q, k, v, offsets.long(), bias), (q, k, v, offsets[::2][:0], bias), (q, k, v, offsets[None], bias), (q, k, v, None, bias),
              (q, k, v, torch.zeros(5, dtype=torch.int32), bias), (q, k, v, offsets, None), (q, k, v, offsets, bias[:2]),
              (q, k, v, offsets, bias.half()), (q, k, v, offsets, bias.T.contiguous()), (big[0], big[1], big[2], offsets, bias),
              (q.mT.contiguous().mT, k, v, offsets, bias)):
        refused(op.forward, *a)
    refused(op.forward, q, k, v, offsets, bias, out=out[:5])
    for a in ((out[:5], lse, grad), (out, lse.T.contiguous(), grad), (out, lse.double(), grad), (out, lse, grad.float()),
              (out, lse, None)):
        refused(op.backward, q, k, v, offsets, *a, bias)
    refused(op.backward, q, k, v, offsets, out, lse, grad, bias, dk=q)
    refused(op.backward, q, k, v, offsets, out, lse, grad, bias, dbias=bias.half())
    refused(training.Attention, 4, 1, 1, 1, 8, device="cpu")
    refused(training.Attention, 4, 1, 1, 1, 8, dtype=torch.float32)


@pytest.fixture
def keep(monkeypatch):
    calls = []
    for name in ("pack", "unpack", "activate", "activate_backward"):
        monkeypatch.setattr(binding, "psops_keep_" + name, lambda *a, name=name: calls.append((name, a)))
    monkeypatch.setattr(training.Keep8, "_destroy", staticmethod(lambda ctx: None))
    monkeypatch.setattr(training.Keep8, "_follow", lambda op, *tensors: calls.append(("follow", tensors)))
    op = training.Keep8.__new__(training.Keep8)
    op.device = type("Cpu", (), {"index": -1})()
    op._follows, op.ctx = True, 5
    yield op, calls
    op.ctx = None                                         # no context behind it


def test_keep8_holder_shapes_and_strides(keep):
    op, calls = keep
    x = torch.zeros(3, 5, 300, dtype=torch.float16)
    codes, scales = op.pack(x)
    assert codes.shape == (3, 5, 304) and codes.dtype == torch.int8 and scales.shape == (3, 5, 3)
    assert calls[-1][1][1:4] == (F16, 15, 300) and calls[-1][1][5] == 300
    assert op.unpack(codes, scales, x.shape, x.dtype).shape == x.shape
    joint = torch.zeros(6, 40, dtype=torch.bfloat16)
    a, b = joint[:, :20], joint[:, 20:]
    y, kept = op.activate(a, b, "gelu")
    c = calls[-1][1]
    assert c[1] == binding.PSOPS_GELU and c[3:5] == (6, 20) and c[6] == 40 and c[8] == 40 and c[10] == 20 and len(kept) == 4
    room = torch.zeros(6, 40, dtype=torch.bfloat16)
    da, db = op.activate_backward(kept, y, "gelu", da=room[:, :20], db=room[:, 20:])
    c = calls[-1][1]
    assert c[12] == 40 and c[14] == 40 and c[15] is None and da.data_ptr() == room.data_ptr()
    y, kept = op.activate(a, kind="relu")
    assert len(kept) == 2 and calls[-1][1][7] is None
    da, db, again = op.activate_backward(kept, y, "relu", again=True)
    assert db is None and again.shape == y.shape


def test_keep8_holder_refuses(keep):
    op, _ = keep
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    codes, scales = op.pack(x)
    _, kept = op.activate(x, x)

    def refused(f, *a, **kw):
        with pytest.raises(binding.PsopsError) as e:
            f(*a, **kw)
        assert e.value.code == binding.PSOPS_EINVAL

    refused(op.pack, x.float())
    refused(op.pack, x.T)
    refused(op.pack, x[0, 0])
    refused(op.pack, x[:, :0])
    refused(op.pack, x[:1].expand(4, 64)[:, ::2])
    refused(op.pack, x[:1].expand(4, 64))
    refused(op.unpack, codes, scales, (4, 65), x.dtype)
    refused(op.unpack, codes.float(), scales, x.shape, x.dtype)
    refused(op.unpack, codes, scales.half(), x.shape, x.dtype)
    refused(op.unpack, codes, scales, x.shape, torch.float32)
    refused(op.unpack, codes, scales, x.shape, x.dtype, out=x[:3])
    refused(op.activate, x, x[:, :32])
    refused(op.activate, x, x.half())
    refused(op.activate, x, kind="tanh")
    refused(op.activate_backward, kept[:3], x)
    refused(op.activate_backward, kept, x[:3])
    refused(op.activate_backward, kept, x, da=x.half())
    refused(training.Keep8, device="cpu")
