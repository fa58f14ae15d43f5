"""Argument checks of the training operators' C entries that need no GPU."""
import ctypes

import pytest

from paper_2009_03816_b200 import binding
from paper_2009_03816_b200 import build as _build


@pytest.fixture(scope="module")
def lib():
    _build.build_library()
    return binding.load()


def _adamw(n=(1000,), **kw):
    cfg = binding.psops_adamw_config(0.9, 0.999, 1e-8, 0, 32, binding.PSOPS_F32, binding.PSOPS_NONE, len(n))
    for k, v in kw.items():
        setattr(cfg, k, v)
    t = (binding.psops_adamw_tensor * len(n))()
    for i, c in enumerate(n):
        t[i].n = c
    return cfg, t


def test_adamw_struct_layouts_match_the_header():
    assert ctypes.sizeof(binding.psops_adamw_config) == 48
    assert ctypes.sizeof(binding.psops_adamw_tensor) == 72


def test_adamw_workspace(lib):
    small = binding.psops_adamw_workspace_bytes(*_adamw((1,)))
    assert small > 0 and small % 256 == 0
    assert binding.psops_adamw_workspace_bytes(*_adamw((1 << 30,))) > small
    assert binding.psops_adamw_workspace_bytes(*_adamw((0,))) > 0
    for kw in ({"beta1": 1.0}, {"beta2": -0.5}, {"beta1": float("nan")}, {"eps": -1e-8}, {"eps": float("inf")},
               {"steps_done": -1}, {"state_bits": 16}, {"grad_type": 0}, {"grad_type": 9}, {"copy_type": binding.PSOPS_F32},
               {"n_tensors": 0}):
        assert binding.psops_adamw_workspace_bytes(*_adamw(**kw)) == 0, kw
    assert binding.psops_adamw_workspace_bytes(*_adamw((-1,))) == 0
    assert binding.psops_adamw_workspace_bytes(*_adamw((1 << 41,))) == 0


def test_adamw_create_refuses_before_touching_cuda(lib):
    out = ctypes.c_void_p(1)
    cfg, t = _adamw()
    make = lambda: lib.psops_adamw_create(ctypes.byref(out), ctypes.byref(cfg), t, 0x100, 1 << 20, None)
    assert make() == binding.PSOPS_EINVAL and not out.value          # null arrays
    t[0].p = t[0].g = t[0].m = t[0].v = 0x1000
    t[0].g = 0x1002
    assert make() == binding.PSOPS_EALIGN
    t[0].g = 0x1000
    t[0].copy = 0x1000
    assert make() == binding.PSOPS_EINVAL                            # a copy without a type
    t[0].copy = None
    t[0].weight_decay = float("nan")
    assert make() == binding.PSOPS_EINVAL
    t[0].weight_decay = 0.0
    for ws, size in ((None, 1 << 20), (0x101, 1 << 20), (0x100, 16)):
        assert lib.psops_adamw_create(ctypes.byref(out), ctypes.byref(cfg), t, ws, size, None) == binding.PSOPS_EWORKSPACE
    cfg.state_bits = 8
    assert make() == binding.PSOPS_EINVAL                            # no scales
    assert lib.psops_adamw_step(None, 0.1, None) == binding.PSOPS_EINVAL
    assert lib.psops_adamw_destroy(None) == binding.PSOPS_EINVAL
    assert lib.psops_adamw_set_grads(None, None) == binding.PSOPS_EINVAL


def test_gradnorm_refuses_before_touching_cuda(lib):
    assert binding.psops_gradnorm_workspace_bytes([5, 0]) > 0
    assert binding.psops_gradnorm_workspace_bytes([-1]) == 0
    assert binding.psops_gradnorm_workspace_bytes([]) == 0
    for grads, sizes, kind, code in (([0], [4], binding.PSOPS_F32, binding.PSOPS_EINVAL),
                                     ([0x1001], [4], binding.PSOPS_F16, binding.PSOPS_EALIGN),
                                     ([0x1000], [4], 7, binding.PSOPS_EINVAL),
                                     ([0x1000], [4], binding.PSOPS_F32, binding.PSOPS_EWORKSPACE)):
        with pytest.raises(binding.PsopsError) as e:
            binding.psops_gradnorm_create(grads, sizes, kind, None)
        assert e.value.code == code
    assert lib.psops_gradnorm_run(None, 1.0, None) == binding.PSOPS_EINVAL
    assert lib.psops_gradnorm_destroy(None) == binding.PSOPS_EINVAL


def test_xent_config_and_workspace(lib):
    assert ctypes.sizeof(binding.psops_xent_config) == 32
    make = lambda T=64, D=32, V=100, kind=binding.PSOPS_BF16, flags=0: \
        binding.psops_xent_workspace_bytes(binding.psops_xent_config(T, D, V, kind, flags))
    assert make() > 0 and make(flags=binding.PSOPS_XENT_GRADS) > make()
    assert make(flags=binding.PSOPS_XENT_STAGED) > make() and make(D=33) > make(D=40)
    # the gradients' workspace stays far below the logits of a large call
    assert make(8192, 4096, 131072, flags=binding.PSOPS_XENT_GRADS) < 8192 * 131072 * 2 / 2
    for kw in ({"T": 0}, {"T": 1 << 25}, {"D": 0}, {"D": 1 << 21}, {"V": 0}, {"V": 1 << 31}, {"kind": binding.PSOPS_F32},
               {"kind": 0}, {"flags": 4}):
        assert make(**kw) == 0, kw


def test_xent_refuses_before_touching_cuda(lib):
    out = ctypes.c_void_p(1)
    cfg = binding.psops_xent_config(64, 32, 100, binding.PSOPS_BF16, 0)
    for ws, size in ((None, 1 << 30), (0x101, 1 << 30), (0x100, 64)):
        assert lib.psops_xent_create(ctypes.byref(out), ctypes.byref(cfg), ws, size, None) == binding.PSOPS_EWORKSPACE
        assert not out.value
    assert lib.psops_xent_create(ctypes.byref(out), None, 0x100, 1 << 30, None) == binding.PSOPS_EINVAL
    assert lib.psops_xent_forward(None, None, 0, None, 0, None, 0, 0, None, None, None) == binding.PSOPS_EINVAL
    assert lib.psops_xent_backward(None, None, 0, None, 0, None, 0, None, None, None, 0, None, 0, None, 0) == binding.PSOPS_EINVAL
    assert lib.psops_xent_destroy(None) == binding.PSOPS_EINVAL
