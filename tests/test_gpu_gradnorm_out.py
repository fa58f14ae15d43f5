"""Where the norm and the factor of psops_gradnorm_run go."""
import pytest
import torch

from paper_2009_03816_b200 import binding, training

import gpu_util

pytestmark = pytest.mark.gpu


def test_any_shape_of_two_numbers():
    gpu_util.ensure_library()
    gn = training.GradNorm([torch.tensor([3.0, -4.0], device="cuda")])
    for shape in ((2,), (1, 2), (2, 1)):
        out = torch.zeros(shape, device="cuda")
        norm, factor = gn.norm(2.5, out=out)
        assert norm.shape == factor.shape == ()
        assert float(norm) == 5.0 and float(factor) == pytest.approx(0.5, rel=1e-6)
        assert out.flatten().tolist() == [float(norm), float(factor)]
    for bad in ([0.0, 0.0], torch.zeros(3, device="cuda"), torch.zeros(2, 2, device="cuda")[:, 0]):
        with pytest.raises(binding.PsopsError) as e:
            gn.norm(1.0, out=bad)
        assert e.value.code == binding.PSOPS_EINVAL
    gn.close()
