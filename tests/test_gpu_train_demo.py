"""The language-model example: local steps with the training operators inside
Algorithm 1, fitness straight from the loss kernel."""
import json
import math

import pytest

from paper_2009_03816_b200 import train_demo

import gpu_util

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("method", ["pso", "pa"])
@pytest.mark.parametrize("bits", [8, 32])
def test_workers_learn(method, bits):
    gpu_util.ensure_library()
    cfg = train_demo.TrainConfig(K=3, vocab=509, dim=72, tokens=512, epochs=2, iters_per_epoch=30, state_bits=bits)
    out = train_demo.run(method, cfg)
    # random weights predict nothing; the source can be learned down to its noise
    assert abs(out["initial_loss"] - math.log(cfg.vocab)) < 0.6
    assert len(out["best_loss"]) == 6 and out["steps"] == 60
    assert out["best_loss"][-1] < 0.8 * out["initial_loss"]
    assert all(b <= m for b, m in zip(out["best_loss"], out["mean_loss"]))
    if method == "pso":
        assert all(0 <= g < cfg.K for g in out["gbest"])
    else:                                            # after averaging all workers are the same
        assert out["best_loss"] == pytest.approx(out["mean_loss"], rel=1e-6)


def test_command_line(capsys):
    out = train_demo.main(["--k", "2", "--vocab", "300", "--dim", "40", "--tokens", "128", "--epochs", "1",
                           "--iters-per-epoch", "20"])
    assert json.loads(capsys.readouterr().out) == out
    assert set(out["methods"]) == {"pso", "pa"}
