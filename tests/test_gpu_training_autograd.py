"""The training operators among torch's automatic differentiation."""
import pytest
import torch

from paper_2009_03816_b200 import training

import gpu_util

pytestmark = pytest.mark.gpu


def _inputs(T=40, D=64, V=300):
    gpu_util.ensure_library()
    g = torch.Generator(device="cuda").manual_seed(3)
    h = torch.empty(T, D, device="cuda").normal_(generator=g).bfloat16()
    w = (0.1 * torch.empty(V, D, device="cuda").normal_(generator=g)).bfloat16()
    return h, w, torch.randint(0, V, (T,), device="cuda", generator=g)


def test_a_weight_stepped_before_its_backward_pass_is_noticed():
    h, w, y = _inputs()
    master = w.float()
    w.requires_grad_()
    op = training.LinearXent(40, 64, 300)
    opt = training.AdamW([master], [torch.ones_like(master)], copies=[w.detach()])
    loss = op(h, w, y)
    opt.step(1e-3)
    with pytest.raises(RuntimeError, match="inplace operation"):
        loss.backward()
    op(h, w, y).backward()
    assert bool(w.grad.isfinite().all())
    op.close(), opt.close()


def test_what_a_step_writes_counts_as_changed():
    flat = torch.zeros(1000, device="cuda")
    params = [flat[:300], flat[300:301], flat[301:].view(3, 233), torch.zeros(8, device="cuda"), torch.zeros(0, device="cuda")]
    copies = [torch.zeros_like(p, dtype=torch.float16) if i != 1 else None for i, p in enumerate(params)]
    opt = training.AdamW(params, [torch.ones_like(p) for p in params], copies=copies)
    seen = [t for t in params + copies if t is not None and t.numel()]
    before = [t._version for t in seen]
    opt.step(1e-3)
    assert all(t._version > b for t, b in zip(seen, before))
    opt.close()


def test_results_in_given_tensors_count_as_changed():
    h, w, y = _inputs()
    op = training.LinearXent(40, 64, 300)
    loss, dh, dw = torch.zeros(3, device="cuda"), torch.zeros_like(h), torch.zeros_like(w)
    _, rows, lse = op.forward(h, w, y, loss=loss[1])
    op.backward(h, w, y, lse, loss[:1], dh=dh, dw=dw)
    norm = training.GradNorm([dw])
    out = torch.zeros(2, device="cuda")
    norm.norm(1.0, out=out)
    assert all(t._version > 0 for t in (loss, dh, dw, out))
    op.close(), norm.close()
