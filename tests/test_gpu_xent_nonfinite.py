"""Linear cross entropy where something is not finite: upstream gradients that
overflowed, and a context whose tensor-core products gave up."""
import pytest
import torch

from paper_2009_03816_b200 import training

import gpu_util

pytestmark = pytest.mark.gpu

# pairs of CTAs, single CTAs, dw in shares, rows of w through the workspace, few tokens, few classes
FORMS = [(300, 64, 500), (100, 64, 300), (1600, 200, 700), (140, 61, 400), (4, 64, 300), (50, 32, 20)]


def _inputs(T, D, V, dtype, seed=1):
    gpu_util.ensure_library()
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.empty(T, D, device="cuda").normal_(generator=g).to(dtype)
    w = (torch.empty(V, D, device="cuda").normal_(generator=g) * D ** -0.5).to(dtype)
    y = torch.randint(0, V, (T,), device="cuda", generator=g)
    return h, w, y


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,V", FORMS)
def test_left_out_tokens_get_no_gradient_from_an_upstream_gradient_that_is_not_finite(T, D, V, dtype):
    h, w, y = _inputs(T, D, V, dtype)
    out = torch.arange(T, device="cuda") % 3 == 1
    y[out] = -100
    op = training.LinearXent(T, D, V, dtype=dtype)
    _, rows, lse = op.forward(h, w, y)
    for bad in (float("inf"), -float("inf"), float("nan")):
        grad = torch.tensor(bad, device="cuda")
        for reduction in ("mean", "sum"):
            dh, dw = op.backward(h, w, y, lse, grad, reduction, rows=rows)
            assert bool((dh[out] == 0).all()), (bad, reduction)
            # the overflow itself stays to be seen by whoever looks at the gradients
            assert not bool(dh[~out].isfinite().all()) and not bool(dw.isfinite().all())
    op.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,V", FORMS)
def test_no_token_left_and_an_upstream_gradient_that_is_not_finite(T, D, V, dtype):
    h, w, y = _inputs(T, D, V, dtype)
    y.fill_(-100)
    op = training.LinearXent(T, D, V, dtype=dtype)
    loss, rows, lse = op.forward(h, w, y)
    assert float(loss) == 0.0
    for bad in (float("inf"), float("nan")):
        for reduction in ("mean", "sum"):
            dh, dw = op.backward(h, w, y, lse, torch.tensor(bad, device="cuda"), reduction)
            assert bool((dh == 0).all()) and bool((dw == 0).all()), (bad, reduction)
        dh, dw = op.backward(h, w, y, lse, torch.full((T,), bad, device="cuda"), "none")
        assert bool((dh == 0).all()) and bool((dw == 0).all()), bad
    op.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,V", FORMS)
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_one_tokens_overflowed_gradient_stays_with_that_token(T, D, V, dtype, bad):
    h, w, y = _inputs(T, D, V, dtype)
    op = training.LinearXent(T, D, V, dtype=dtype)
    _, rows, lse = op.forward(h, w, y)
    grad = torch.full((T,), 7.5, device="cuda")
    want, _ = op.backward(h, w, y, lse, grad, "none", rows=rows)
    grad[2] = bad
    got, dw = op.backward(h, w, y, lse, grad, "none", rows=rows)
    others = torch.arange(T, device="cuda") != 2
    assert bool(want.isfinite().all()) and torch.equal(got[others], want[others])
    assert not bool(got[2].isfinite().all()) and not bool(dw.isfinite().all())
    op.close()


def _give_up(workspace):
    """Sets the error word that a product sets which waited in vain (the fourth of the control block)."""
    workspace.view(torch.int32)[3] = 1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,V", FORMS[:4] + [(700, 64, 9000)])
def test_a_context_that_gave_up_leaves_no_numbers(T, D, V, dtype):
    h, w, y = _inputs(T, D, V, dtype)
    y[1] = -100
    one = torch.tensor(1.0, device="cuda")
    op = training.LinearXent(32_768 if V == 9000 else T, D, V, dtype=dtype)          # 9,000 entries: two pieces
    _, rows, lse = op.forward(h, w, y)
    assert bool(rows.isfinite().all())
    flat = torch.full((V * (D + 3) + 9,), 3.25, device="cuda", dtype=dtype)
    apart = flat[5:5 + V * (D + 3)].view(V, D + 3)[:, :D]                             # through the workspace
    op.backward(h, w, y, lse, one, dw=apart)
    assert bool(apart.isfinite().all())
    _give_up(op._workspace)
    if op._staged is not None:
        _give_up(op._staged_workspace)
    for reduction in ("mean", "sum"):
        loss, rows1, lse1 = op.forward(h, w, y, reduction)
        counts = y >= 0
        assert bool(loss.isnan()) and bool(rows1[counts].isnan().all()) and bool(lse1[counts].isnan().all())
        for want in ((True, True), (True, False), (False, True)):
            for dw in (None, apart):
                dh, dw = op.backward(h, w, y, lse, one, reduction, rows=rows, dw=dw, want=want)
                assert (dh is None or bool(dh.isnan().all())) and (dw is None or bool(dw.isnan().all())), want
    none = y.clone().fill_(-1)
    assert bool(op.forward(h, w, none)[0].isnan())
    assert all(bool(t.isnan().all()) for t in op.backward(h, w, none, lse, one))
    assert bool(op.backward(h[:0], w, y[:0], lse[:0], one)[1].isnan().all())          # no tokens at all
    apart.fill_(3.25)
    assert bool((flat == 3.25).all()), "wrote beside the rows"
    op.close()
