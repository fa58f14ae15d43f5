"""The training operators' holders without a GPU: the C entries are stood in for by
Python functions that record their calls."""
import pytest
import torch

from paper_2009_03816_b200 import binding, training


class _Entries:
    """psops_xent_* that hand out numbers as contexts."""

    def __init__(self, monkeypatch):
        self.calls, self.made, self.fail = [], 0, None
        monkeypatch.setattr(binding, "psops_xent_forward", lambda ctx, *a: self.calls.append(("forward", ctx)))
        monkeypatch.setattr(binding, "psops_xent_backward", lambda ctx, *a: self.calls.append(("backward", ctx)))
        monkeypatch.setattr(training.LinearXent, "_destroy", staticmethod(lambda ctx: self.calls.append(("destroy", ctx))))
        monkeypatch.setattr(training.LinearXent, "_launch_count", staticmethod(lambda ctx: 10 * ctx))
        monkeypatch.setattr(training.LinearXent, "_open", lambda op, flags: self.open(flags))
        monkeypatch.setattr(training.LinearXent, "_capturing", lambda op: self.capturing)
        monkeypatch.setattr(training.LinearXent, "_follow", lambda op, *tensors: None)
        self.capturing = False

    def open(self, flags):
        if self.fail:
            raise self.fail
        self.made += 1
        return f"workspace {flags}", self.made


def _xent(monkeypatch):
    entries = _Entries(monkeypatch)
    op = training.LinearXent.__new__(training.LinearXent)
    op.device, op.tokens, op.dim, op.vocab, op.dtype = torch.device("cpu"), 4, 8, 6, torch.bfloat16
    op.device = type("Cpu", (), {"index": -1})()          # get_device() of a tensor in host memory
    op._w_shape, op._flags, op._follows = torch.Size((6, 8)), binding.PSOPS_XENT_GRADS, False
    op._workspace, op.ctx = op._open(op._flags)
    return op, entries


def _rows_not_aligned():
    flat = torch.zeros(6 * 8 + 8, dtype=torch.bfloat16)
    first = next(i for i in range(8) if (flat.data_ptr() + 2 * i) % 16)
    return flat[first:first + 48].view(6, 8)


def test_rows_that_are_not_aligned_get_a_context_beside_the_first(monkeypatch):
    op, entries = _xent(monkeypatch)
    h, w, y = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(6, 8, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    lse = torch.zeros(4)
    assert w.data_ptr() % 16 == 0
    run = lambda w: op._context("test", (w,), w, op._rows("test", "w", w))
    assert run(w) == 1
    kept = op._workspace
    entries.fail = RuntimeError("out of memory")
    with pytest.raises(RuntimeError, match="out of memory"):
        run(_rows_not_aligned())
    assert run(w) == 1                                    # still there, and the next attempt is a new one
    entries.fail, entries.capturing = None, True
    with pytest.raises(binding.PsopsError) as e:
        run(_rows_not_aligned())
    assert e.value.code == binding.PSOPS_ESTATE and entries.made == 1 and run(w) == 1
    entries.capturing = False
    assert run(_rows_not_aligned()) == 2
    entries.capturing = True
    assert run(_rows_not_aligned()) == 2 and run(w) == 1
    op.backward(h, w, y, lse, torch.zeros(()), dh=torch.zeros_like(h), dw=_rows_not_aligned())
    assert entries.calls == [("backward", 2)]
    assert op._workspace is kept and op._staged_workspace != kept and entries.made == 2
    assert op.launches == 30
    op.close()
    assert sorted(entries.calls[1:]) == [("destroy", 1), ("destroy", 2)] and op.ctx is None and op._staged is None
    assert op.launches == 30
    op.close()
    assert len(entries.calls) == 3


def _holder(cls, destroy):
    holder = cls.__new__(cls)
    holder.ctx = object()
    holder._destroy = destroy
    holder._launch_count = lambda ctx: 3
    return holder


@pytest.mark.parametrize("cls", [training.LinearXent, training.AdamW, training.GradNorm])
def test_a_context_is_destroyed_once_whatever_the_entry_answers(cls):
    seen = []

    def destroy(ctx):
        seen.append(ctx)
        raise binding.PsopsError(binding.PSOPS_ECUDA, "destroy", "the stream could not be waited for")

    holder = _holder(cls, destroy)
    ctx = holder.ctx
    with pytest.raises(binding.PsopsError):
        holder.close()
    assert holder.ctx is None and seen == [ctx]       # the library has freed it: the handle is gone
    holder.close()
    holder.__del__()
    assert seen == [ctx]


def test_both_contexts_are_destroyed_once_whatever_the_entry_answers():
    seen = []

    def destroy(ctx):
        seen.append(ctx)
        raise binding.PsopsError(binding.PSOPS_ECUDA, "destroy")

    op = _holder(training.LinearXent, destroy)
    op.ctx, op._staged = 1, 2
    with pytest.raises(binding.PsopsError):
        op.close()
    assert sorted(seen) == [1, 2] and op.ctx is None and op._staged is None
    op.close()
    assert len(seen) == 2


def test_a_swarm_is_destroyed_once_whatever_the_entry_answers(monkeypatch):
    seen = []

    def destroy(ctx):
        seen.append(ctx)
        raise binding.PsopsError(binding.PSOPS_ECUDA, "psops_destroy")

    monkeypatch.setattr(binding, "psops_destroy", destroy)
    swarm = binding.Swarm.__new__(binding.Swarm)
    swarm.ctx = 17
    with pytest.raises(binding.PsopsError):
        swarm.close()
    assert swarm.ctx is None
    swarm.close()
    assert seen == [17]


class _PlainXent:
    """Forward and backward of the linear cross entropy in torch operations, unseen by autograd as the kernels are."""

    def _join(self):
        pass

    def forward(self, h, w, targets, reduction):
        logits = h.float() @ w.float().T
        lse = torch.logsumexp(logits, 1)
        rows = lse - logits.gather(1, targets[:, None])[:, 0]
        return rows.mean() if reduction == "mean" else rows.sum(), rows, lse

    @torch.no_grad()
    def backward(self, h, w, targets, lse, grad, reduction, *, rows=None, want=(True, True)):
        d = torch.exp(h.float() @ w.float().T - lse[:, None])
        d[torch.arange(len(targets)), targets] -= 1.0
        d = d * grad / len(targets)
        return (d @ w.float()).to(h.dtype), (d.T @ h.float()).to(w.dtype)


def test_a_second_derivative_is_refused_rather_than_left_out():
    torch.manual_seed(0)
    h, w = torch.randn(5, 8, requires_grad=True), torch.randn(7, 8)
    y = torch.randint(0, 7, (5,))
    loss = training._LinearXentFunction.apply(h, w, y, _PlainXent(), "mean")
    (dh,) = torch.autograd.grad(loss, h, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (loss + dh.pow(2).sum()).backward()              # a gradient penalty
    loss = training._LinearXentFunction.apply(h, w, y, _PlainXent(), "mean")
    loss.backward()
    assert torch.equal(h.grad, dh)
