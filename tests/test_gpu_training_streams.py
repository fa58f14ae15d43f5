"""The training operators with CUDA graphs, captures and streams of their own."""
import pytest
import torch

from paper_2009_03816_b200 import binding, training

import gpu_util

pytestmark = pytest.mark.gpu


def _inputs(T, D, V, dtype=torch.bfloat16, seed=1):
    gpu_util.ensure_library()
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.empty(T, D, device="cuda").normal_(generator=g).to(dtype)
    w = (torch.empty(V, D, device="cuda").normal_(generator=g) * D ** -0.5).to(dtype)
    return h, w, torch.randint(0, V, (T,), device="cuda", generator=g)


def _not_aligned(t):
    flat = torch.zeros(t.numel() + 8, device="cuda", dtype=t.dtype)
    view = flat[1:1 + t.numel()].view(t.shape)
    view.copy_(t)
    return view


@pytest.mark.parametrize("T,D,V", [(300, 64, 3000), (3, 64, 3000), (60, 64, 40)])
def test_a_captured_graph_survives_rows_that_are_not_aligned(T, D, V):
    h, w, y = _inputs(T, D, V)
    one = torch.tensor(1.0, device="cuda")
    op = training.LinearXent(T, D, V)
    want = op.forward(h, w, y)
    want = (*want, *op.backward(h, w, y, want[2], one, rows=want[1]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = op.forward(h, w, y)
        got = (*got, *op.backward(h, w, y, got[2], one, rows=got[1]))
    before = op.launches
    w2, dw2 = _not_aligned(w), _not_aligned(w)
    for loss, rows, lse in (op.forward(h, w2, y), op.forward(h, w, y)):
        dh, _ = op.backward(h, w2, y, lse, one, rows=rows, dw=dw2)
        for a, b in zip(want, (loss, rows, lse, dh, dw2)):
            assert torch.equal(a, b)
    assert op.launches > before
    # what torch hands out now must not be memory that the graph still writes
    taken = [torch.full((1 << 18,), 1.5, device="cuda") for _ in range(256)]
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert all(bool((t == 1.5).all()) for t in taken)
    # and rows that are not aligned can be captured once the context is there
    second = torch.cuda.CUDAGraph()
    with torch.cuda.graph(second):
        got = op.forward(h, w2, y)
    second.replay()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    del graph, second
    op.close()


def test_rows_that_are_not_aligned_are_refused_if_a_capture_meets_them_first():
    h, w, y = _inputs(100, 64, 300)
    op = training.LinearXent(100, 64, 300)
    want = op.forward(h, w, y)
    w2 = _not_aligned(w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(binding.PsopsError) as e:
            op.forward(h, w2, y)
        got = op.forward(h, w, y)                          # the capture goes on
    assert e.value.code == binding.PSOPS_ESTATE
    graph.replay()
    for a, b, c in zip(want, got, op.forward(h, w2, y)):
        assert torch.equal(a, b) and torch.equal(a, c)
    del graph
    op.close()


# ---- a stream of the holder's own beside the current one -------------------------
# torch.cuda._sleep occupies a stream for some 50 ms: without the order between the two
# streams, and without memory being kept for the one that still uses it, what follows on
# the other stream runs long before it.

def _busy():
    torch.cuda._sleep(100_000_000)


def _adamw(stream, p, g, **kw):
    return training.AdamW([p], [g], stream=stream, **kw)


@pytest.mark.parametrize("bits", [32, 8])
def test_default_moments_are_zero_before_the_first_step_on_a_given_stream(bits):
    gpu_util.ensure_library()
    torch.manual_seed(0)
    n = 1 << 20
    p0, g = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    want, got = p0.clone(), p0.clone()
    opt = _adamw(None, want, g, bits=bits)
    for _ in range(3):
        opt.step(1e-2)
    torch.cuda.synchronize()
    own = torch.cuda.Stream()
    dirt = [torch.full((n,), 7.0, device="cuda") for _ in range(8)]       # what the moments' memory holds before
    del dirt
    _busy()
    opt2 = _adamw(own.cuda_stream, got, g, bits=bits)
    for _ in range(3):
        opt2.step(1e-2)
    own.synchronize()
    assert torch.equal(want, got) and opt2.steps == 3
    for a, b in zip(opt.moments, opt2.moments):
        assert torch.equal(a[0].view(torch.uint8), b[0].view(torch.uint8))
    opt.close(), opt2.close()


def test_a_given_stream_waits_for_what_the_current_one_has_been_given():
    h, w, y = _inputs(300, 64, 500)
    one = torch.ones((), device="cuda")
    own = torch.cuda.Stream()
    plain, op = training.LinearXent(300, 64, 500), training.LinearXent(300, 64, 500, stream=own.cuda_stream)
    want = plain.forward(h, w, y)
    want = (*want, *plain.backward(h, w, y, want[2], one, rows=want[1]))
    torch.cuda.synchronize()
    late = torch.zeros_like(h)
    dirt = [torch.empty_like(t) for t in want for _ in range(4)]
    _busy()
    for t in dirt:
        t.fill_(7.0)                                   # on their way when the outputs take over their memory
    late.copy_(h)
    del dirt, t
    got = op.forward(late, w, y)
    got = (*got, *op.backward(late, w, y, got[2], one, rows=got[1]))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    norm = training.GradNorm([got[4]], stream=own.cuda_stream)
    _busy()
    got[4].mul_(2.0)
    n, factor = norm.norm(1.0)
    own.synchronize()
    assert float(n) == pytest.approx(2.0 * float(want[4].double().norm()), rel=1e-5)
    plain.close(), op.close(), norm.close()


def test_memory_let_go_of_is_not_used_again_before_a_given_stream_is_done():
    h, w, y = _inputs(300, 64, 500)
    own = torch.cuda.Stream()
    op = training.LinearXent(300, 64, 500, stream=own.cuda_stream)
    one = torch.ones((), device="cuda")
    loss, rows, lse = op.forward(h, w, y)
    dh, dw = op.backward(h, w, y, lse, one, rows=rows)
    torch.cuda.synchronize()
    h2, one2 = h.clone(), one.clone()
    out = torch.zeros_like(dw)
    with torch.cuda.stream(own):
        _busy()
    op.forward(h2, w, y)                               # results dropped at once
    op.backward(h2, w, y, lse, one2, rows=rows, dw=out)
    del h2, one2
    taken = [torch.full(s, 1.5, device="cuda", dtype=d) for s, d in (((), torch.float32), ((300,), torch.float32),
                                                                     (h.shape, h.dtype)) for _ in range(8)]
    torch.cuda.synchronize()
    assert all(bool((t == 1.5).all()) for t in taken)
    assert torch.equal(out, dw)
    # AdamW: the scale and the gradients of a step that still waits
    p, g = torch.zeros(5000, device="cuda"), torch.ones(5000, device="cuda")
    opt = _adamw(own.cuda_stream, p, g.clone(), weight_decay=0.0)
    torch.cuda.synchronize()
    with torch.cuda.stream(own):
        _busy()
    scale = torch.full((), 0.5, device="cuda")
    opt.step(1e-2, scale)
    opt.set_grads([g])
    del scale
    taken = [torch.full((), float("nan"), device="cuda") for _ in range(8)] + [torch.full((5000,), float("nan"), device="cuda")
                                                                             for _ in range(4)]
    torch.cuda.synchronize()
    assert opt.steps == 1 and bool((p < -0.0099).all()) and len(taken) == 12
    op.close(), opt.close()


def test_the_differentiable_call_on_a_given_stream():
    h, w, y = _inputs(300, 64, 500)
    own = torch.cuda.Stream()
    plain, op = training.LinearXent(300, 64, 500), training.LinearXent(300, 64, 500, stream=own.cuda_stream)
    grads = []
    for x in (plain, op):
        h1, w1 = h.clone().requires_grad_(), w.clone().requires_grad_()
        with torch.cuda.stream(own):
            _busy()
        loss = 2.0 * x(h1, w1, y)
        with torch.cuda.stream(own):
            _busy()
        loss.backward()
        grads.append((loss.detach().clone(), h1.grad.clone(), w1.grad.clone()))
    for a, b in zip(*grads):
        assert torch.equal(a, b)
    plain.close(), op.close()


def test_a_given_stream_in_a_capture():
    h, w, y = _inputs(300, 64, 500)
    own = torch.cuda.Stream()
    op = training.LinearXent(300, 64, 500, stream=own.cuda_stream)
    want = op.forward(h, w, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=own):
        got = op.forward(h, w, y)
    for t in got:
        t.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    del graph
    op.close()


def test_new_gradient_addresses_are_refused_inside_a_capture():
    gpu_util.ensure_library()
    n = 5000
    p = torch.zeros(n, device="cuda")
    a, b, c = (torch.full((n,), x, device="cuda") for x in (1.0, 2.0, 4.0))
    opt, norm = training.AdamW([p], [a], weight_decay=0.0), training.GradNorm([a])
    out = torch.zeros(2, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for holder in (opt, norm):
            with pytest.raises(binding.PsopsError) as e:
                holder.set_grads([b])
            assert e.value.code == binding.PSOPS_ESTATE
        norm.norm(1.0, out=out)
        opt.step(1e-2)
    graph.replay()
    assert float(out[0]) == pytest.approx(n ** 0.5, rel=1e-6) and opt.steps == 1
    norm.set_grads([c]), opt.set_grads([c])             # outside, and the graph reads them from then on
    graph.replay()
    assert float(out[0]) == pytest.approx(4 * n ** 0.5, rel=1e-6) and opt.steps == 2
    assert opt.grads[0] is c and norm.grads[0] is c
    del graph
    opt.close(), norm.close()


def test_calls_on_two_branches_of_one_capture_come_after_one_another():
    h, w, y = _inputs(2000, 128, 3000)
    h2 = (h.float() * 0.5).bfloat16()
    one = torch.ones((), device="cuda")
    op = training.LinearXent(2000, 128, 3000)

    def both(x):
        loss, rows, lse = op.forward(x, w, y)
        return loss, rows, lse, *op.backward(x, w, y, lse, one, rows=rows)

    want = [both(x) for x in (h, h2, h, h2)]
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=first):
        second.wait_stream(first)                        # the branch: nothing else orders the two
        got = []
        for k, x in enumerate((h, h2, h, h2)):
            with torch.cuda.stream((first, second)[k % 2]):
                got.append(both(x))
        first.wait_stream(second)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for s, t in zip(a, b):
            assert torch.equal(s, t)
    op.close()
    del graph


def test_setting_up_and_waiting_are_refused_inside_a_capture():
    h, w, y = _inputs(60, 64, 40)
    p, g = torch.zeros(100, device="cuda"), torch.ones(100, device="cuda")
    opt = training.AdamW([p], [g], weight_decay=0.0)
    graph = torch.cuda.CUDAGraph()
    refused = [lambda: training.LinearXent(60, 64, 40), lambda: training.AdamW([p], [g], moments=([g.clone()], [g.clone()])),
               lambda: training.GradNorm([g]), lambda: opt.steps]
    with torch.cuda.graph(graph):
        for k, f in enumerate(refused):
            with pytest.raises(binding.PsopsError) as e:
                f()
            assert e.value.code == binding.PSOPS_ESTATE, k
        opt.step(1e-2)
    for _ in range(3):
        graph.replay()
    assert opt.steps == 3 and bool((p < -0.0299).all())
    del graph
    opt.close()
