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
