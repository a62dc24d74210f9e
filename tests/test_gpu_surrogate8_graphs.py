"""GPU tests of what a captured step of Surrogate8 reads and writes: its memory
stays the graph's, whatever eager passes of another size, an optimizer or a
loader exchange afterwards."""
import pytest
import torch

from paper_2407_18352_amd import surrogate8
from test_gpu_surrogatef8_graphs import others, sizes

pytestmark = pytest.mark.gpu


def test_memory_exchanged_after_a_capture():
    g = torch.Generator().manual_seed(12)
    model = surrogate8.Surrogate8([4, 96, 64, 2], seed=3)
    x, dy = torch.randn((300, 4), generator=g).cuda(), torch.randn((300, 2), generator=g).cuda()
    want = model.forward(x)
    model.backward(dy)
    grads = [p.grad.clone() for p in model.parameters()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = model.forward(x)
        model.backward(dy)
    written = [p.grad.data_ptr() for p in model.parameters()]
    held = sizes(model._buffers() + model.parameters() + [p.grad for p in model.parameters()])
    for p in model.parameters():
        p.grad = None
    model.forward(torch.cat([x, x, x]))              # larger: other buffers
    model.backward(torch.cat([dy, dy, dy]))
    for p in model.parameters():
        p.data = p.detach() * 2
    taken = others(held)
    for _ in range(3):
        for t in model.captured.values():
            if t.data_ptr() in written:
                t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        got = {t.data_ptr(): t for t in model.captured.values()}
        assert all(torch.equal(got[a], w) for a, w in zip(written, grads))
        assert all(bool((t == 255).all()) for t in taken)
    model.captured.clear()
