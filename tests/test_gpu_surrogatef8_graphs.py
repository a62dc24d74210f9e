"""GPU tests of what a captured pass of SurrogateF8 reads and writes: its memory
stays the graph's, whatever an optimizer or a loader exchanges afterwards."""
import torch
import pytest

from paper_2407_18352_amd import api, surrogatef8

pytestmark = pytest.mark.gpu


def model_and_batch(n=150):
    g = torch.Generator().manual_seed(11)
    model = surrogatef8.SurrogateF8([4, 32, 64, 2], groups=4, seed=3)
    return model, torch.randn((n, 4), generator=g).cuda(), torch.randn((n, 2), generator=g).cuda()


def others(sizes):
    """Tensors that take the memory that others of these sizes have left, if they have."""
    return [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(8)]


def sizes(tensors):
    return [t.numel() * t.element_size() for t in tensors]


@pytest.mark.parametrize("accumulate", [False, True])
def test_gradients_dropped_after_a_capture(accumulate):
    model, x, dy = model_and_batch()
    model.forward(x)
    model.backward(dy)
    want = [p.grad.clone() for p in model.parameters()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                    # without clipping
        model.forward(x)
        model.backward(dy, accumulate)
    written = [p.grad.detach() for p in model.parameters()]
    addresses = [t.data_ptr() for t in written]
    held = sizes(written)
    del written
    for p in model.parameters():                     # as zero_grad does
        p.grad = None
    taken = others(held)
    assert not set(addresses) & {t.data_ptr() for t in taken}
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool((t == 255).all()) for t in taken)
    model.backward(dy)                               # others, of an eager pass
    assert not set(addresses) & {p.grad.data_ptr() for p in model.parameters()}
    got = [t for a in addresses for (at, _), t in [kv for kv in model.captured.items() if isinstance(kv[0], tuple)] if at == a]
    times = 4 if accumulate else 1                   # the eager pass, or nothing, and three replays
    assert len(got) == len(want)
    for t, w in zip(got, want):
        assert torch.allclose(t, times * w, rtol=1e-6, atol=1e-6 * float(w.abs().max()))


def test_parameters_exchanged_after_a_capture():
    model, x, dy = model_and_batch()
    want = model.answer(x)
    model.forward(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        model.update()
        y = model.answer(x)
    old = sizes(model.parameters())
    for p in model.parameters():                     # as a loader of other weights may do
        p.data = p.detach() * 3 + 1
    taken = others(old)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)                      # the graph's own
    assert all(bool((t == 255).all()) for t in taken)
    model.update()
    assert not torch.equal(model.answer(x), want)


def test_a_backward_pass_alone_in_a_graph():
    """It reads what the eager forward pass before it kept, also when another size has taken that one's place."""
    model, x, dy = model_and_batch()
    model.forward(x)
    model.backward(dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    model.forward(x)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        model.backward(dy)
    want = [p.grad.clone() for p in model.parameters()]
    kept = sizes(model._buffers())
    model.forward(x[:40])
    model.backward(dy[:40])
    taken = others(kept)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p.grad, w) for p, w in zip(model.parameters(), want))
    assert all(bool((t == 255).all()) for t in taken)


def test_gradients_of_another_storage_are_clipped_where_they_are():
    model, x, dy = model_and_batch()
    model.forward(x)
    model.backward(dy)
    model.clip(1e9)
    held = model.set
    model.clip(1e9)
    assert model.set is held                         # where they were: the same set
    old = [p.grad.detach() for p in model.parameters()]
    before = [t.clone() for t in old]
    for i, p in enumerate(model.parameters()):       # the same tensor objects
        if i % 2:
            p.grad.data = p.grad.detach() * 2
        else:
            p.grad.set_(p.grad.detach() * 2)
    total = torch.stack([t.double().norm() for t in before]).norm().item()
    norm = model.clip(total)
    torch.cuda.synchronize()
    assert abs(norm.item() - 2 * total) <= 1e-6 * total
    for p, t, b in zip(model.parameters(), old, before):
        assert torch.equal(t, b) and torch.allclose(p.grad, b, rtol=1e-6)
    assert model.set is not held


def test_a_set_holds_the_memory_it_was_made_of():
    a, b, into = (torch.full((1000,), v, device="cuda") for v in (3.0, 4.0, 0.0))
    grads, norm = api.GradientSet([a, b]), torch.empty(1, device="cuda")
    other = api.GradientSet([a], into=[into])
    assert grads.holds([a, b]) and not grads.holds([a]) and not grads.holds([b, a]) and not grads.holds([a, into])
    assert not other.holds([a])                      # not in place
    was = b.detach()
    b.data = torch.full((1000,), 7.0, device="cuda")
    assert not grads.holds([a, b]) and grads.holds([a, was])
    del was
    taken = others([4000])
    api.clip_gradients(grads, 1e9, norm)
    assert abs(norm.item() - 5 * 1000 ** 0.5) <= 1e-4 and all(bool((t == 255).all()) for t in taken)
    c = torch.ones((4, 6), device="cuda")
    grads = api.GradientSet([c])
    assert not grads.holds([c.t()]) and not grads.holds([c.view(-1)]) and grads.holds([c])
