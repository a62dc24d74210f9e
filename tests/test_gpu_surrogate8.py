"""A surrogate learned with its activations kept in 8 bits and answering in 8
bits: gradients against automatic differentiation in fp32, and the command."""
import numpy as np
import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("dims, n", [((9, 64, 64, 1), 257), ((36, 128, 200, 4), 1000), ((5, 256, 1), 33)])
def test_gradients_near_automatic_differentiation(dims, n):
    import torch
    from paper_2407_18352_amd.surrogate8 import Surrogate8
    m = Surrogate8(dims, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    x, t = torch.randn((n, dims[0]), generator=g, device="cuda"), torch.randn((n, dims[-1]), generator=g, device="cuda")
    off = m.forward(x) - t
    m.backward(off * (2 / off.numel()))
    ws = [w.detach().clone().requires_grad_() for w in m.W]
    bs = [b.detach().clone().requires_grad_() for b in m.b]
    a = x
    for i, (w, b) in enumerate(zip(ws, bs)):
        a = torch.nn.functional.linear(a, w, b)
        a = torch.relu(a) if i + 1 < len(ws) else a
    ((a - t) ** 2).mean().backward()
    # bf16 products and activations (2^-9 each, relative) and kept activations
    # (2^-9 of a block's largest) through len(ws) layers: a few per cent of
    # the gradients' norm at most
    for p, q in zip(m.parameters(), ws + bs):
        d = (p.grad - q.grad).norm() / q.grad.norm()
        assert d < 0.05, d


def test_accumulated_batches_equal_their_sum():
    import torch
    from paper_2407_18352_amd.surrogate8 import Surrogate8
    m = Surrogate8((6, 64, 1), seed=1)
    x, dy = torch.randn((300, 6), device="cuda"), torch.randn((300, 1), device="cuda") / 300
    parts = []
    for s in (slice(0, 100), slice(100, 300)):
        m.forward(x[s])
        m.backward(dy[s])
        parts.append([p.grad.clone() for p in m.parameters()])
    m.forward(x[:100])
    m.backward(dy[:100])
    m.forward(x[100:])
    m.backward(dy[100:], accumulate=True)
    for p, a, b in zip(m.parameters(), *parts):
        assert torch.allclose(p.grad, a + b, rtol=0, atol=2.0 ** -22 * float((a.abs() + b.abs()).max()))


def test_the_command_learns_and_answers(capsys):
    from paper_2407_18352_amd import surrogate8
    learned, answered = surrogate8.main(["--points", "8192", "--dims", "5,128,128,1", "--steps", "150"])
    assert np.isfinite([learned, answered]).all()
    # the prices' spread is 1: an untrained model is off by about that
    assert learned < 0.2 and answered < learned + 0.1
