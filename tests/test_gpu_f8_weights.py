"""GPU tests of LinearF8's weights: whatever the constructor takes, update takes,
with the same codes; on a stream of its own only what is read where it lies."""
import numpy as np
import pytest
import torch

from paper_2407_18352_amd import api
from test_gpu_f8 import loaded

pytestmark = pytest.mark.gpu

FORMS = {
    "float16": lambda t: t.half().cuda(), "float64": lambda t: t.double().cuda(), "float64 on the CPU": lambda t: t.double(),
    "float32": lambda t: t.cuda(), "bfloat16": lambda t: t.bfloat16().cuda(), "int32": lambda t: (t * 4).int().cuda(),
    "numpy float64": lambda t: t.double().numpy(), "numpy float32": lambda t: t.numpy(), "bfloat16 on the CPU": lambda t: t.bfloat16(),
    "a parameter": lambda t: t.cuda().requires_grad_(),
}


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("bias", [True, False])
def test_update_takes_what_the_constructor_takes(form, bias):
    g = torch.Generator().manual_seed(1)
    W, b = FORMS[form](torch.randn((70, 200), generator=g)), FORMS[form](torch.randn(70, generator=g)) if bias else None
    made = api.LinearF8(W, b, learn=True)
    other = api.LinearF8(torch.zeros((70, 200)), torch.zeros(70) if bias else None, learn=True)
    other.update(W, b)
    want = api.LinearF8(torch.as_tensor(np.asarray(W)).float() if isinstance(W, np.ndarray) else W.detach().float(),
                        None if b is None else torch.as_tensor(np.asarray(b)).float() if isinstance(b, np.ndarray) else b.detach().float(), learn=True)
    for layer in (made, other):
        assert torch.equal(loaded(layer.W), loaded(want.W)) and torch.equal(loaded(layer.Wt), loaded(want.Wt))
        assert layer.b is None if b is None else torch.equal(layer.b, want.b)


def test_weights_in_other_orders():
    W = torch.randn((200, 70), generator=torch.Generator().manual_seed(2))
    layer, want = api.LinearF8(torch.zeros((70, 200)), learn=True), api.LinearF8(W.t().contiguous(), learn=True)
    for t in (W.cuda().t(), W.double().cuda().t(), W.t(), torch.cat([W, W], 1).cuda()[:, 70:].t()):
        layer.update(t)
        assert torch.equal(loaded(layer.W), loaded(want.W)) and torch.equal(loaded(layer.Wt), loaded(want.Wt))


def test_a_stream_of_its_own_takes_what_lies_ready():
    layer, s = api.LinearF8(torch.zeros((8, 16))), torch.cuda.Stream()
    W = torch.randn((8, 16), device="cuda")
    torch.cuda.synchronize()
    for t in (W.double(), W.half(), W.cpu(), W.t().contiguous().t(), W.cpu().numpy()):
        with pytest.raises(ValueError):
            layer.update(t, stream=s)
    for t in (W, W.bfloat16()):
        torch.cuda.synchronize()
        layer.update(t, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(loaded(layer.W), loaded(api.LinearF8(t).W))
    with pytest.raises(ValueError):
        layer.update(W[:, :8])
    with pytest.raises(ValueError):
        layer.update(W, torch.zeros(8, device="cuda"))
