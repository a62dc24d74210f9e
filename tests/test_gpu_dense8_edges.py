"""The 8-bit dense layers at the ends of their ranges: the longest operands,
the largest and smallest values, infinities, and what a training loop does
between its steps."""
import numpy as np
import pytest

from paper_2407_18352_amd import _abi, api
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

RELU, IDENT = _abi.ACT_RELU, _abi.ACT_IDENTITY


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def test_the_longest_operands_are_refused():
    """2^31 - 1 rows as far apart as can be described lie in no allocation."""
    import torch
    L, big = _abi.lib(), 2 ** 31 - 1
    layer = api.Linear8(torch.ones((8, 16)))
    x, y, s = (torch.zeros(1 << 12, device="cuda") for _ in range(3))
    args = x.data_ptr(), y.data_ptr(), s.data_ptr()

    def run(kind, n, ldx, ldy):
        return L.hpacml8_linear_run(layer.handle, args[0], kind, ldx, n, args[1], kind, ldy, 0, args[2], 1 << 60, None)

    for kind in (_abi.F32, _abi.BF16):
        assert run(kind, big, big, 8) == _abi.E_RANGE
        assert run(kind, big, 16, big) == _abi.E_RANGE
        assert run(kind, big, big, big) == _abi.E_RANGE
    kept = api.Checkpoint8(2, 32, RELU)
    kept.desc.rows = kept.desc.ld_exps = big
    kept.desc.ld_codes = big // 32 * 32
    assert L.hpacml8_checkpoint_load(kept.desc, args[0], _abi.F32, big, None) == _abi.E_RANGE
    assert L.hpacml8_checkpoint_save(kept.desc, args[0], _abi.F32, big, None, 0, 0, None) == _abi.E_RANGE
    assert L.hpacml8_backward(kept.desc, args[0], _abi.F32, big, 8, args[1], 32, None, 0, None, args[1], big, 0, args[2],
                              1 << 60, None) == _abi.E_RANGE
    torch.cuda.synchronize()
    assert not any(t.any() for t in (x, y, s))
