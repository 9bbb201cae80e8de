"""A token's products do not depend on the values of the other tokens, whatever these are: with the same routing its bits stay."""
import math

import pytest
import torch

from test_gpu_q4 import _gpu, _inputs, _routed, _run, _weights  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("T, E, k, K", [(2, 16, 2, 512), (3, 40, 4, 200), (50, 16, 4, 512), (67, 2, 2, 296), (200, 8, 2, 256)])
def test_values_of_other_tokens(T, E, k, K, mode, dtype):
    N, group = 96, 64
    for zeros in (False, True):
        w = _weights(7, E, N, K, group, dtype, zeros)
        ids = _routed(7, T, E, k)
        x, gate = _inputs(7, T, k, K, mode, dtype)
        first = _run(x, ids, w, group, mode, E, gate=gate)
        assert torch.isfinite(first).all()
        other = x.clone()
        other[1::2] = _inputs(8, T, k, K, mode, dtype)[0][1::2] * 100
        other[1, ..., K - 1] = math.inf
        other[T // 2 | 1 if T > 3 else 1, ..., 0] = math.nan
        got = _run(other, ids, w, group, mode, E, gate=gate)
        assert torch.equal(got[::2], first[::2])
        assert torch.isnan(got[1]).all()                   # the offset of the levels is subtracted: an infinity ends as NaN


def test_values_of_other_slots():
    """Slots with values of their own: those of experts that are held elsewhere are not read into the sum."""
    T, E, k, K, N = 30, 12, 4, 288, 64
    w = _weights(3, 3, N, K, 32, torch.bfloat16, False)
    slot = torch.full((E,), -1, dtype=torch.int32)
    slot[::4] = torch.arange(3, dtype=torch.int32)
    for few in (False, True):
        t = 2 if few else T
        ids = _routed(3, t, E, k)
        x, gate = _inputs(3, t, k, K, "sum", torch.bfloat16)
        first = _run(x, ids, w, 32, "sum", E, slot=slot, gate=gate)
        x[slot[ids.long()] < 0] = math.nan
        gate[slot[ids.long()] < 0] = math.nan
        assert torch.isfinite(first).all() and torch.equal(first, _run(x, ids, w, 32, "sum", E, slot=slot, gate=gate))
