"""Sigmoid scores whose sums are close to the smallest 32-bit number, where a reciprocal of the sum times a gradient or a scale, or a
score times a gradient, would not be a normal 32-bit number any more.

Tolerances: as in test_gpu_route, where the logits' range is 40; here it is 88, so a score is off by 88 * 2^-24 * 2 + 64 * 2^-24 < 2 REL."""
import math

import pytest
import torch

import moe_reference as ref
import paper_2606_01007_amd as tacg
from test_gpu_route import HALF, REL, TINY, _gpu, _near  # noqa: F401

pytestmark = pytest.mark.gpu


def _low(seed, N, E, dtype):
    """Logits from -87.2 to -84: their sigmoids are from 1.3e-38 to 3.3e-37 and normal 32-bit numbers."""
    x = torch.rand((1, N, E), generator=torch.Generator().manual_seed(seed)) * 3.2 - 87.2
    if E > 2:
        x[0, ::3, 1] = -math.inf
    x[0, 0] = -87.0
    return x.to(dtype).clamp_min(-math.inf if E > 2 else -87.2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("E, k", [(2, 1), (2, 2), (8, 1), (8, 4), (24, 10)])
def test_small_sigmoid_scores(E, k, renorm, dtype):
    N, off, scale = 20, [0, 1, 2, 20], 8.0
    x = _low(E + k, N, E, dtype)
    assert float(x[x > -math.inf].min()) > -87.3
    out = tacg.route(x.cuda(), k, off, score="sigmoid", renorm=renorm, scale=scale, balance=True)
    ids = out["trace"].cpu().long()
    assert torch.equal(ids, ref.select(x.double(), k, "sigmoid"))
    want = ref.gates(x.double(), ids, "sigmoid", renorm, scale)
    _near(out["gate"], want, 2 * REL * want + 1e-44)
    _, _, balance, _ = ref.losses(x.double(), ids, off, "sigmoid")
    _near(out["balance"], balance, 2 * REL * balance)
    g = torch.Generator().manual_seed(E)
    gg, gb = torch.randn((1, N, k), generator=g), torch.randn((3, 1), generator=g)
    for up in ((30 * gg, None), (None, 50 * gb), (30 * gg, 50 * gb), (1e-5 * gg, None), (None, 1e-5 * gb)):
        wide = [None if v is None else v.double() for v in up]
        cuda = [None if v is None else v.cuda() for v in up]
        got = tacg.route_backward(x.cuda(), out["trace"], out["norm"], off, D=out["D"], tokens=out["tokens"], grad_gate=cuda[0],
                                  grad_balance=cuda[1], score="sigmoid", renorm=renorm, scale=scale)
        want, mag = ref.gradient(x.double(), ids, off, "sigmoid", renorm, scale, *wide)
        _near(got, want, 10 * REL * mag + HALF[dtype] * (1 + 1e-4) * want.abs() + TINY[dtype])
