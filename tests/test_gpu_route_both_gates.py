"""The router and its gradient at the sizes of test_router_and_gradient, with the other of the two forms of the gates, so that each (E, k,
type, score) runs with and without renormalisation, lists of more than eight ids a row among them."""
import pytest
import torch

import paper_2606_01007_amd as tacg
from test_gpu_route import _check_backward, _check_forward, _gpu, _logits, _upstream  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E, k", [(1, 1), (2, 2), (7, 3), (8, 8), (33, 4), (60, 4), (61, 9), (64, 6), (65, 1), (128, 8), (130, 16),
                                  (200, 10), (255, 7), (256, 8), (256, 16)])
def test_router_and_gradient_in_the_other_form(dtype, score, E, k):
    L, N, renorm = 2, 71, (E + k) % 2 != 0
    off = [0, 5, 5, 40, 71]
    x = _logits(E * 100 + k, L, N, E, dtype, mask=0.1 if E > 8 else 0.0, empty=(0, 39, 70))
    dx = x.cuda()
    out = tacg.route(dx, k, off, score=score, renorm=renorm, scale=1.5, balance=True)
    ids = _check_forward(x, out, k, off, score, renorm, 1.5, True)
    gg, gb, gz = _upstream(E, L, N, k, 4, score)
    _check_backward(x, dx, out, ids, off, score, renorm, 1.5, (gg, gb, gz))
    _check_backward(x, dx, out, ids, off, score, renorm, 1.5, (gg, None, None))
    assert int(out["err"].item()) == 0
