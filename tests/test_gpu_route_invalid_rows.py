"""Gradients of rows that are not routed: a NaN or +inf logit makes a row one without available experts, in both scores and for every
gradient, and leaves the other rows as they are."""
import math

import pytest
import torch

import paper_2606_01007_amd as tacg
from test_gpu_route import _gpu, _logits, _upstream  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [math.nan, -math.nan, math.inf])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E, k", [(60, 4), (61, 3), (256, 12)])
def test_gradient_of_rows_without_logits(score, dtype, bad, E, k):
    L, N, off = 2, 40, [0, 33, 40]
    x = _logits(5, L, N, E, dtype)
    x[1, 7, E - 1] = bad
    x[0, 33, 0] = bad
    x[0, 39, :] = bad
    rows = ((1, 7), (0, 33), (0, 39))
    clean = x.clone()
    for row in rows:
        clean[row] = -math.inf
    gg, gb, gz = (None if v is None else v.cuda() for v in _upstream(3, L, N, k, 2, score))
    for renorm in (False, True):
        out, want = (tacg.route(v.cuda(), k, off, score=score, renorm=renorm, balance=True) for v in (x, clean))
        assert int(out["err"].item()) == tacg.ERR_VALUE and int(want["err"].item()) == 0
        for name in ("trace", "gate", "norm", "D", "tokens", "balance") + (("z",) if score == "softmax" else ()):
            assert torch.equal(out[name], want[name]), name
        for up in ((gg, None, None), (None, gb, None), (None, None, gz), (gg, gb, gz)):
            a, b = (tacg.route_backward(v.cuda(), r["trace"], r["norm"], off, D=r["D"], tokens=r["tokens"], grad_gate=up[0],
                                        grad_balance=up[1], grad_z=up[2], score=score, renorm=renorm)
                    for v, r in ((x, out), (clean, want)))
            for row in rows:
                assert not a[row].any()              # a NaN counts as true here
            assert torch.equal(a, b)                 # and differs from itself here
