"""The example that joins router, trace, placement and experts, and the router under automatic differentiation."""
import importlib.util
import os

import pytest
import torch

import moe_reference as ref
import paper_2606_01007_amd as tacg
from paper_2606_01007_amd.training import balanced_route

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_example():
    spec = importlib.util.spec_from_file_location("moe_layer", os.path.join(ROOT, "examples", "moe_layer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    out = example.run(say=lambda *_: None)
    assert out["balance"][-1] < out["balance"][0]
    assert sum(out["load"]) == out["pairs"]
    # every share is rounded to bfloat16 once, and so is the whole: 2^-8 of values no larger than a few times their sum
    assert out["off"] < 4 * 2.0 ** -8


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_balanced_route_is_differentiable(score):
    L, N, E, k, off = 2, 40, 24, 4, [0, 15, 40]
    x = torch.randn((L, N, E), generator=torch.Generator().manual_seed(3))
    g = torch.Generator().manual_seed(4)
    gg, gb, gz = torch.randn((L, N, k), generator=g), torch.randn((2, L), generator=g), torch.randn((2, L), generator=g)
    dx = x.cuda().requires_grad_(True)
    gate, balance, z, r = balanced_route(dx, k, off, score=score, renorm=True, scale=1.5)
    ((gate * gg.cuda()).sum() + (balance * gb.cuda()).sum() + (z * gz.cuda()).sum()).backward()
    ids = r["trace"].cpu().long()
    want, mag = ref.gradient(x.double(), ids, off, score, True, 1.5, gg.double(), gb.double(),
                             gz.double() if score == "softmax" else None)
    assert ((dx.grad.cpu().double() - want).abs() <= 5e-5 * mag).all()
    plain = tacg.route(x.cuda(), k, off, score=score, renorm=True, scale=1.5, balance=True)
    assert torch.equal(plain["gate"], gate) and torch.equal(plain["balance"], balance)
    only = x.cuda().requires_grad_(True)
    balanced_route(only, k, off, score=score)[1].sum().backward()      # the other outputs have no gradient
    want, mag = ref.gradient(x.double(), ref.select(x.double(), k, score), off, score, False, 1.0, None,
                             torch.ones((2, L), dtype=torch.float64))
    assert ((only.grad.cpu().double() - want).abs() <= 5e-5 * mag).all()
