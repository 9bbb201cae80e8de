"""The 64-bit forms that the router's and the products' tests compare with: the gradient's formula against differences of the losses
and against automatic differentiation, and the layout of the 4-bit weights against a byte-by-byte reading."""
import math

import pytest
import torch

import moe_reference as ref


def _case(seed, L, N, E, k, score, mask):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((L, N, E), generator=g, dtype=torch.float64) * 2
    if mask:
        x[torch.rand((L, N, E), generator=g) < 0.3] = -math.inf
        x[:, N // 2] = -math.inf
    ids = ref.select(x, k, score)
    off = [0, N // 3, N // 3, N]
    gg = torch.randn((L, N, k), generator=g, dtype=torch.float64)
    gb = torch.randn((3, L), generator=g, dtype=torch.float64)
    gz = torch.randn((3, L), generator=g, dtype=torch.float64) if score == "softmax" else None
    return x, ids, off, gg, gb, gz


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("E, k", [(1, 1), (5, 2), (9, 4)])
def test_gradient_formula(score, renorm, mask, E, k):
    x, ids, off, gg, gb, gz = _case(E, 2, 7, E, k, score, mask)
    want, mag = ref.gradient(x, ids, off, score, renorm, 1.5, gg, gb, gz)
    assert torch.isfinite(want).all() and (want[x == -math.inf] == 0).all() and (mag >= want.abs() * (1 - 1e-12)).all()
    h = 1e-6
    for i in range(0, x.numel(), 3):
        at = (i // (7 * E), i // E % 7, i % E)
        if x[at] == -math.inf:
            continue
        hi, lo = x.clone(), x.clone()
        hi[at] += h
        lo[at] -= h
        args = (ids, off, score, renorm, 1.5, gg, gb, gz)
        slope = (ref.total(hi, *args) - ref.total(lo, *args)) / (2 * h)
        # the third derivative times h^2, and the rounding of numbers of magnitude 1 over h
        assert abs(float(slope - want[at])) < 1e-7 * (1 + float(gg.abs().max()) + float(gb.abs().max())) * 10


def test_gradient_against_automatic_differentiation():
    for score in ("softmax", "sigmoid"):
        x, ids, off, gg, gb, gz = _case(3, 2, 8, 6, 3, score, False)
        x.requires_grad_(True)
        ref.total(x, ids, off, score, True, 0.7, gg, gb, gz).backward()
        want, _ = ref.gradient(x.detach(), ids, off, score, True, 0.7, gg, gb, gz)
        assert torch.allclose(x.grad, want, rtol=1e-10, atol=1e-13)


def test_selection_order():
    x = torch.tensor([[1.0, 3.0, 3.0, -math.inf, 0.0, -0.0]], dtype=torch.float64)
    assert ref.select(x, 6, "softmax").tolist() == [[1, 2, 0, 4, 5, -1]]
    bias = torch.tensor([9.0, 0, 0, 99.0, 0, 0], dtype=torch.float64)
    assert ref.select(x, 2, "sigmoid", bias).tolist() == [[0, 1]]


def test_weights_layout():
    q = torch.tensor([[[0x21, 0x43] + [0] * 14]], dtype=torch.uint8)
    s = torch.tensor([[[0.5]]], dtype=torch.float16)
    assert ref.dequantise(q, s, None, 3, 32).tolist() == [[[-3.5, -3.0, -2.5]]]
    z = torch.tensor([[[1]]], dtype=torch.uint8)
    assert ref.dequantise(q, s, z, 4, 32).tolist() == [[[0.0, 0.5, 1.0, 1.5]]]
