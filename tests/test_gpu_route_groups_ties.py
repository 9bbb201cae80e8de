"""Routing limited to groups where the last that is chosen and the first that is not are equal, and others behind them are larger by less than
32 bits can tell: the selection is that of 64 bits (test_gpu_route_groups.select), gates are as near as there."""
import math

import pytest
import torch

import paper_2606_01007_amd as tacg
from test_gpu_route_groups import _check, _gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def _rows(seed, n, E, k, value, step, first=None, before=0):
    """n rows whose experts are all in one half: `before` of the logit `value` + 1 at the lowest ids (bias makes them larger), then k + 1 or
    more of `value`, and behind them some of `value` - step or + step.  first: the logit of one more, at id 0 of the half."""
    g = torch.Generator().manual_seed(seed)
    room = 16 if k < 8 else 2 * k                      # what is ordered without further doubt
    x = torch.full((1, n, E), -math.inf)
    for r in range(n):
        at = int(torch.randint(0, 2, (), generator=g)) * (E // 2)
        lead = before + (first is not None)
        free = torch.randperm(E // 2 - lead, generator=g)[:room - lead].sort().values + lead + at
        m = int(torch.randint(k + 1 - lead, room - lead + 1, (), generator=g))
        same = int(torch.randint(k + 1 - lead, m + 1, (), generator=g))
        ids = free[torch.randperm(free.numel(), generator=g)[:m].sort().values]
        v = value + step * torch.randint(-1, 2, (m,), generator=g)
        v[:same] = value
        x[0, r, ids] = v.float()
        x[0, r, at:at + before] = value + 1
        if first is not None:
            x[0, r, at + before] = first
        x[0, r, E // 2 - at:E - at] = -200.0           # the other half's
    return x


def _bias(E, value, before=0):
    b = torch.full((1, E), value)
    b[0, :before] += 0.25
    b[0, E // 2:E // 2 + before] += 0.25
    return b


def test_a_larger_one_behind_two_equal_ones():
    x = torch.tensor([[[20.0, 20, 21, -5, -5, -5, -5, -5], [-5, -5, -5, -5, 20, 20, 20, 21], [20, 20, 20, 20, -5, -5, -5, -5],
                       [20, 21, 20, 21, -5, -5, -5, -5], [20, 20, 19, 21, -5, -5, -5, -5]]])
    for bias in (0.0, 0.5, -3.0):
        r = tacg.route(x.cuda(), 1, score="sigmoid", bias=torch.full((1, 8), bias, device="cuda"), groups=2, top_groups=1, group_best=1)
        assert r["trace"].flatten().tolist() == [2, 7, 0, 1, 3]


@pytest.mark.parametrize("k", [1, 3, 4, 7, 8, 12, 16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("groups, top, best", [(2, 1, 1), (2, 1, 2), (8, 8, 2), (24, 24, 1)])
def test_equal_ones_on_both_sides_of_the_last_place(k, dtype, groups, top, best):
    E, n = 96, 150
    off = [0, 70, n]
    for bias in (0.0, 0.5):                                            # sigmoid scores that 32 bits hold as 1
        _check(_rows(k, n, E, k, 20, 1).to(dtype), k, "sigmoid", _bias(E, bias), True, 2.5, groups, top, best, off)
        if k > 2:
            x = _rows(k, n, E, k, 20, 1, before=2).to(dtype)
            _check(x, k, "sigmoid", _bias(E, bias, before=2), True, 2.5, groups, top, best, off)
    # scores that vanish next to their bias, or are below the normal range
    _check(_rows(k, n, E, k, -30, 1).to(dtype), k, "sigmoid", _bias(E, 0.5), False, 1.0, groups, top, best)
    if k > 1:
        _check(_rows(k, n, E, k, -30, 1, first=0.0).to(dtype), k, "softmax", _bias(E, 0.5), False, 1.0, groups, top, best)
        _check(_rows(k, n, E, k, -110, 1, first=0.0).to(dtype), k, "softmax", _bias(E, 0.0), False, 1.0, groups, top, best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("k", [1, 4, 8, 16])
def test_equal_logits_with_biases_that_32_bit_sums_do_not_show(score, k):
    """All logits of a row's choice are equal; behind the last place some have a bias that is larger by one step of the bias."""
    E, n = 64, 60
    g = torch.Generator().manual_seed(k)
    x = torch.full((1, n, E), -20.0)
    bias = torch.full((1, E), 2.0 ** -4)
    bias[0, 20:32] += 2.0 ** -27                       # one step of the bias, an eighth of half a step of sums of 1 or more
    for r in range(n):
        low = torch.randperm(20, generator=g)[:k + 1]
        high = 20 + torch.randperm(12, generator=g)[:int(torch.randint(0, 4, (), generator=g))]
        x[0, r, torch.cat([low, high])] = 20.0 if score == "sigmoid" else -1.0
    for dtype in (torch.float32, torch.bfloat16):
        _check(x.to(dtype), k, score, bias, True, 1.0, 2, 1, 2)
