"""The router with a selection bias in every variant of its kernel: types, widths and numbers of experts.  Tolerances as in
test_gpu_route."""
import math

import pytest
import torch

import moe_reference as ref
import paper_2606_01007_amd as tacg
from test_gpu_route import REL, _check_forward, _gpu, _logits, _near  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("balance", [False, True])
@pytest.mark.parametrize("E, k", [(5, 2), (33, 3), (64, 7), (64, 13), (120, 4), (128, 6), (97, 11), (256, 2), (250, 5), (256, 15)])
def test_bias(dtype, balance, E, k):
    L, N, off = 2, 67, [0, 30, 67]
    for score in ("softmax", "sigmoid"):
        x = _logits(E + k, L, N, E, dtype, mask=0.1, empty=(0, 66))
        bias = torch.randn((L, E), generator=torch.Generator().manual_seed(E)) * 0.5
        out = tacg.route(x.cuda(), k, off, score=score, bias=bias.cuda(), balance=balance)
        ids = _check_forward(x, out, k, off, score, False, 1.0, balance, exact_ids=False)
        p, _, ok = ref.scores(x.double(), score)
        key = torch.where(ok, p + bias.double()[:, None], torch.full_like(p, -math.inf))
        best = torch.sort(key, dim=2, descending=True, stable=True).values[..., :k]
        got = torch.where(ids >= 0, key.gather(2, ids.clamp_min(0)), torch.full_like(best, -math.inf))
        _near(got.float(), best, torch.where(best > -math.inf, 3 * REL, 0.0).double())
        for row in ids.reshape(-1, k).tolist():
            chosen = [e for e in row if e >= 0]
            assert len(set(chosen)) == len(chosen)


@pytest.mark.parametrize("E, k", [(64, 4), (256, 8), (256, 16)])
def test_no_bias_and_a_bias_of_nothing_select_alike(E, k):
    x = torch.round(_logits(1, 2, 100, E, torch.float32) * 8) / 8      # logits whose scores differ by more than their rounding
    a = tacg.route(x.cuda(), k)
    b = tacg.route(x.cuda(), k, bias=torch.zeros((2, E), device="cuda"))
    assert torch.equal(a["trace"], b["trace"]) and torch.equal(a["gate"], b["gate"])


@pytest.mark.parametrize("k", [1, 3, 4, 5, 8, 9, 16])
def test_more_ties_than_a_list_holds(k):
    """Rows with 1 to 40 equal values at and above the k-th place, in all three widths of the list."""
    E, N = 256, 80
    g = torch.Generator().manual_seed(k)
    x = torch.randn((1, N, E), generator=g) - 10.0
    for t in range(N):
        at = torch.randperm(E, generator=g)
        x[0, t, at[:t // 2 + 1]] = 1.0
        x[0, t, at[t // 2 + 1:t // 2 + 1 + t % 3]] = 2.0
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        d = x.to(dtype)
        out = tacg.route(d.cuda(), k, renorm=True, balance=True)
        assert torch.equal(out["trace"].cpu().long(), ref.select(d.double(), k, "softmax"))
