"""Routing limited to groups of experts on the GPU, against 64 bits: the selection is equal, gates, norms, losses and gradients are as near as
those of the router without groups (tests/test_gpu_route.py)."""
import math

import pytest
import torch

import moe_reference as ref
import paper_2606_01007_amd as tacg
from paper_2606_01007_amd.training import balanced_route

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def select(x, k, score, bias, groups, top, best):
    """ids [L][N][k] (-1 where none is left) of x float64 [L][N][E]."""
    p, _, ok = ref.scores(x, score)
    v = p if bias is None else p + bias.double()[:, None, :]
    v = torch.where(ok, v, torch.full_like(v, -math.inf))
    order = x if bias is None else v
    L, N, E = x.shape
    parts = (order if best == 1 else v).reshape(L, N, groups, E // groups)
    first = torch.sort(parts, dim=3, descending=True).values[..., :best]
    there = first > -math.inf
    total = torch.where(there, first, torch.zeros_like(first)).sum(3)
    total = torch.where(there[..., 0], total, torch.full_like(total, -math.inf))
    value, at = torch.sort(total, dim=2, descending=True, stable=True)
    keep = torch.zeros((L, N, groups), dtype=torch.bool).scatter_(2, at[..., :top], value[..., :top] > -math.inf)
    key = torch.where(keep.repeat_interleave(E // groups, 2), order, torch.full_like(order, -math.inf))
    value, at = torch.sort(key, dim=2, descending=True, stable=True)
    return torch.where(value[..., :k] > -math.inf, at[..., :k], torch.full_like(at[..., :k], -1))


def _logits(seed, L, N, E, dtype, drop=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((L, N, E), generator=g) * 1.5
    if drop:
        x[torch.rand(x.shape, generator=g) < drop] = -math.inf
    return x.to(dtype)


def _check(x, k, score, bias, renorm, scale, groups, top, best, off=None):
    L, N, E = x.shape
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = dict(score=score, renorm=renorm, scale=scale, groups=groups, top_groups=top, group_best=best,
              bias=None if bias is None else bias.cuda())
    r = tacg.route(x.cuda(), k, off, err=err, balance=off is not None, want_norm=True, **kw)
    v = x.double()
    ids = select(v, k, score, bias, groups, top, best)
    assert int(err) == 0
    assert torch.equal(r["trace"].cpu().long(), ids)
    gate = ref.gates(v, ids, score, renorm, scale)
    assert ((r["gate"].cpu().double() - gate).abs() <= 2e-5 * gate.abs() + 1e-36).all()
    if off is not None:
        D, tokens, balance, z = ref.losses(v, ids, off, score)
        assert torch.equal(tacg.as_u32(r["D"]).cpu(), D) and torch.equal(tacg.as_u32(r["tokens"]).cpu(), tokens)
        assert ((r["balance"].cpu().double() - balance).abs() <= 2e-5 * balance.abs()).all()
        plain = tacg.route(x.cuda(), k, off, err=err, want_norm=True, **kw)
        assert torch.equal(plain["trace"], r["trace"]) and torch.equal(plain["gate"], r["gate"])
    return r


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("L, N, E, k, groups, top, best", [
    (1, 1, 2, 1, 2, 1, 1),          # the smallest: one expert a group
    (1, 1, 64, 6, 8, 3, 1),         # a decode step
    (1, 1, 256, 8, 8, 4, 2),
    (2, 37, 256, 8, 8, 4, 2),
    (1, 33, 60, 4, 4, 2, 1),        # groups of fifteen
    (1, 65, 60, 4, 4, 1, 2),
    (2, 40, 128, 8, 16, 3, 2),
    (1, 40, 96, 16, 32, 9, 2),      # groups of three, as many as there may be
    (1, 50, 24, 5, 8, 7, 1),
    (1, 50, 7, 3, 7, 4, 2),         # one expert a group: no second
    (1, 50, 250, 10, 2, 1, 1),      # large groups
    (1, 30, 160, 6, 8, 8, 2),       # no limit
    (1, 30, 255, 16, 17, 5, 2),
    (1, 20, 40, 12, 8, 2, 1),       # fewer experts in the groups than slots
    (3, 70, 16, 2, 4, 2, 2),
])
def test_selection(score, dtype, biased, L, N, E, k, groups, top, best):
    x = _logits(L * N + E, L, N, E, dtype)
    bias = 0.2 * torch.randn((L, E), generator=torch.Generator().manual_seed(E)) if biased else None
    if best == 2 and not biased and score == "sigmoid":
        x = x + 4 * 0.25  # sums of the scores of x and -x are 1, whatever x: no such pairs
        x = x.abs().to(dtype)
    _check(x, k, score, bias, E % 2 == 0, 2.5, groups, top, best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("best, biased", [(1, False), (2, False), (1, True), (2, True)])
def test_masks(score, best, biased):
    """Masked experts, groups and rows: a group of one available expert counts that one, a group of none is never kept."""
    x = _logits(5, 2, 90, 48, torch.float32).abs()
    x[torch.rand(x.shape, generator=torch.Generator().manual_seed(6)) < 0.6] = -math.inf
    x[:, 3] = -math.inf
    x[:, 4, 6:] = -math.inf                                            # one group
    x[:, 5, :42] = -math.inf
    x[:, 6, 1:47] = -math.inf                                          # two experts in two groups
    x[:, 7] = torch.finfo(torch.float32).min                           # the lowest value is a logit as any other
    x[:, 8, ::6] = -math.inf
    bias = -0.5 + 0.1 * torch.randn((2, 48), generator=torch.Generator().manual_seed(1)) if biased else None   # values below 0
    for top in (1, 3, 8):
        _check(x, 6, score, bias, True, 1.0, 8, top, best, off=[0, 40, 40, 90])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("biased", [False, True])
def test_ties_go_to_the_lower_number(score, best, biased):
    """Few different values: equal experts and equal groups everywhere, and rows where all are equal."""
    g = torch.Generator().manual_seed(3)
    x = torch.randint(1, 4, (1, 120, 64), generator=g).float() * 0.5
    x[:, 0] = 1.0
    x[:, 1] = -200.0                                                   # scores that 32 bits hold as 0, or not
    bias = torch.randint(0, 2, (1, 64), generator=g).float() * 0.25 if biased else None
    for top in (1, 3, 5):
        _check(x, 8, score, bias, False, 1.0, 8, top, best)
        _check(x.to(torch.bfloat16), 8, score, bias, False, 1.0, 8, top, best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("best", [1, 2])
def test_values_nearer_than_32_bits_can_tell(score, best):
    """Neighbouring 32-bit logits with a bias that nearly undoes their scores' difference."""
    g = torch.Generator().manual_seed(8)
    base = torch.randn((1, 1, 64), generator=g)
    step = torch.randint(-2, 3, (1, 400, 64), generator=g).float()
    x = base + step * 2.0 ** -22
    s, _, _ = ref.scores(base.double(), score)
    bias = (0.3 - s[:, 0]).float()                                     # all sums near 0.3
    for top in (2, 5):
        _check(x, 6, score, bias, True, 1.0, 8, top, best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_far_apart_and_tiny_scores(score, dtype):
    x = _logits(9, 1, 60, 64, dtype) * 40
    bias = 1e-6 * torch.randn((1, 64), generator=torch.Generator().manual_seed(2))
    zero = torch.zeros((1, 64))
    for b in (None, bias, zero):
        for best in (1, 2):
            if b is None and best == 2 and score == "sigmoid":
                continue                                               # 1 - e for many: sums that 64 bits do not order alike
            _check(x.abs() * -1 if score == "sigmoid" else x, 6, score, b, True, 1.0, 8, 3, best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("L, N, E, k, groups, top, off", [
    (2, 300, 256, 8, 8, 4, [0, 100, 101, 300]), (3, 77, 60, 4, 4, 2, [0, 77]), (1, 700, 64, 6, 8, 3, [0, 0, 512, 700]),
    (1, 2, 32, 2, 4, 1, [0, 1, 2]),
])
def test_counts_and_losses(score, L, N, E, k, groups, top, off):
    bias = 0.05 * torch.randn((L, E), generator=torch.Generator().manual_seed(E))
    for b, best, dtype in ((None, 1, torch.float32), (bias, 2, torch.float32), (bias, 2, torch.bfloat16)):
        r = _check(_logits(N, L, N, E, dtype), k, score, b, True, 2.5, groups, top, best, off)
        # the trace is one that the counting takes
        D, _, err = tacg.coact_build(r["trace"], off, E)
        assert torch.equal(D, r["D"]) and int(err) == 0


def test_invalid_rows_are_not_routed():
    x = _logits(2, 1, 50, 64, torch.float32)
    x[0, 7, 3], x[0, 8, 63] = math.nan, math.inf
    for bias in (None, torch.zeros((1, 64), device="cuda")):
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        r = tacg.route(x.cuda(), 4, bias=bias, groups=8, top_groups=2, err=err)
        assert int(err) == tacg.ERR_VALUE
        assert (r["trace"][0, 7:9] == -1).all() and not r["gate"][0, 7:9].any()
        assert (r["trace"][0, :7] >= 0).all() and (r["trace"][0, 9:] >= 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strided_logits(dtype):
    base = _logits(6, 3, 40, 70, dtype).cuda()
    for view in (base[:, :, 3:67], base[1:, ::2, :64], base.transpose(0, 1)[:, :, :64]):
        a = tacg.route(view, 5, groups=4, top_groups=2, group_best=2)
        b = tacg.route(view.contiguous(), 5, groups=4, top_groups=2, group_best=2)
        assert torch.equal(a["trace"], b["trace"]) and torch.equal(a["gate"], b["gate"])


def test_one_group_is_the_router():
    x = _logits(6, 2, 40, 64, torch.float32).cuda()
    bias = 0.1 * torch.randn((2, 64), generator=torch.Generator().manual_seed(1)).cuda()
    for b in (None, bias):
        p, q = tacg.route(x, 5, bias=b, renorm=True), tacg.route(x, 5, bias=b, renorm=True, groups=1, top_groups=1)
        assert torch.equal(p["trace"], q["trace"]) and torch.equal(p["gate"], q["gate"])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [False, True])
def test_gradient(score, biased):
    """Through balanced_route, against the formula, and against differences where the selection does not change."""
    L, N, E, k, off = 2, 40, 24, 4, [0, 15, 40]
    g = torch.Generator().manual_seed(4)
    x = torch.randn((L, N, E), generator=g)
    bias = 0.1 * torch.randn((L, E), generator=g) if biased else None
    gg, gb, gz = torch.randn((L, N, k), generator=g), torch.randn((2, L), generator=g), torch.randn((2, L), generator=g)
    dx = x.cuda().requires_grad_(True)
    kw = dict(score=score, renorm=True, scale=1.5, groups=4, top_groups=2, group_best=2)
    gate, balance, z, r = balanced_route(dx, k, off, bias=None if bias is None else bias.cuda(), **kw)
    ((gate * gg.cuda()).sum() + (balance * gb.cuda()).sum() + (z * gz.cuda()).sum()).backward()
    ids = select(x.double(), k, score, bias, 4, 2, 2)
    assert torch.equal(r["trace"].cpu().long(), ids)
    zed = gz.double() if score == "softmax" else None
    want, mag = ref.gradient(x.double(), ids, off, score, True, 1.5, gg.double(), gb.double(), zed)
    assert ((dx.grad.cpu().double() - want).abs() <= 5e-5 * mag).all()
    value = lambda v: float(ref.total(v, ids, off, score, True, 1.5, gg.double(), gb.double(), zed))  # noqa: E731
    h = 1e-6
    for l, t, e in ((0, 0, 0), (1, 39, 23), (0, 17, int(ids[0, 17, 0])), (1, 3, int(ids[1, 3, 3]))):
        up, down = x.double(), x.double()
        up[l, t, e] += h
        down[l, t, e] -= h
        d = (value(up) - value(down)) / (2 * h)
        assert abs(d - float(dx.grad[l, t, e])) <= 1e-6 + 5e-5 * float(mag[l, t, e])


def test_captured_and_replayed():
    L, N, E, k, off = 2, 300, 64, 6, [0, 120, 300]
    x = torch.zeros((L, N, E), device="cuda")
    bias = 0.05 * torch.randn((L, E), generator=torch.Generator().manual_seed(1)).cuda()
    kw = dict(score="sigmoid", bias=bias, renorm=True, balance=True, groups=8, top_groups=4)
    out = tacg.route(x, k, off, **kw)
    ws = tacg.workspace(tacg.lib().tacg_route_workspace_bytes(N, L, E, 2))
    err = out.pop("err")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tacg.route(x, k, off, out=out, err=err, ws=ws, **kw)
    for i in range(4):
        x.copy_(_logits(i, L, N, E, torch.float32).cuda())
        graph.replay()
        torch.cuda.synchronize()
        want = tacg.route(x, k, off, **kw)
        torch.cuda.synchronize()
        for n in ("trace", "gate", "D", "tokens", "balance", "norm"):
            assert torch.equal(out[n], want[n]), n


def test_other_stream():
    x = _logits(1, 1, 200, 64, torch.float32).cuda()
    want = tacg.route(x, 4, groups=8, top_groups=2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = tacg.route(x, 4, groups=8, top_groups=2, stream=side)
    side.synchronize()
    assert torch.equal(got["trace"], want["trace"]) and torch.equal(got["gate"], want["gate"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_equal_neighbours_with_equal_and_other_biases(dtype, score):
    """Lists whose neighbours have equal logits: with equal biases they are in order as they are, with others 64 bits tell."""
    g = torch.Generator().manual_seed(12)
    x = (torch.randn((2, 300, 128), generator=g) * 2).mul(8).round().div(8).to(dtype)     # many equal pairs, few a row
    for bias in (torch.zeros((2, 128)), torch.full((2, 128), -0.25), 2.0 ** -23 * torch.randint(-2, 3, (2, 128), generator=g).float(),
                 torch.where(torch.rand((2, 128), generator=g) < 0.5, 0.0, 2.0 ** -24)):
        for best in (1, 2):
            _check(x, 8, score, bias, True, 1.0, 8, 4, best)
