"""The experts' products with many pairs: every number of weight rows a wave and of token tiles that the sizes choose, lists over several
runs of pairs, and pairs at the rules' edges.  Tolerances as in test_gpu_q4."""
import math

import pytest
import torch

import moe_reference as ref
from test_gpu_q4 import HALF, TINY, _gpu, _inputs, _routed, _run, _weights  # noqa: F401

pytestmark = pytest.mark.gpu


def _reference(x, ids, w, group, mode, slot=None, gate=None):
    """products() of moe_reference, expert by expert."""
    T, k = ids.shape
    q, s, z = (None if v is None else v.cuda() for v in w)
    x = x.cuda()
    K, (H, N) = x.shape[-1], q.shape[:2]
    y = torch.zeros((T, k, N), dtype=torch.float64, device="cuda")
    off = torch.zeros_like(y)
    for e in torch.unique(ids).tolist():
        h = -1 if e < 0 else e if slot is None else int(slot[e])
        if h < 0:
            continue
        one = ref.dequantise(q[h:h + 1], s[h:h + 1], None if z is None else z[h:h + 1], K, group)[0]
        wide = s[h].double().abs().repeat_interleave(group, 1)[:, :K]
        t, j = torch.nonzero(ids == e, as_tuple=True)
        t, j = t.cuda(), j.cuda()
        v = (x[t, j] if x.dim() == 3 else x[t]).double()
        y[t, j] = v @ one.t().contiguous()
        off[t, j] = 16 * 2.0 ** -24 * 151 * (v.abs() @ wide.t().contiguous())
    if mode == "glu":
        a, b, da, db = y[..., :N // 2], y[..., N // 2:], off[..., :N // 2], off[..., N // 2:]
        g = a * torch.sigmoid(a)
        return g * b, 1.1 * da * b.abs() + g.abs() * db + 1.1 * da * db + 2.0 ** -20 * (g * b).abs()
    if mode == "sum":
        g = gate.cuda().double().unsqueeze(-1)
        return (g * y).sum(1), (g * off).sum(1) + 16 * 2.0 ** -24 * (g * y).abs().sum(1)
    return y, off


def _check(got, x, ids, w, group, mode, slot=None, gate=None):
    want, off = _reference(x, ids, w, group, mode, slot, gate)
    assert got.shape == want.shape
    d = (got.double() - want).abs()
    tol = off * (1 + HALF[x.dtype]) + HALF[x.dtype] * (1 + 1e-6) * want.abs() + TINY[x.dtype]
    assert not torch.isnan(d).any() and float((d - tol).max()) <= 0, float((d / tol).max())


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("group, zeros", [(32, False), (32, True), (64, False), (64, True), (128, False), (128, True), (256, False),
                                          (256, True)])
def test_every_shape_of_workgroup(mode, dtype, group, zeros):
    K = 512 if group == 256 else 640
    for T, E, k, N in ((40, 128, 4, 250),       # one tile of tokens, 32 rows a wave
                       (400, 128, 4, 250),      # two tiles, 32 rows
                       (600, 128, 8, 1000),     # two tiles, 64 rows; more pairs than one list holds
                       (12, 8, 2, 130),         # one tile, 16 rows
                       (60, 8, 2, 130)):        # two tiles, 16 rows
        w = _weights(T + group, E, N, K, group, dtype, zeros)
        ids = _routed(T, T, E, k)
        x, gate = _inputs(T, T, k, K, mode, dtype)
        _check(_run(x, ids, w, group, mode, E, gate=gate), x, ids, w, group, mode, gate=gate)


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("K", [200, 256, 257, 300, 511, 512, 513, 777])
def test_ends_of_the_columns(mode, K):
    for T, E, k, group in ((2, 32, 3, 64), (30, 8, 2, 64), (90, 8, 2, 128)):
        w = _weights(K, E, 70, K, group, torch.bfloat16, K % 2 == 1)
        ids = _routed(K, T, E, k)
        x, gate = _inputs(K, T, k, K, mode, torch.bfloat16)
        _check(_run(x, ids, w, group, mode, E, gate=gate), x, ids, w, group, mode, gate=gate)


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
def test_tokens_of_an_expert_at_the_edges_of_a_tile(mode):
    """Experts with 0, 1, 2, 3, 15, 16, 17, 31, 32, 33, 34, 35 and 70 tokens in one call."""
    counts = [0, 1, 2, 3, 15, 16, 17, 31, 32, 33, 34, 35, 70]
    T, E, N, K, group = sum(counts), len(counts), 66, 320, 64
    ids = torch.repeat_interleave(torch.arange(E), torch.tensor(counts))
    ids = ids[torch.randperm(T, generator=torch.Generator().manual_seed(1))].to(torch.int16).reshape(T, 1)
    w = _weights(4, E, N, K, group, torch.float16, True)
    x, gate = _inputs(4, T, 1, K, mode, torch.float16)
    _check(_run(x, ids, w, group, mode, E, gate=gate), x, ids, w, group, mode, gate=gate)


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
def test_a_share_over_several_runs_of_pairs(mode):
    E, k, N, K, group, T = 64, 8, 96, 256, 32, 1100
    slot = torch.full((E,), -1, dtype=torch.int32)
    slot[3::4] = torch.arange(16, dtype=torch.int32)
    w = _weights(8, 16, N, K, group, torch.bfloat16, False)
    ids = _routed(8, T, E, k, unused=0.1)
    x, gate = _inputs(8, T, k, K, mode, torch.bfloat16)
    _check(_run(x, ids, w, group, mode, E, slot=slot, gate=gate), x, ids, w, group, mode, slot=slot, gate=gate)


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("N, K", [(256, 320), (248, 300), (70, 512), (2, 256)])
@pytest.mark.parametrize("held", [0, 1, 3, 5])
def test_many_tokens_of_few_experts(mode, N, K, held):
    """Small grids, whose experts' tiles of tokens go to several workgroups; rows without a held expert are zero, into memory that was
    not, at an address that holds 16 bytes' alignment and at one that does not."""
    T, E, k, group = 333, 5, 2, 64
    slot = torch.tensor([3, -1, 0, 2, 1] if held == 5 else [v if v < held else -1 for v in (2, 4, 0, 3, 1)], dtype=torch.int32)
    w = _weights(N + held, held, N, K, group, torch.bfloat16, held == 3)
    ids = _routed(held, T, E, k, unused=0.05)
    x, gate = _inputs(held, T, k, K, mode, torch.bfloat16)
    shape = {"each": (T, k, N), "glu": (T, k, N // 2), "sum": (T, N)}[mode]
    size = math.prod(shape)
    for skip in (0, 1):
        room = torch.full((skip + size + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
        out = room[skip:skip + size].view(shape)
        _run(x, ids, w, group, mode, E, slot=slot, gate=gate, out=out)
        _check(out, x, ids, w, group, mode, slot=slot, gate=gate)
        assert torch.all(room[:skip] == 7) and torch.all(room[skip + size:] == 7)


def test_a_row_has_the_same_bits_however_many_workgroups_share_its_expert():
    """The tiles' places do not change with the number of workgroups: a call of fewer rows of weights, with more workgroups an expert, gives
    the same bits for these rows."""
    T, E, k, K, group = 400, 6, 2, 512, 64
    q, s, z = _weights(3, E, 2048, K, group, torch.float16, True)
    ids = _routed(3, T, E, k)
    x, _ = _inputs(3, T, k, K, "each", torch.float16)
    whole = _run(x, ids, (q, s, z), group, "each", E)
    part = _run(x, ids, tuple(v[:, :64].contiguous() for v in (q, s, z)), group, "each", E)
    assert torch.equal(part, whole[..., :64])
