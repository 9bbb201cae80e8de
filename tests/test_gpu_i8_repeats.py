"""Products in 8-bit integers where a matrix has more pairs than there are tokens: an expert that stands twice in a token's row, and tables
that give several experts one matrix.  Not a router's output, but defined ones.

Tolerances are those of test_gpu_i8: what i8_reference.products derives, and one rounding to the output's type."""
import math

import pytest
import torch

import i8_reference as ref
import paper_2606_01007_amd as tacg
from test_gpu_i8 import _check, _err, _gpu, _inputs, _run, _weights  # noqa: F401

pytestmark = pytest.mark.gpu


def _one_launch(T, k, E, H, N, K, mode, per_slot=False):
    return tacg.lib().tacg_expert_i8_workspace_bytes(T, k, E, H, N, K, tacg.Q4_MODES[mode], tacg.DTYPES[torch.bfloat16], per_slot) == 0


def _ids(kind, seed, T, k, E):
    """(ids, table, matrices): all slots one expert; any experts, some twice; different experts of few matrices."""
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        return torch.full((T, k), E - 1, dtype=torch.int16), None, E
    if kind == "some":
        return torch.randint(-1, E, (T, k), generator=g).to(torch.int16), None, E
    table = torch.randint(-1, 2, (E,), generator=g).to(torch.int32)
    table[:2] = 1
    return torch.rand((T, E), generator=g).argsort(1)[:, :k].to(torch.int16), table, 2


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("kind", ["one", "some", "table"])
@pytest.mark.parametrize("T, k, E, N, K", [
    (1, 2, 8, 34, 2048), (1, 6, 16, 130, 2048), (1, 16, 16, 66, 1000), (2, 3, 4, 34, 130), (3, 16, 16, 34, 2048), (5, 4, 8, 66, 2047),
    (12, 2, 8, 66, 2048), (12, 4, 12, 34, 64), (16, 3, 13, 34, 1408), (17, 2, 9, 34, 2048), (24, 2, 12, 34, 1024), (40, 4, 8, 66, 130),
    (300, 3, 6, 34, 200),
])
def test_one_x_for_all_slots(mode, kind, T, k, E, N, K):
    ids, table, H = _ids(kind, T + k, T, k, E)
    w = _weights(N + K, H, N, K)
    x, _ = _inputs(T, T, k, K, "each", torch.bfloat16)
    gate = torch.rand((T, k), generator=torch.Generator().manual_seed(T)) if mode == "sum" else None
    assert mode == "sum" or _one_launch(T, k, E, H, N, K, mode) == (T * k <= 48)
    err = _err()
    got = _run(x, ids, w, mode, E=E, slot=table, gate=gate, err=err)
    assert int(err) == 0
    _check(got, x, ids, w, mode, table, gate)
    pair = _run(tacg.token_i8(x.cuda()), ids, w, mode, E=E, slot=table, gate=gate, dtype=torch.bfloat16)
    assert torch.equal(pair, got)
    many = 400 // T + 1                                                # the same tokens among many
    whole = _run(x.repeat(many, 1), ids.repeat(many, 1), w, mode, E=E, slot=table, gate=None if gate is None else gate.repeat(many, 1))
    assert torch.equal(whole[:T], got) and torch.equal(whole[-T:], got)


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("kind", ["one", "some", "table"])
@pytest.mark.parametrize("T, k, E, N, K", [(1, 2, 8, 34, 2048), (1, 16, 16, 34, 700), (5, 4, 8, 34, 500), (6, 8, 12, 34, 130), (16, 3, 13, 34, 1408)])
def test_an_x_for_each_slot(mode, kind, T, k, E, N, K):
    ids, table, H = _ids(kind, T + k, T, k, E)
    w = _weights(N + K, H, N, K)
    x, gate = _inputs(T, T, k, K, "sum", torch.float16)
    gate = gate if mode == "sum" else None
    assert mode == "sum" or _one_launch(T, k, E, H, N, K, mode, True)
    got = _run(x, ids, w, mode, E=E, slot=table, gate=gate)
    _check(got, x, ids, w, mode, table, gate)


@pytest.mark.parametrize("mode", ["each", "glu"])
@pytest.mark.parametrize("T", [2, 12])
def test_a_token_that_is_not_finite_at_an_expert_that_it_has_twice(mode, T):
    w = _weights(7, 8, 66, 2048)
    ids = torch.full((T, 3), 5, dtype=torch.int16)
    ids[:, 1] = torch.arange(T) % 8
    x, _ = _inputs(7, T, 3, 2048, "each", torch.bfloat16)
    clean = _run(x, ids, w, mode)
    x[T // 2, 2047] = math.inf
    err = _err()
    got = _run(x, ids, w, mode, err=err)
    assert int(err) == tacg.ERR_VALUE and torch.isnan(got[T // 2]).all()
    rest = [t for t in range(T) if t != T // 2]
    assert torch.equal(got[rest], clean[rest])


def test_captured_and_replayed_with_repeated_experts():
    T, k, N, K = 12, 3, 66, 2048
    w = _weights(4, 8, N, K)
    q, s = ref.tiles(w[0]).cuda(), w[1].cuda()
    x = torch.zeros((T, K), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros((T, k), dtype=torch.int16, device="cuda")
    err, h = _err(), torch.empty((T, k, N // 2), dtype=torch.bfloat16, device="cuda")

    def call():
        tacg.expert_i8(x, ids, q, s, mode="glu", out=h, err=err)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i, kind in enumerate(("some", "one", "some", "one")):
        nx, _ = _inputs(i, T, k, K, "each", torch.bfloat16)
        ni = _ids(kind, i, T, k, 8)[0]
        x.copy_(nx.cuda())
        ids.copy_(ni.cuda())
        graph.replay()
        torch.cuda.synchronize()
        got = h.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, h) and int(err) == 0
        _check(got, nx, ni, w, "glu")
