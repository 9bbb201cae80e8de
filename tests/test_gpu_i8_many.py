"""The experts' products in 8-bit integers over the whole range of batches, so that every way of taking the pairs is met: one launch, streamed
weights in all splits, tiles of all sizes, pairs put in order by few and by many threads and in several readings, tokens whose only
product is written at once.  Expert by expert against 64 bits, with the tolerance of tests/test_gpu_i8.py."""
import pytest
import torch

import i8_reference as ref
import paper_2606_01007_amd as tacg
from test_gpu_i8 import _err, _gpu, _weights  # noqa: F401

pytestmark = pytest.mark.gpu


def _products(qx, sx, ids, qw, sw, mode, slot, gate):
    """i8_reference.products, an expert's tokens at a time."""
    T, (H, N, K) = qx.shape[0], qw.shape
    k = H if ids is None else ids.shape[1]
    ids = torch.arange(H).expand(T, H) if ids is None else ids.long()
    place = ids if slot is None else torch.where(ids >= 0, slot.long()[ids.clamp_min(0)], -1)
    y = torch.zeros((T, k, N), dtype=torch.float64)
    for h in range(H):
        t, j = torch.nonzero(place == h, as_tuple=True)
        if t.numel():
            x, s = (qx[t, j], sx[t, j]) if qx.dim() == 3 else (qx[t], sx[t])
            y[t, j] = (x[:, :K].double() @ qw[h].double().t()) * (s.double()[:, None] * sw[h].double())
    if mode == "each":
        return y, 4 * ref.U * y.abs()
    if mode == "glu":
        a, b = y[..., :N // 2], y[..., N // 2:]
        v = a * torch.sigmoid(a) * b
        return v, 16 * ref.U * (1 + a.abs()) * v.abs() + 1e-37 * b.abs()
    g = torch.where(place >= 0, torch.ones(()) if gate is None else gate, torch.zeros(())).double()[:, :, None]
    return (g * y).sum(1), (5 + k) * ref.U * (g * y).abs().sum(1)


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("T, k, E, N, K, G, pick", [
    (9001, 8, 12, 34, 70, 1, 0.0),       # more pairs than one reading holds
    (20000, 4, 9, 18, 64, 3, 0.0),       # the same on one of three GPUs
    (3000, 4, 16, 66, 130, 1, 0.0),      # put in order by many threads
    (2500, 6, 40, 34, 100, 5, 0.1),      # unused slots, most tokens served elsewhere
    (700, 2, 200, 98, 64, 1, 0.0),       # more experts than tiles
    (64, 2, 200, 4098, 64, 1, 0.0),      # streamed, four blocks of rows a wave
    (40, 2, 64, 2050, 192, 1, 0.0),      # streamed, two
    (30, 1, 60, 258, 1000, 4, 0.0),      # streamed, columns shared by the waves
    (900, 1, 2, 1026, 320, 1, 0.0),      # tiles of all sizes
    (1600, 1, 2, 2050, 256, 1, 0.0),
    (4000, 2, 2, 2052, 64, 1, 0.0),
    (2049, 1, 1, 4100, 128, 1, 0.0),
    (5, 8, 256, 66, 4160, 8, 0.0),       # one launch, long rows
    (16, 3, 16, 66, 200, 2, 0.2),
    (12, 4, 12, 130, 65, 1, 0.0),        # an expert of all tokens among the pairs of one launch
    (64, 1, 64, 34, 64, 1, 0.0),
])
def test_every_way_of_taking_pairs(mode, T, k, E, N, K, G, pick):
    g = torch.Generator().manual_seed(T + E)
    ids = (torch.rand((T, E), generator=g) + 0.3 * torch.rand((E,), generator=g)).argsort(1)[:, :k].to(torch.int16)
    if T == 12:
        ids[:, 0] = 3
    if pick:
        ids[torch.rand((T, k), generator=g) < pick] = -1
    held = torch.arange(G - 1, E, G)
    slot = None
    if G > 1:
        slot = torch.full((E,), -1, dtype=torch.int32)
        slot[held] = torch.arange(held.numel(), dtype=torch.int32)
    qw, sw = _weights(N, held.numel(), N, K)
    x = torch.randn((T, k, K) if mode == "sum" else (T, K), generator=g).to(torch.bfloat16)
    gate = torch.rand((T, k), generator=g) if mode == "sum" else None
    out = torch.full({"each": (T, k, N), "glu": (T, k, N // 2), "sum": (T, N)}[mode], float("nan"), dtype=torch.bfloat16, device="cuda")
    err = _err()
    cuda = lambda v: None if v is None else v.cuda()  # noqa: E731
    full = torch.nn.functional.pad(qw.to(torch.int8), (0, -K % 64, 0, -N % 16))
    q = full.view(held.numel(), -(-N // 16), 16, -(-K // 64), 4, 16).permute(0, 1, 3, 4, 2, 5).contiguous().cuda()
    got = tacg.expert_i8(x.cuda(), ids.cuda(), q, sw.cuda(), mode=mode, n_experts=E, slot_of_expert=cuda(slot), gate=cuda(gate), out=out, err=err)
    assert int(err) == 0
    qx, sx = ref.levels(x)
    want, off = _products(qx, sx, ids, qw, sw, mode, slot, gate)
    assert ref.within(got, want, off, torch.bfloat16)
    # levels in hand give the same bits
    pair = tacg.expert_i8(tacg.token_i8(x.cuda()), ids.cuda(), q, sw.cuda(), mode=mode, n_experts=E, slot_of_expert=cuda(slot), gate=cuda(gate))
    assert torch.equal(pair, got)


@pytest.mark.parametrize("mode", ["each", "sum"])
@pytest.mark.parametrize("T, H, N, K", [(3001, 1, 1026, 192), (500, 2, 514, 64), (100, 1, 1000, 1000), (40, 3, 66, 4096), (4, 1, 4100, 256)])
def test_shared_experts_of_every_batch(mode, T, H, N, K):
    g = torch.Generator().manual_seed(T)
    qw, sw = _weights(T, H, N, K)
    x = torch.randn((T, K), generator=g).to(torch.float16)
    full = torch.nn.functional.pad(qw.to(torch.int8), (0, -K % 64, 0, -N % 16))
    q = full.view(H, -(-N // 16), 16, -(-K // 64), 4, 16).permute(0, 1, 3, 4, 2, 5).contiguous().cuda()
    qx, sx = ref.levels(x)
    want, off = _products(qx, sx, None, qw, sw, mode, None, None)
    assert ref.within(tacg.expert_i8(x.cuda(), None, q, sw.cuda(), mode=mode), want, off, torch.float16)


def test_two_captured_graphs_and_their_workspaces():
    """Two graphs with a workspace each, replayed in turn and on two streams at once."""
    qw, sw = _weights(1, 8, 130, 128)
    full = torch.nn.functional.pad(qw.to(torch.int8), (0, 0, 0, -130 % 16))
    q, s = full.view(8, 9, 16, 2, 4, 16).permute(0, 1, 3, 4, 2, 5).contiguous().cuda(), sw.cuda()
    g = torch.Generator().manual_seed(2)
    err = _err()
    made = []
    for T in (300, 90):
        x = torch.randn((T, 3, 128), generator=g).to(torch.bfloat16).cuda()
        ids = torch.rand((T, 8), generator=g).argsort(1)[:, :3].to(torch.int16).cuda()
        gate = torch.rand((T, 3), generator=g).cuda()
        ws, out = tacg.workspace(1 << 21), torch.empty((T, 130), dtype=torch.bfloat16, device="cuda")
        call = lambda x=x, ids=ids, gate=gate, ws=ws, out=out: tacg.expert_i8(x, ids, q, s, mode="sum", gate=gate, ws=ws, out=out, err=err)  # noqa: E731
        want = call().clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        made.append((graph, out, want, torch.cuda.Stream(), (x, ids, gate, ws)))   # what a graph reads lives as long as it does
    for _ in range(3):
        for _, out, *_ in made:
            out.fill_(0)
        torch.cuda.synchronize()
        for graph, _, _, stream, _ in made:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for _, out, want, *_ in made:
            assert torch.equal(out, want)
    assert int(err) == 0
