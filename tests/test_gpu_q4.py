"""The experts' products with 4-bit weights on the GPU, against the dequantised weights in 64 bits.

Tolerance: one rounding to the output's type, and what 32-bit sums of terms scale * level * x may be off (moe_reference.products)."""
import pytest
import torch

import moe_reference as ref
import paper_2606_01007_amd as tacg

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _weights(seed, H, N, K, group, dtype, zeros):
    g = torch.Generator().manual_seed(seed)
    q = torch.randint(0, 256, (H, N, -(-K // 32) * 16), generator=g, dtype=torch.uint8)
    s = ((torch.rand((H, N, -(-K // group)), generator=g) + 0.5) * 0.2 / K ** 0.5).to(dtype)
    z = torch.randint(0, 16, s.shape, generator=g, dtype=torch.uint8) if zeros else None
    return q, s, z


def _routed(seed, T, E, k, unused=0.0):
    g = torch.Generator().manual_seed(seed)
    ids = torch.rand((T, E), generator=g).argsort(1)[:, :k].to(torch.int16)
    if unused:
        ids[torch.rand((T, k), generator=g) < unused] = -1
    return ids


def _run(x, ids, w, group, mode, E, slot=None, gate=None, **kw):
    cuda = lambda v: None if v is None else v.cuda()  # noqa: E731
    q, s, z = w
    return tacg.expert_q4(x if x.is_cuda else x.cuda(), ids.cuda(), q.cuda(), s.cuda(), cuda(z), group=group, mode=mode,
                          n_experts=E, slot_of_expert=cuda(slot), gate=cuda(gate), **kw)


def _check(got, x, ids, w, group, mode, slot=None, gate=None):
    want, off = ref.products(x.cuda(), ids, *(None if v is None else v.cuda() for v in w), group, mode, slot,
                             None if gate is None else gate.cuda())
    assert got.shape == want.shape and got.dtype == x.dtype
    d = (got.double() - want).abs()
    tol = off * (1 + HALF[x.dtype]) + HALF[x.dtype] * (1 + 1e-6) * want.abs() + TINY[x.dtype]
    assert not torch.isnan(d).any() and float((d - tol).max()) <= 0, float((d / tol).max())


def _inputs(seed, T, k, K, mode, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, k, K) if mode == "sum" else (T, K), generator=g).to(dtype)
    gate = torch.rand((T, k), generator=g) if mode == "sum" else None
    return x, gate


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T, E, k, N, K, group, zeros", [
    (1, 1, 1, 2, 1, 32, False),            # the smallest of all
    (1, 8, 2, 16, 32, 32, True),
    (1, 8, 8, 64, 256, 64, False),
    (1, 16, 6, 130, 1408, 128, False),     # one token: the serving form
    (2, 4, 2, 34, 33, 32, False),          # a group of one column at the end
    (3, 8, 3, 66, 127, 128, True),
    (5, 8, 4, 100, 1000, 128, False),      # groups end inside the row
    (16, 4, 1, 64, 512, 256, True),
    (17, 2, 2, 48, 160, 64, False),        # every token at both experts
    (40, 60, 4, 130, 250, 32, True),
    (33, 3, 3, 258, 640, 128, False),
    (70, 4, 2, 96, 288, 32, False),        # many tokens an expert
    (150, 2, 1, 64, 384, 128, True),
])
def test_products(mode, dtype, T, E, k, N, K, group, zeros):
    w = _weights(T + N + K, E, N, K, group, dtype, zeros)
    ids = _routed(T, T, E, k)
    x, gate = _inputs(K, T, k, K, mode, dtype)
    _check(_run(x, ids, w, group, mode, E, gate=gate), x, ids, w, group, mode, gate=gate)


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("T", [1, 7, 64, 200])
def test_share_of_the_experts(mode, T):
    """A GPU that holds some of the experts, in an order of its own; unused slots; a token that has no expert here."""
    E, k, N, K, group = 24, 4, 70, 320, 64
    slot = torch.full((E,), -1, dtype=torch.int32)
    slot[torch.tensor([3, 20, 4, 9, 11])] = torch.tensor([4, 0, 3, 1, 2], dtype=torch.int32)
    w = _weights(T, 5, N, K, group, torch.bfloat16, False)
    ids = _routed(T, T, E, k, unused=0.2)
    ids[0] = torch.tensor([0, 1, 2, -1], dtype=torch.int16)
    x, gate = _inputs(T, T, k, K, mode, torch.bfloat16)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = _run(x, ids, w, group, mode, E, slot=slot, gate=gate, err=err)
    assert not got[0].any() and int(err.item()) == 0
    _check(got, x, ids, w, group, mode, slot=slot, gate=gate)


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
def test_nothing_is_held(mode):
    ids = _routed(1, 5, 8, 2)
    x, gate = _inputs(1, 5, 2, 64, mode, torch.float16)
    w = _weights(1, 2, 32, 64, 32, torch.float16, False)
    slot = torch.full((8,), -1, dtype=torch.int32)
    assert not _run(x, ids, w, 32, mode, 8, slot=slot, gate=gate).any()
    none = tuple(None if v is None else v[:0] for v in w)
    assert not _run(x, ids, none, 32, mode, 8, slot=slot, gate=gate).any()
    empty = _run(x[:0], ids[:0], w, 32, mode, 8, slot=slot, gate=None if gate is None else gate[:0])
    assert empty.shape[0] == 0


@pytest.mark.parametrize("T", [1, 40])
def test_bad_entries_are_reported_and_left_out(T):
    ids = _routed(T, T, 8, 2)
    w = _weights(3, 8, 32, 64, 32, torch.bfloat16, False)
    x, _ = _inputs(3, T, 2, 64, "each", torch.bfloat16)
    for value, bit in ((8, tacg.ERR_ID_RANGE), (-2, tacg.ERR_ID_RANGE), (32767, tacg.ERR_ID_RANGE)):
        bad = ids.clone()
        bad[0, 1] = value
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = _run(x, bad, w, 32, "each", 8, err=err)
        assert int(err.item()) == bit and not got[0, 1].any()
        _check(got, x, torch.where((bad < 0) | (bad > 7), -1, bad), w, 32, "each")
    slot = torch.arange(8, dtype=torch.int32)
    slot[int(ids[0, 0])] = 8
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = _run(x, ids, w, 32, "each", 8, slot=slot, err=err)
    assert int(err.item()) == tacg.ERR_TABLE and not got[0, 0].any()


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("T", [1, 30])
def test_all_tokens_at_one_expert_and_repeated_ids(mode, T):
    E, k, N, K = 16, 3, 64, 256
    ids = torch.full((T, k), 5, dtype=torch.int16)   # not a router's output, but a defined one
    w = _weights(2, E, N, K, 128, torch.float16, True)
    x, gate = _inputs(2, T, k, K, mode, torch.float16)
    _check(_run(x, ids, w, 128, mode, E, gate=gate), x, ids, w, 128, mode, gate=gate)


def test_strides_of_x():
    E, k, T, N, K = 8, 2, 9, 48, 96
    w = _weights(4, E, N, K, 32, torch.bfloat16, False)
    ids = _routed(4, T, E, k)
    g = torch.Generator().manual_seed(1)
    wide = torch.randn((T, k, K + 11), generator=g).to(torch.bfloat16).cuda()
    for start in (0, 1, 3, 8):
        per_slot = wide[:, :, start:start + K]
        per_token = wide[:, 0, start:start + K]
        one = wide[:1, 0, start:start + K].expand(T, K)
        for x in (per_slot, per_token, one, wide.transpose(0, 1).contiguous().transpose(0, 1)[:, :, start:start + K]):
            for mode in ("each", "glu"):
                got = _run(x, ids, w, 32, mode, E)
                assert torch.equal(got, _run(x.contiguous(), ids, w, 32, mode, E))
                _check(got, x, ids, w, 32, mode)


def test_values_of_x_that_are_not_finite_stay_with_their_token():
    E, k, T, N, K = 4, 2, 20, 40, 256
    w = _weights(7, E, N, K, 128, torch.bfloat16, False)
    ids = _routed(7, T, E, k)
    x, _ = _inputs(7, T, k, K, "each", torch.bfloat16)
    clean = _run(x, ids, w, 128, "each", E)
    x[3, 17], x[4, 200] = float("nan"), float("inf")
    got = _run(x, ids, w, 128, "each", E)
    keep = [t for t in range(T) if t not in (3, 4)]
    assert torch.equal(got[keep], clean[keep]) and torch.isnan(got[3]).all() and not torch.isfinite(got[4]).any()


def test_padding_of_a_row_is_not_read_into_the_product():
    E, k, T, N, K = 2, 1, 3, 16, 40
    q, s, z = _weights(9, E, N, K, 32, torch.float16, True)
    ids = _routed(9, T, E, k)
    x, _ = _inputs(9, T, k, K, "each", torch.float16)
    a = _run(x, ids, (q, s, z), 32, "each", E)
    q[:, :, K // 2:] ^= 0xFF
    assert torch.equal(a, _run(x, ids, (q, s, z), 32, "each", E))


def test_results_do_not_depend_on_the_run_or_on_other_tokens():
    E, k, T, N, K = 16, 4, 50, 160, 512
    w = _weights(5, E, N, K, 64, torch.bfloat16, False)
    ids = _routed(5, T, E, k)
    for mode in ("each", "glu", "sum"):
        x, gate = _inputs(5, T, k, K, mode, torch.bfloat16)
        first = _run(x, ids, w, 64, mode, E, gate=gate)
        for _ in range(3):
            assert torch.equal(first, _run(x, ids, w, 64, mode, E, gate=gate))


def test_another_stream_and_a_graph():
    E, k, T, N, K = 32, 4, 48, 128, 256
    w = tuple(None if v is None else v.cuda() for v in _weights(6, E, N, K, 64, torch.bfloat16, True))
    ids = _routed(6, T, E, k).cuda()
    x, gate = (v.cuda() for v in _inputs(6, T, k, K, "sum", torch.bfloat16))
    call = lambda **kw: tacg.expert_q4(x, ids, *w, group=64, mode="sum", gate=gate, **kw)  # noqa: E731
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = call(stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = tacg.workspace(tacg.lib().tacg_expert_q4_workspace_bytes(T, k, E, N, K, tacg.Q4_MODES["sum"]))
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(err=err, ws=ws, out=out)
    for seed in range(3):
        ids.copy_(_routed(60 + seed, T, E, k))
        x.copy_(_inputs(60 + seed, T, k, K, "sum", torch.bfloat16)[0])
        graph.replay()
        torch.cuda.synchronize()
        want = call()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_weights_past_four_gigabytes():
    """Offsets past 32 bits in the levels: the last expert of a large set."""
    H, N, K = 140, 4096, 16384
    q = torch.zeros((H, N, K // 2), dtype=torch.uint8, device="cuda")
    s = torch.full((H, N, K // 128), 0.01, dtype=torch.bfloat16, device="cuda")
    q[-1] = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda")
    x = torch.randn((2, K), device="cuda").to(torch.bfloat16)
    ids = torch.tensor([[0, H - 1], [H - 1, 3]], dtype=torch.int16, device="cuda")
    got = tacg.expert_q4(x, ids, q, s, group=128, mode="each")
    last = (q[-1:].contiguous(), s[-1:].contiguous(), None)
    only = torch.tensor([[-1, 0], [0, -1]], dtype=torch.int16)
    want, off = ref.products(x, only, *last, 128, "each")
    for t, j in ((0, 1), (1, 0)):
        d = (got[t, j].double() - want[t, j]).abs()
        assert (d <= off[t, j] * 1.01 + HALF[torch.bfloat16] * 1.001 * want[t, j].abs()).all()


# ---- packing --------------------------------------------------------------------------------------

def _packed(w, group, symmetric, scale_dtype):
    """The definition, in 32-bit arithmetic as it states."""
    H, N, K = w.shape
    G = -(-K // group)
    v = torch.zeros((H, N, G * group))
    v[:, :, :K] = w.float()
    v = v.reshape(H, N, G, group)
    if symmetric:
        scale = (v.abs().amax(3) / 7.0).to(scale_dtype)
        zero = torch.full_like(scale, 8, dtype=torch.float32)
    else:
        lo, hi = v.amin(3).clamp_max(0), v.amax(3).clamp_min(0)
        scale = ((hi - lo) / 15.0).to(scale_dtype)
        s = scale.float()
        zero = torch.where(s > 0, torch.round(-lo / torch.where(s > 0, s, 1.0)).clamp(0, 15), 8.0)
    s = scale.float()[..., None]
    level = torch.where(s > 0, (torch.round(v / torch.where(s > 0, s, 1.0)) + zero[..., None]).clamp(0, 15), zero[..., None])
    level = level.reshape(H, N, G * group)[:, :, :-(-K // 32) * 32].to(torch.uint8)
    return level[:, :, 0::2] | level[:, :, 1::2] << 4, scale, zero.to(torch.uint8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("symmetric", [True, False])
@pytest.mark.parametrize("H, N, K, group", [(1, 1, 1, 32), (2, 5, 64, 32), (3, 7, 100, 64), (1, 33, 1000, 128), (2, 16, 384, 256),
                                            (1, 3, 33, 256)])
def test_packing(dtype, symmetric, H, N, K, group):
    w = (torch.randn((H, N, K), generator=torch.Generator().manual_seed(K + N)) * 0.05).to(dtype)
    w[0, 0] = 0.0                                   # a group without a scale
    q, s, z = tacg.q4_pack(w.cuda(), group=group, symmetric=symmetric)
    want = _packed(w, group, symmetric, s.dtype)
    assert s.dtype == (torch.bfloat16 if dtype == torch.float32 else dtype)
    assert torch.equal(q.cpu(), want[0]) and torch.equal(s.cpu(), want[1])
    assert z is None if symmetric else torch.equal(z.cpu(), want[2])
    # what comes back is within half a level (symmetric: the scale is rounded, so seven levels may end up to 7 * 2^-8 short)
    back = ref.dequantise(q.cpu(), s.cpu(), None if z is None else z.cpu(), K, group)
    step = s.cpu().double().repeat_interleave(group, 2)[:, :, :K]
    assert ((back - w.double()).abs() <= step * (0.5 + 15 * 2.0 ** -8) + 1e-6).all()


def test_packing_reports_values_that_are_not_finite():
    for v in (float("nan"), float("inf"), -float("inf")):
        w = torch.zeros((1, 2, 64), device="cuda")
        w[0, 1, 40] = v
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        tacg.q4_pack(w, group=32, err=err)
        assert int(err.item()) == tacg.ERR_VALUE
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    tacg.q4_pack(torch.full((1, 1, 32), 1e9, device="cuda"), group=32, scale_dtype=torch.float16, err=err)
    assert int(err.item()) == tacg.ERR_VALUE
