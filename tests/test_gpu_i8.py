"""Products in 8-bit integers on the GPU: levels of tokens and weights and the experts' products, against 64 bits.

Tolerance: levels of 16-bit values are equal; products are off by one rounding to the output's type and what 32-bit scales
and sums over slots may be off (i8_reference.products)."""
import math

import pytest
import torch

import i8_reference as ref
import paper_2606_01007_amd as tacg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _err():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def _scales(got, want):
    return bool(((got.cpu().double() - want).abs() <= ref.U * want * (1 + 1e-6) + 1e-45).all())


# ---- levels -------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R, K", [(1, 1), (3, 2), (5, 7), (2, 63), (4, 64), (3, 65), (7, 127), (9, 257), (33, 1000), (2, 1408), (17, 2048),
                                  (5, 4099), (3, 5120), (2, 8192), (2, 16392), (1, 65536)])
def test_levels_of_tokens(dtype, R, K):
    g = torch.Generator().manual_seed(R * K)
    x = (torch.randn((R, K), generator=g) * torch.exp(torch.randn((R, 1), generator=g) * 3)).to(dtype)
    x[0, K // 2] = x[0].abs().max() / 2      # 63.5 levels: a half that goes to the even one, 64
    q, s = tacg.token_i8(x.cuda())
    want, scale = ref.levels(x)
    assert q.shape == (R, -(-K // 64) * 64) and torch.equal(q[:, :K].cpu().long(), want) and not q[:, K:].any()
    assert _scales(s, scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_halves_go_to_the_even_level(dtype):
    x = torch.zeros((254, 130), dtype=dtype)
    n = torch.arange(1, 128)
    for r in range(254):                       # 254 is twice 127: n / 2 of a level, exactly, at a largest value of 127 * 2^r
        p = 2.0 ** ((r % 16) - 8)
        x[r, 0] = 127 * p * (-1 if r % 2 else 1)
        x[r, 1:128] = n * p / (2 if r < 127 else 1)
    want, _ = ref.levels(x)
    assert torch.equal(tacg.token_i8(x.cuda())[0][:, :130].cpu().long(), want)


def test_levels_of_values_of_32_bits():
    g = torch.Generator().manual_seed(4)
    x = torch.randn((40, 777), generator=g)
    x[3] *= 1e30
    x[4] *= 1e-36
    x[5] *= 1e-42                              # below the normal range
    x[6] *= 3e38 / x[6].abs().max()
    x[7] = 0
    q, s = tacg.token_i8(x.cuda())
    v = x.double()
    top = v.abs().amax(1, keepdim=True)
    exact = 127 * v / torch.where(top > 0, top, 1.0)
    # 127 x and the quotient are rounded to 24 bits each: 127 * 2 * 2^-24 of a level
    assert float((q[:, :777].cpu().double() - exact).abs().max()) <= 0.5 + 254 * ref.U
    assert _scales(s, (top / 127).squeeze(1))


def test_smallest_and_largest_values_of_16_bits():
    for dtype in (torch.bfloat16, torch.float16):
        i = torch.finfo(dtype)
        x = torch.zeros((6, 70), dtype=dtype)
        x[0, 3], x[0, 4] = i.max, -i.max
        x[1, 5], x[1, 69] = i.tiny, i.tiny / 2
        x[2, 1] = i.smallest_normal * 2.0 ** -5
        x[3, 0], x[3, 1] = i.max, i.tiny
        x[4, 0] = -1.0
        q, s = tacg.token_i8(x.cuda())
        want, scale = ref.levels(x)
        assert torch.equal(q[:, :70].cpu().long(), want)
        assert _scales(s[:1], scale[:1]) and float(s[5]) == 0


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_a_token_that_is_not_finite(dtype, value):
    x = torch.randn((5, 300), generator=torch.Generator().manual_seed(1)).to(dtype)
    clean = tacg.token_i8(x.cuda())
    x[2, 299] = value
    err = _err()
    q, s = tacg.token_i8(x.cuda(), err=err)
    assert int(err) == tacg.ERR_VALUE and math.isnan(float(s[2])) and not q[2].any()
    rest = [0, 1, 3, 4]
    assert torch.equal(q[rest], clean[0][rest]) and torch.equal(s[rest], clean[1][rest])


def test_strides_and_shapes_of_tokens():
    base = torch.randn((9, 3, 131), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    want = tacg.token_i8(base[:, 1, 1:130].contiguous())
    got = tacg.token_i8(base[:, 1, 1:130])               # rows apart, and not at multiples of 16 bytes
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q, s = tacg.token_i8(base)
    assert q.shape == (9, 3, 192) and s.shape == (9, 3)
    assert torch.equal(tacg.token_i8(base.reshape(27, 131))[0], q.reshape(27, 192))
    assert torch.equal(tacg.token_i8(base[0, 0])[0], q[0, 0])
    assert tacg.token_i8(base[:0])[0].shape == (0, 3, 192)
    row = base[0, 0, :64].expand(4, 64)                  # one row four times
    assert torch.equal(tacg.token_i8(row)[0], tacg.token_i8(row.contiguous())[0])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("H, N, K", [(1, 1, 1), (2, 16, 64), (3, 17, 65), (1, 130, 250), (4, 48, 1408), (2, 31, 4100)])
def test_packing(dtype, H, N, K):
    w = torch.randn((H, N, K), generator=torch.Generator().manual_seed(N)).to(dtype)
    w[H - 1, N - 1] = 0
    err = _err()
    q, s = tacg.i8_pack(w.cuda(), err=err)
    want, scale = ref.levels(w)
    assert torch.equal(q.cpu(), ref.tiles(want)) and _scales(s, scale) and int(err) == 0
    w[0, N // 2, K - 1] = math.inf
    bad, sb = tacg.i8_pack(w.cuda(), err=err)
    assert int(err) == tacg.ERR_VALUE and math.isnan(float(sb[0, N // 2]))
    want[0, N // 2] = 0
    assert torch.equal(bad.cpu(), ref.tiles(want))


def test_packing_of_32_bit_weights():
    w = torch.randn((2, 33, 200), generator=torch.Generator().manual_seed(5))
    q, s = tacg.i8_pack(w.cuda())
    got = torch.stack([tacg.token_i8(w[h].cuda())[0][:, :200] for h in range(2)]).cpu()
    assert torch.equal(q.cpu(), ref.tiles(got))
    assert _scales(s, ref.levels(w)[1])


# ---- products -----------------------------------------------------------------------------------

def _weights(seed, H, N, K):
    g = torch.Generator().manual_seed(seed)
    qw = torch.randint(-127, 128, (H, N, K), generator=g)
    return qw, (torch.rand((H, N), generator=g) + 0.5) / (73 * K ** 0.5)


def _routed(seed, T, E, k, unused=0.0):
    g = torch.Generator().manual_seed(seed)
    ids = torch.rand((T, E), generator=g).argsort(1)[:, :k].to(torch.int16)
    if unused:
        ids[torch.rand((T, k), generator=g) < unused] = -1
    return ids


def _inputs(seed, T, k, K, mode, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, k, K) if mode == "sum" else (T, K), generator=g).to(dtype)
    return x, torch.rand((T, k), generator=g) if mode == "sum" else None


def _run(x, ids, w, mode, E=None, slot=None, gate=None, **kw):
    cuda = lambda v: None if v is None else v.cuda()  # noqa: E731
    return tacg.expert_i8(x.cuda() if isinstance(x, torch.Tensor) else x, cuda(ids), ref.tiles(w[0]).cuda(), w[1].cuda(), mode=mode,
                          n_experts=E, slot_of_expert=cuda(slot), gate=cuda(gate), **kw)


def _check(got, x, ids, w, mode, slot=None, gate=None):
    qx, sx = ref.levels(x)
    want, off = ref.products(qx, sx, ids, *w, mode, slot, gate)
    assert got.shape == want.shape
    assert ref.within(got, want, off, got.dtype), float((got.double().cpu() - want).abs().max())


SIZES = [
    (1, 1, 1, 2, 1),            # the smallest of all
    (1, 8, 2, 16, 32),
    (1, 8, 8, 64, 256),
    (1, 16, 6, 130, 1408),      # one token: the serving form
    (2, 4, 2, 34, 33),
    (3, 8, 3, 66, 127),
    (5, 8, 4, 100, 1000),
    (16, 4, 1, 64, 512),
    (17, 2, 2, 48, 160),        # every token at both experts
    (40, 60, 4, 130, 250),
    (33, 3, 3, 258, 640),
    (70, 4, 2, 96, 288),        # many tokens an expert
    (150, 2, 1, 64, 384),
    (300, 1, 1, 274, 200),      # all at one
    (131, 16, 4, 514, 130),
]


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T, E, k, N, K", SIZES)
def test_products(mode, dtype, T, E, k, N, K):
    w, ids = _weights(T + N + K, E, N, K), _routed(T, T, E, k)
    x, gate = _inputs(K, T, k, K, mode, dtype)
    err = _err()
    _check(_run(x, ids, w, mode, gate=gate, err=err), x, ids, w, mode, gate=gate)
    assert int(err) == 0


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("T, E, k, N, K", [(1, 8, 2, 34, 100), (20, 16, 4, 66, 130), (90, 4, 2, 130, 70)])
def test_products_of_32_bit_tokens_and_results(mode, T, E, k, N, K):
    """Levels of 32-bit values are compared in a test of their own: here they are given."""
    w, ids = _weights(T + N + K, E, N, K), _routed(T, T, E, k)
    x, gate = _inputs(K, T, k, K, mode, torch.float32)
    q, s = tacg.token_i8(x.cuda())
    want, off = ref.products(q.cpu(), s.cpu().double(), ids, *w, mode, None, gate)
    got = _run(x, ids, w, mode, gate=gate)
    assert got.dtype == torch.float32 and ref.within(got, want, off, torch.float32)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):       # the pair, with any type of result
        pair = _run((q, s), ids, w, mode, gate=gate, dtype=dtype)
        assert pair.dtype == dtype and torch.equal(pair, got.to(dtype))
    assert _run((q, s), ids, w, mode, gate=gate).dtype == torch.bfloat16


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("T, E, k, N, K, G", [(1, 8, 4, 64, 64, 2), (3, 60, 4, 64, 192, 4), (50, 60, 6, 130, 192, 4), (200, 16, 8, 64, 96, 8),
                                              (64, 8, 2, 66, 100, 8)])
def test_shares_of_several_gpus(mode, T, E, k, N, K, G):
    ids = _routed(T, T, E, k, unused=0.1)
    if T > 2:
        ids[1] = -1                                                    # a token without any expert
    x, gate = _inputs(K, T, k, K, mode, torch.bfloat16)
    for m in {0, G - 1}:
        held = torch.arange(m, E, G)
        slot = torch.full((E,), -1, dtype=torch.int32)
        slot[held] = torch.arange(held.numel(), dtype=torch.int32)
        w = _weights(m, held.numel(), N, K)
        out = torch.full({"each": (T, k, N), "glu": (T, k, N // 2), "sum": (T, N)}[mode], math.nan, dtype=torch.bfloat16, device="cuda")
        got = _run(x, ids, w, mode, E=E, slot=slot, gate=gate, out=out)
        assert got is out
        _check(got, x, ids, w, mode, slot, gate)


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
def test_no_expert_held_here(mode):
    x, gate = _inputs(3, 37, 2, 64, mode, torch.bfloat16)
    ids = _routed(3, 37, 8, 2)
    w = (torch.zeros((0, 32, 64), dtype=torch.int64), torch.zeros((0, 32)))
    got = _run(x, ids, w, mode, E=8, slot=torch.full((8,), -1, dtype=torch.int32), gate=gate)
    assert not got.any()
    w = _weights(1, 3, 32, 64)
    ids[:] = -1
    assert not _run(x, ids, w, mode, E=8, slot=torch.zeros(8, dtype=torch.int32), gate=gate).any()


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("T, H, N, K", [(1, 1, 64, 64), (1, 2, 130, 200), (19, 1, 66, 130), (130, 1, 514, 320), (70, 3, 96, 100), (600, 1, 34, 64)])
def test_shared_experts(mode, T, H, N, K):
    w = _weights(T, H, N, K)
    x, gate = _inputs(T, T, H, K, mode, torch.float16)
    _check(_run(x, None, w, mode, gate=gate), x, None, w, mode, gate=gate)
    if mode == "sum":                                                  # a gate of 1, and one x per token
        _check(_run(x, None, w, mode), x, None, w, mode)
        _check(_run(x[:, 0], None, w, mode), x[:, 0], None, w, mode)


@pytest.mark.parametrize("T", [1, 30, 200])
def test_sums_of_one_x_per_token(T):
    w, ids = _weights(2, 8, 70, 130), _routed(2, T, 8, 3)
    x, _ = _inputs(2, T, 3, 130, "each", torch.bfloat16)
    gate = torch.rand((T, 3), generator=torch.Generator().manual_seed(9))
    _check(_run(x, ids, w, "sum", gate=gate), x, ids, w, "sum", gate=gate)
    y, _ = _inputs(2, T, 3, 130, "sum", torch.bfloat16)                # and an x of its own for every slot of the other modes
    for mode in ("each", "glu"):
        _check(_run(y, ids, w, mode), y, ids, w, mode)


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("T", [1, 5, 64, 300])
def test_a_token_that_is_not_finite_leaves_the_others(mode, T):
    w, ids = _weights(7, 4, 66, 100), _routed(7, T, 4, 2)
    x, gate = _inputs(7, T, 2, 100, mode, torch.bfloat16)
    clean = _run(x, ids, w, mode, gate=gate)
    x[T // 2, ..., 99] = math.inf
    err = _err()
    got = _run(x, ids, w, mode, gate=gate, err=err)
    assert int(err) == tacg.ERR_VALUE and torch.isnan(got[T // 2]).all()
    rest = [t for t in range(T) if t != T // 2]
    assert torch.equal(got[rest], clean[rest])


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
@pytest.mark.parametrize("T", [1, 6, 90])
def test_bad_ids_and_tables_are_reported(mode, T):
    w, ids = _weights(5, 4, 64, 96), _routed(5, T, 6, 2)
    x, gate = _inputs(5, T, 2, 96, mode, torch.bfloat16)
    slot = torch.tensor([0, 1, 2, 3, -1, -5], dtype=torch.int32)
    err = _err()
    _check(_run(x, ids, w, mode, E=6, slot=slot, gate=gate, err=err), x, ids, w, mode, slot, gate)
    assert int(err) == 0
    for bad in (6, -2, 32767, -32768):
        err, wrong = _err(), ids.clone()
        wrong[T - 1, 1] = bad
        got = _run(x, wrong, w, mode, E=6, slot=slot, gate=gate, err=err)
        assert int(err) == tacg.ERR_ID_RANGE
        none = wrong.clone()
        none[T - 1, 1] = -1
        assert torch.equal(got, _run(x, none, w, mode, E=6, slot=slot, gate=gate))
    err = _err()
    wrong = slot.clone()
    wrong[int(ids[0, 0])] = 4
    got = _run(x, ids, w, mode, E=6, slot=wrong, gate=gate, err=err)
    assert int(err) == tacg.ERR_TABLE
    wrong[int(ids[0, 0])] = -1
    assert torch.equal(got, _run(x, ids, w, mode, E=6, slot=wrong, gate=gate))


def test_the_same_expert_twice_and_strided_tokens():
    w = _weights(3, 5, 64, 128)
    ids = torch.tensor([[2, 2, 1], [4, 4, 4], [0, 1, 0]], dtype=torch.int16)
    base = torch.randn((3, 3, 300), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    x = base.cuda()[:, :, 37:165]                                      # rows apart, not at multiples of 16 bytes
    gate = torch.rand((3, 3), generator=torch.Generator().manual_seed(4))
    for mode in ("each", "glu", "sum"):
        _check(_run(x, ids, w, mode, gate=gate if mode == "sum" else None), x.cpu(), ids, w, mode, gate=gate if mode == "sum" else None)
    one = x[:1, 0].expand(3, 128)                                      # one row for all tokens
    _check(_run(one, ids, w, "each"), one.cpu(), ids, w, "each")


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
def test_bits_do_not_depend_on_the_other_tokens(mode):
    """Sums are exact: alone, in a small batch and in a large one a token's result is the same."""
    w, ids = _weights(8, 6, 130, 300), _routed(8, 400, 6, 2)
    x, gate = _inputs(8, 400, 2, 300, mode, torch.bfloat16)
    whole = _run(x, ids, w, mode, gate=gate)
    for n in (1, 2, 7, 40, 129):
        g = None if gate is None else gate[:n].contiguous()
        assert torch.equal(_run(x[:n], ids[:n].contiguous(), w, mode, gate=g), whole[:n]), n


@pytest.mark.parametrize("mode", ["each", "glu", "sum"])
def test_levels_at_their_ends(mode):
    """All levels at 127 or -127 (and -128, which a caller may give): the largest sums, exactly."""
    K = 4160
    qw = torch.full((2, 32, K), -127)
    qw[1] = 127
    sw = torch.full((2, 32), 2.0 ** -12)
    q = torch.full((20, K), -128, dtype=torch.int8)
    q[1] = 127
    s = torch.full((20,), 2.0 ** -10)
    ids = torch.tensor([[0, 1]] * 20, dtype=torch.int16)
    gate = torch.full((20, 2), 0.5) if mode == "sum" else None
    want, off = ref.products(q, s.double(), ids, qw, sw, mode, None, gate)
    got = _run((q.cuda(), s.cuda()), ids, (qw, sw), mode, gate=gate, dtype=torch.float32)
    assert ref.within(got, want, off, torch.float32)


def test_widest_rows():
    g = torch.Generator().manual_seed(6)
    K = 65536
    qw = torch.randint(-127, 128, (2, 16, K), generator=g)
    sw = torch.full((2, 16), 2.0 ** -14)
    for T in (1, 40):
        x = torch.randn((T, K), generator=g).to(torch.bfloat16)
        ids = _routed(T, T, 2, 1)
        _check(_run(x, ids, (qw, sw), "each"), x, ids, (qw, sw), "each")
    qw = torch.randint(-127, 128, (1, 65536, 64), generator=g)
    sw = torch.full((1, 65536), 2.0 ** -10)
    x = torch.randn((3, 64), generator=g).to(torch.bfloat16)
    _check(_run(x, None, (qw, sw), "glu"), x, None, (qw, sw), "glu")


def test_no_tokens_and_other_streams():
    w = _weights(1, 4, 64, 64)
    assert _run(torch.empty((0, 64), dtype=torch.bfloat16), torch.empty((0, 2), dtype=torch.int16), w, "glu").shape == (0, 2, 32)
    x, _ = _inputs(1, 100, 2, 64, "each", torch.bfloat16)
    ids = _routed(1, 100, 4, 2)
    want = _run(x, ids, w, "glu")
    q, s = ref.tiles(w[0]).cuda(), w[1].cuda()
    dx, di = x.cuda(), ids.cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = tacg.expert_i8(dx, di, q, s, mode="glu", stream=side)
    lv = tacg.token_i8(dx, stream=side)
    pair = tacg.expert_i8(lv, di, q, s, mode="glu", stream=side)
    packed = tacg.i8_pack(torch.ones((2, 16, 64), device="cuda"), stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(pair, want) and int(packed[0].min()) == 127


@pytest.mark.parametrize("T", [1, 12, 150])
def test_captured_and_replayed(T):
    w = _weights(4, 8, 130, 192)
    q, s = ref.tiles(w[0]).cuda(), w[1].cuda()
    x = torch.zeros((T, 192), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros((T, 2), dtype=torch.int16, device="cuda")
    gate = torch.ones((T, 2), device="cuda")
    err = _err()
    h, y = torch.empty((T, 2, 65), dtype=torch.bfloat16, device="cuda"), torch.empty((T, 130), dtype=torch.bfloat16, device="cuda")
    ws = tacg.workspace(1 << 22)

    def call():
        tacg.expert_i8(x, ids, q, s, mode="glu", out=h, err=err, ws=ws)
        tacg.expert_i8(x, ids, q, s, mode="sum", gate=gate, out=y, err=err, ws=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        nx, _ = _inputs(i, T, 2, 192, "each", torch.bfloat16)
        x.copy_(nx.cuda())
        ids.copy_(_routed(i, T, 8, 2).cuda())
        gate.copy_(torch.rand((T, 2), generator=torch.Generator().manual_seed(i)).cuda())
        graph.replay()
        torch.cuda.synchronize()
        gh, gy = h.clone(), y.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(gh, h) and torch.equal(gy, y) and int(err) == 0
        _check(gy, nx, ids.cpu(), w, "sum", gate=gate.cpu())


def test_the_whole_layer():
    """Router with groups, gated products, closing products, as they are used together, against 64 bits from the same levels."""
    g = torch.Generator().manual_seed(11)
    T, E, k, D, I = 50, 16, 4, 128, 96
    r = tacg.route(torch.randn((1, T, E), generator=g).cuda(), k, score="sigmoid", renorm=True, scale=2.5, groups=4, top_groups=2,
                   bias=0.1 * torch.randn((1, E), generator=g).cuda())
    up, down = (torch.randn((E, 2 * I, D), generator=g) / D ** 0.5).to(torch.bfloat16), (torch.randn((E, D, I), generator=g) / I ** 0.5).to(torch.bfloat16)
    x = torch.randn((T, D), generator=g).to(torch.bfloat16)
    qu, su = tacg.i8_pack(up.cuda())
    qd, sd = tacg.i8_pack(down.cuda())
    ids, gate = r["trace"][0], r["gate"][0]
    h = tacg.expert_i8(x.cuda(), ids, qu, su, mode="glu")
    y = tacg.expert_i8(h, ids, qd, sd, mode="sum", gate=gate)
    lu, ld = ref.levels(up), ref.levels(down)
    _check(h, x, ids.cpu(), (lu[0], lu[1]), "glu")
    _check(y, h.cpu(), ids.cpu(), (ld[0], ld[1]), "sum", gate=gate.cpu())
