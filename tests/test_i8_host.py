"""Host-side checks of the 8-bit products' and the grouped router's entry points (CPU only): exports, sizes of workspaces, refused
arguments, and the binding's checks of types, shapes and strides."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import i8_reference as ref
import paper_2606_01007_amd as tacg

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "tacg.h")
FAKE = ctypes.c_void_p(1 << 20)   # never dereferenced: every call below fails validation first
odd = lambda n: ctypes.c_void_p((1 << 20) + n)  # noqa: E731


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(tacg.LIB_PATH):
        pytest.skip("libtacg.so not built")
    return tacg.lib()


def test_exports_and_constants(L):
    text = open(HEADER).read()
    for name in ("tacg_route_grouped", "tacg_token_i8", "tacg_i8_pack", "tacg_expert_i8", "tacg_expert_i8_workspace_bytes"):
        assert re.search(rf"\b{name}\(", text) and hasattr(L, name), name
    assert int(re.search(r"#define TACG_I8 (\d+)", text).group(1)) == tacg.I8


def _grouped(L, **kw):
    off = np.array([0, 50, 100], dtype=np.int64)
    a = dict(x=FAKE, dtype=0, k=2, E=8, bias=None, groups=4, top=2, best=2, trace=FAKE, gate=FAKE, D=None, err=FAKE, scale=1.0)
    a.update(kw)
    return L.tacg_route_grouped(a["x"], a["dtype"], 800, 8, 100, 2, a["k"], a["E"], off.ctypes.data_as(ctypes.c_void_p), 2, 0,
                                a["bias"], 0, a["scale"], a["groups"], a["top"], a["best"], a["trace"], a["gate"], None, a["D"], None,
                                None, None, a["err"], None, 0, None)


def test_grouped_router_refuses(L):
    for kw in (dict(groups=0), dict(groups=-1), dict(groups=3), dict(groups=16), dict(top=0), dict(top=5), dict(top=-1), dict(best=0),
               dict(best=3), dict(x=None), dict(trace=None), dict(gate=None), dict(err=None), dict(D=FAKE), dict(dtype=3), dict(k=9),
               dict(scale=float("nan"))):
        assert _grouped(L, **kw) == tacg.E_INVAL, kw
    assert _grouped(L, E=66, groups=33, top=1) == tacg.E_UNSUPPORTED


def _tokens(L, **kw):
    a = dict(x=FAKE, dtype=1, rows=8, cols=64, stride=64, q=FAKE, s=FAKE, err=FAKE)
    a.update(kw)
    return L.tacg_token_i8(a["x"], a["dtype"], a["rows"], a["cols"], a["stride"], a["q"], a["s"], a["err"], None)


def _pack(L, **kw):
    a = dict(w=FAKE, dtype=1, H=2, rows=8, cols=64, q=FAKE, s=FAKE, err=FAKE)
    a.update(kw)
    return L.tacg_i8_pack(a["w"], a["dtype"], a["H"], a["rows"], a["cols"], a["q"], a["s"], a["err"], None)


def test_rounding_refuses(L):
    for kw in (dict(x=None), dict(x=odd(1)), dict(x=odd(2), dtype=0), dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(cols=0),
               dict(stride=-1), dict(q=None), dict(q=odd(8)), dict(s=None), dict(s=odd(2)), dict(err=None)):
        assert _tokens(L, **kw) == tacg.E_INVAL, kw
    for kw in (dict(cols=65537), dict(rows=1 << 31)):
        assert _tokens(L, **kw) == tacg.E_UNSUPPORTED, kw
    assert _tokens(L, rows=0, x=None) == tacg.OK
    for kw in (dict(w=None), dict(w=odd(1)), dict(dtype=3), dict(H=-1), dict(rows=0), dict(cols=0), dict(q=None), dict(q=odd(8)),
               dict(s=None), dict(s=odd(2)), dict(err=None)):
        assert _pack(L, **kw) == tacg.E_INVAL, kw
    for kw in (dict(cols=65537), dict(rows=65537), dict(H=257)):
        assert _pack(L, **kw) == tacg.E_UNSUPPORTED, kw
    assert _pack(L, H=0, w=None) == tacg.OK


def _expert(L, **kw):
    a = dict(x=FAKE, dtype=1, xs=None, st=64, ss=0, T=4, k=2, E=8, ids=FAKE, slot=None, H=8, w=FAKE, s=FAKE, N=16, K=64, mode=0,
             gate=None, out=FAKE, od=1, err=FAKE, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    return L.tacg_expert_i8(a["x"], a["dtype"], a["xs"], a["st"], a["ss"], a["T"], a["k"], a["E"], a["ids"], a["slot"], a["H"],
                            a["w"], a["s"], a["N"], a["K"], a["mode"], a["gate"], a["out"], a["od"], a["err"], a["ws"], a["wsb"],
                            None)


def test_products_refuse(L):
    for kw in (dict(x=None), dict(x=odd(1)), dict(x=odd(2), dtype=0), dict(dtype=4), dict(dtype=-1), dict(xs=FAKE), dict(st=-1),
               dict(ss=-1), dict(T=-1), dict(k=0), dict(k=9), dict(E=0), dict(H=-1), dict(w=None), dict(w=odd(8)), dict(s=None),
               dict(s=odd(2)), dict(N=0), dict(K=0), dict(mode=3), dict(mode=-1), dict(mode=1, N=17), dict(out=None), dict(out=odd(1)),
               dict(out=odd(2), od=0), dict(od=3), dict(err=None), dict(T=400, ws=None), dict(T=400, wsb=64), dict(T=400, ws=odd(64)),
               dict(ids=None), dict(ids=None, k=8, slot=FAKE),                                  # shared: k experts, no table
               dict(dtype=3), dict(dtype=3, xs=FAKE, x=odd(8)), dict(dtype=3, xs=FAKE, st=72), dict(dtype=3, xs=FAKE, ss=8),
               dict(dtype=3, xs=odd(2))):
        assert _expert(L, **kw) == tacg.E_INVAL, kw
    for kw in (dict(N=65537), dict(K=65537), dict(H=257), dict(E=257), dict(k=17, E=32), dict(T=1 << 26), dict(ids=None, k=17, H=17)):
        assert _expert(L, **kw) == tacg.E_UNSUPPORTED, kw
    assert _expert(L, T=0, x=None, ids=None, k=8, out=None, ws=None, wsb=0) == tacg.OK


def test_workspace(L):
    need = lambda *a: L.tacg_expert_i8_workspace_bytes(*a)  # noqa: E731
    assert need(4, 2, 8, 8, 16, 64, 0, 1, 0) == 0                                  # few pairs: none
    assert need(400, 2, 8, 8, 16, 64, 0, 1, 0) % 256 == 0
    assert need(400, 2, 8, 8, 16, 64, 0, 1, 0) >= 400 * 64 + 4 * 400 + 4 * 800     # levels, scales, the order of the pairs
    assert need(400, 2, 8, 8, 16, 65, 2, 1, 1) >= 800 * 128 + 4 * 800 + 4 * 800 * 17
    assert need(400, 2, 8, 8, 16, 64, 0, 3, 0) < 400 * 64                          # levels are there
    for bad in ((-1, 2, 8, 8, 16, 64, 0, 1, 0), (4, 0, 8, 8, 16, 64, 0, 1, 0), (4, 2, -1, 8, 16, 64, 0, 1, 0), (4, 2, 8, -1, 16, 64, 0, 1, 0),
                (4, 2, 8, 8, 0, 64, 0, 1, 0), (4, 2, 8, 8, 16, 0, 0, 1, 0)):
        assert need(*bad) == 0


def test_binding_checks():
    x, ids = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((4, 2), dtype=torch.int16)
    q, s = torch.zeros((3, 1, 1, 4, 16, 16), dtype=torch.int8), torch.zeros((3, 16))
    bad = lambda *a, **kw: pytest.raises(ValueError, tacg.expert_i8, *a, **kw)  # noqa: E731
    bad(x, ids, q, s)                                    # not on a device
    bad(x, ids, q, s, mode="mean")
    bad(x.double(), ids, q, s)
    bad((x, s), ids, q, s)
    bad(x, ids, q[0], s)
    bad(x, ids, q, s[0])
    pytest.raises(ValueError, tacg.token_i8, x)
    pytest.raises(ValueError, tacg.token_i8, x.double())
    pytest.raises(ValueError, tacg.i8_pack, torch.zeros((2, 4, 64)))
    pytest.raises(ValueError, tacg.i8_pack, torch.zeros((4, 64)))


def test_reference_against_closed_forms():
    q, s = ref.levels(torch.tensor([[1.0, -2.0, 0.5, 1.0]]))
    assert q.tolist() == [[64, -127, 32, 64]] and abs(float(s[0]) - 2 / 127) < 1e-15       # 63.5 and 31.75
    assert ref.levels(torch.zeros((1, 3)))[0].tolist() == [[0, 0, 0]]
    level = torch.arange(2 * 17 * 70).reshape(2, 17, 70) % 255 - 127
    t = ref.tiles(level)
    assert t.shape == (2, 2, 2, 4, 16, 16) and int(t[1, 1, 1, 0, 0, 5]) == int(level[1, 16, 69]) and not t[:, 1, :, :, 1:].any()
    y, _ = ref.products(torch.tensor([[1, 2]]), torch.tensor([0.5]), torch.tensor([[1, -1]]), torch.tensor([[[9, 9]], [[3, 4]]]),
                        torch.ones((2, 1)), "each")
    assert y.tolist() == [[[5.5], [0.0]]]
