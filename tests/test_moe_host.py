"""Host-side checks of the router's and the experts' entry points (CPU only): sizes of workspaces, refused arguments, and the binding's
checks of types, shapes and strides."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2606_01007_amd as tacg

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "tacg.h")
FAKE = ctypes.c_void_p(1 << 20)   # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(tacg.LIB_PATH):
        pytest.skip("libtacg.so not built")
    return tacg.lib()


def test_exports_and_constants(L):
    text = open(HEADER).read()
    for name in ("tacg_route", "tacg_route_workspace_bytes", "tacg_route_backward", "tacg_q4_pack", "tacg_expert_q4",
                 "tacg_expert_q4_workspace_bytes"):
        assert re.search(rf"\b{name}\(", text) and hasattr(L, name), name
    value = lambda n: int(re.search(rf"#define {n} (\S+?)u?\s", text).group(1), 0)  # noqa: E731
    assert [value(f"TACG_{n}") for n in ("F32", "BF16", "F16")] == [
        tacg.DTYPES[t] for t in (torch.float32, torch.bfloat16, torch.float16)]
    assert {m: value(f"TACG_Q4_{m.upper()}") for m in tacg.Q4_MODES} == tacg.Q4_MODES
    assert {m: value(f"TACG_{m.upper()}") for m in tacg.SCORES} == tacg.SCORES
    assert value("TACG_ERR_VALUE") == tacg.ERR_VALUE


def _off(*v):
    return np.array(v, dtype=np.int64)


def _route(L, **kw):
    a = dict(x=FAKE, dtype=0, sl=800, st=8, N=100, Ly=2, k=2, E=8, off=_off(0, 50, 100), F=2, score=0, bias=None, renorm=0,
             scale=1.0, trace=FAKE, gate=FAKE, norm=None, D=None, tokens=None, balance=None, z=None, err=FAKE, ws=None, wsb=0)
    a.update(kw)
    off = a["off"]
    return L.tacg_route(a["x"], a["dtype"], a["sl"], a["st"], a["N"], a["Ly"], a["k"], a["E"],
                        None if off is None else off.ctypes.data_as(ctypes.c_void_p), a["F"], a["score"], a["bias"],
                        a["renorm"], a["scale"], a["trace"], a["gate"], a["norm"], a["D"], a["tokens"], a["balance"], a["z"],
                        a["err"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(x=ctypes.c_void_p((1 << 20) + 2)), dict(x=ctypes.c_void_p((1 << 20) + 1), dtype=1), dict(dtype=3),
    dict(dtype=-1), dict(sl=-1), dict(st=-8), dict(N=-1), dict(Ly=0), dict(k=0), dict(k=9), dict(E=0), dict(off=None),
    dict(off=_off(0, 60, 50)), dict(off=_off(1, 60, 100)), dict(off=_off(0, 60, 99)), dict(F=0), dict(score=2), dict(renorm=2),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(trace=None), dict(gate=None), dict(err=None),
    dict(D=FAKE), dict(tokens=FAKE, balance=FAKE), dict(z=FAKE),
    dict(D=FAKE, tokens=FAKE, balance=FAKE),                                                        # no workspace
    dict(D=FAKE, tokens=FAKE, balance=FAKE, ws=FAKE, wsb=64),
    dict(D=FAKE, tokens=FAKE, balance=FAKE, ws=ctypes.c_void_p((1 << 20) + 64), wsb=1 << 30),
    dict(D=FAKE, tokens=FAKE, balance=FAKE, z=FAKE, score=1, ws=FAKE, wsb=1 << 30),
])
def test_route_refuses(L, kw):
    assert _route(L, **kw) == tacg.E_INVAL


def test_route_limits(L):
    assert _route(L, E=257, k=2) == tacg.E_UNSUPPORTED
    assert _route(L, E=32, k=17) == tacg.E_UNSUPPORTED
    assert _route(L, F=65, off=np.zeros(66, dtype=np.int64), N=0) == tacg.E_UNSUPPORTED
    assert _route(L, Ly=65536) == tacg.E_UNSUPPORTED
    assert _route(L, N=1 << 31, off=_off(0, 1, 1 << 31)) == tacg.E_UNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(norm=None), dict(grad=None), dict(grad=ctypes.c_void_p((1 << 20) + 2)), dict(dtype=7), dict(k=9),
    dict(gg=FAKE, trace=None), dict(gb=FAKE, D=None), dict(gb=FAKE, tokens=None), dict(gz=FAKE, tokens=None),
    dict(gz=FAKE, score=1), dict(off=_off(0, 5)), dict(sl=-1), dict(scale=float("nan")),
])
def test_route_backward_refuses(L, kw):
    a = dict(x=FAKE, dtype=0, sl=800, st=8, N=100, Ly=2, k=2, E=8, off=_off(0, 100), F=1, score=0, renorm=0, scale=1.0,
             trace=FAKE, norm=FAKE, D=FAKE, tokens=FAKE, gg=None, gb=None, gz=None, grad=FAKE)
    a.update(kw)
    st = L.tacg_route_backward(a["x"], a["dtype"], a["sl"], a["st"], a["N"], a["Ly"], a["k"], a["E"],
                               a["off"].ctypes.data_as(ctypes.c_void_p), a["F"], a["score"], a["renorm"], a["scale"],
                               a["trace"], a["norm"], a["D"], a["tokens"], a["gg"], a["gb"], a["gz"], a["grad"], None)
    assert st == tacg.E_INVAL


def _pack(L, **kw):
    a = dict(w=FAKE, dtype=0, rows=8, cols=64, stride=64, group=32, sd=1, q=FAKE, s=FAKE, z=None, err=FAKE)
    a.update(kw)
    return L.tacg_q4_pack(a["w"], a["dtype"], a["rows"], a["cols"], a["stride"], a["group"], a["sd"], a["q"], a["s"], a["z"],
                          a["err"], None)


def test_pack_refuses(L):
    for kw in (dict(w=None), dict(dtype=3), dict(rows=-1), dict(cols=0), dict(stride=-1), dict(sd=0), dict(q=None),
               dict(q=ctypes.c_void_p((1 << 20) + 8)), dict(s=None), dict(s=ctypes.c_void_p((1 << 20) + 1)), dict(err=None),
               dict(w=ctypes.c_void_p((1 << 20) + 2))):
        assert _pack(L, **kw) == tacg.E_INVAL, kw
    for kw in (dict(group=48), dict(group=16), dict(group=512), dict(cols=65537), dict(rows=(1 << 26) + 1)):
        assert _pack(L, **kw) == tacg.E_UNSUPPORTED, kw
    assert _pack(L, rows=0) == tacg.OK


def _expert(L, **kw):
    a = dict(x=FAKE, dtype=1, st=64, ss=0, T=4, k=2, E=8, ids=FAKE, slot=None, H=8, q=FAKE, s=FAKE, z=None, group=32, N=16,
             K=64, mode=0, gate=None, out=FAKE, err=FAKE, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    return L.tacg_expert_q4(a["x"], a["dtype"], a["st"], a["ss"], a["T"], a["k"], a["E"], a["ids"], a["slot"], a["H"], a["q"],
                            a["s"], a["z"], a["group"], a["N"], a["K"], a["mode"], a["gate"], a["out"], a["err"], a["ws"],
                            a["wsb"], None)


def test_expert_refuses(L):
    for kw in (dict(x=None), dict(x=ctypes.c_void_p((1 << 20) + 1)), dict(dtype=0), dict(dtype=5), dict(st=-1), dict(ss=-1),
               dict(T=-1), dict(k=0), dict(k=9), dict(E=0), dict(ids=None), dict(H=-1), dict(q=None), dict(s=None),
               dict(q=ctypes.c_void_p((1 << 20) + 8)), dict(N=0), dict(K=0), dict(mode=3), dict(mode=1, N=15), dict(mode=2),
               dict(out=None), dict(err=None)):
        assert _expert(L, **kw) == tacg.E_INVAL, kw
    for kw in (dict(E=257), dict(k=17, E=32), dict(H=257), dict(group=33), dict(group=0), dict(N=65537), dict(K=65537),
               dict(T=1 << 30)):
        assert _expert(L, **kw) == tacg.E_UNSUPPORTED, kw
    assert _expert(L, T=0, x=None, ids=None, out=None) == tacg.OK
    for mode in (0, 1, 2):
        need = L.tacg_expert_q4_workspace_bytes(400, 8, 256, 64, 64, mode)
        if need:
            assert _expert(L, T=400, k=8, E=256, H=256, N=64, mode=mode, gate=FAKE, wsb=need - 1) == tacg.E_INVAL
            assert _expert(L, T=400, k=8, E=256, H=256, N=64, mode=mode, gate=FAKE, ws=None) == tacg.E_INVAL


def test_workspace_sizes(L):
    assert L.tacg_route_workspace_bytes(-1, 1, 8, 1) == 0 and L.tacg_route_workspace_bytes(8, 0, 8, 1) == 0
    a, b = L.tacg_route_workspace_bytes(1 << 20, 58, 256, 16), L.tacg_route_workspace_bytes(1 << 10, 58, 256, 16)
    assert a > b > 58 * 16 * 256 * 8 and a % 256 == 0
    assert L.tacg_expert_q4_workspace_bytes(-1, 1, 1, 1, 1, 0) == 0


def test_binding_checks():
    x = torch.zeros((2, 4, 8))
    with pytest.raises(ValueError, match="device"):
        tacg.route(x, 2)
    with pytest.raises(ValueError, match="logits"):
        tacg.route(x[0], 2)
    with pytest.raises(ValueError, match="logits"):
        tacg.route(x.double(), 2)
    with pytest.raises(ValueError, match="device"):
        tacg.route_backward(x, torch.zeros((2, 4, 2), dtype=torch.int16), x[:, :, 0])
    with pytest.raises(ValueError, match="weight"):
        tacg.q4_pack(x)
    ids = torch.zeros((4, 2), dtype=torch.int16)
    q, s = torch.zeros((8, 16, 16), dtype=torch.uint8), torch.zeros((8, 16, 1), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="ids"):
        tacg.expert_q4(x, ids.int(), q, s)
    with pytest.raises(ValueError, match="mode"):
        tacg.expert_q4(x, ids, q, s, mode="all")
    with pytest.raises(ValueError, match="x:"):
        tacg.expert_q4(x, ids, q, s)


@pytest.mark.gpu
def test_binding_checks_on_the_device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    x = torch.zeros((2, 4, 8), device="cuda")
    r = tacg.route(x, 2, balance=True)
    with pytest.raises(tacg.TacgError):
        tacg.route(x, 9)
    with pytest.raises(tacg.TacgError):
        tacg.route(x, 2, [0, 3])
    with pytest.raises(ValueError, match="score"):
        tacg.route(x, 2, score="linear")
    with pytest.raises(ValueError, match="contiguous"):
        tacg.route(x.transpose(1, 2), 2)
    with pytest.raises(ValueError, match="bias"):
        tacg.route(x, 2, bias=torch.zeros((8,), device="cuda"))
    with pytest.raises(ValueError, match="trace"):
        tacg.route(x, 2, out=dict(r, trace=r["trace"][:1]))
    with pytest.raises(ValueError, match="grad_balance"):
        tacg.route_backward(x, r["trace"], r["norm"], D=r["D"], tokens=r["tokens"],
                            grad_balance=torch.zeros((2, 1), device="cuda"))
    w = torch.zeros((4, 16, 64), device="cuda", dtype=torch.bfloat16)
    q, s, _ = tacg.q4_pack(w, group=32)
    ids = torch.zeros((3, 2), dtype=torch.int16, device="cuda")
    v = torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (dict(x=v[:, :32]), dict(x=v.half()), dict(x=v[:2]), dict(q=q[:, :, :16].contiguous()), dict(scales=s[:, :8]),
                dict(zeros=s), dict(group=64), dict(group=0), dict(out=v), dict(gate=v, mode="sum"),
                dict(slot_of_expert=torch.zeros(3, dtype=torch.int32, device="cuda")),
                dict(x=torch.zeros((64, 3), dtype=torch.bfloat16, device="cuda").t())):
        with pytest.raises(ValueError):
            tacg.expert_q4(**{**dict(x=v, ids=ids, q=q, scales=s, group=32), **bad})
    with pytest.raises(tacg.TacgError):
        tacg.expert_q4(v, ids, q, s, group=32, mode="sum")
    with pytest.raises(tacg.TacgError):
        tacg.q4_pack(w, group=48)
