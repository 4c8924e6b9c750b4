"""What the routing calls and the norm refuse, before anything reaches a device."""
import ctypes

import pytest
import torch

from util import ensure_built

ensure_built()
import paper_2511_18297_amd as G  # noqa: E402

L = G.binding._lib
MB = 1 << 20
FIRST = 1 << 30                                            # where the first buffer lies


class Buffers:
    """Addresses that are never read: a few megabytes apart, 256-byte aligned."""

    def __init__(self):
        self.at = FIRST

    def __call__(self, mb=1):
        p = self.at
        self.at += mb * MB
        return p


def route(**change):
    b = Buffers()
    a = dict(dtype=1, s=b(), ss=64, bias=b(), gate=0, sets=8, open=2, best=2, renorm=1, factor=1.0, e=b(), w=b(), p=b(), off=b(), n=100, E=64, k=4, ws=b(),
             wb=MB)
    a.update(change)
    return L.groot_route(a["dtype"], a["s"], a["ss"], a["bias"], a["gate"], a["sets"], a["open"], a["best"], a["renorm"], a["factor"], a["e"], a["w"], a["p"],
                         a["off"], a["n"], a["E"], a["k"], a["ws"], a["wb"], None)


def route_backward(**change):
    b = Buffers()
    a = dict(dtype=1, s=b(), ss=64, gate=0, renorm=1, factor=1.0, e=b(), dw=b(), ds=b(), dss=64, n=100, E=64, k=4)
    a.update(change)
    return L.groot_route_backward(a["dtype"], a["s"], a["ss"], a["gate"], a["renorm"], a["factor"], a["e"], a["dw"], a["ds"], a["dss"], a["n"], a["E"],
                                  a["k"], None)


def rows(**change):
    b = Buffers()
    a = dict(dtype=1, X=b(), xs=64, sc=b(), p=b(), k=4, R=b(), rs=64, rsc=b(), n=100, m=400, K=64)
    a.update(change)
    return L.groot_routed_rows(a["dtype"], a["X"], a["xs"], a["sc"], a["p"], a["k"], a["R"], a["rs"], a["rsc"], a["n"], a["m"], a["K"], None)


def total(**change):
    b = Buffers()
    a = dict(dtype=1, R=b(), rs=64, p=b(), w=b(), add=b(), adds=64, k=4, out=b(), os=64, n=100, m=400, K=64)
    a.update(change)
    return L.groot_routed_sum(a["dtype"], a["R"], a["rs"], a["p"], a["w"], a["add"], a["adds"], a["k"], a["out"], a["os"], a["n"], a["m"], a["K"], None)


def total_backward(**change):
    b = Buffers()
    a = dict(dtype=1, d=b(), dstr=64, R=b(), rs=64, p=b(), w=b(), k=4, dR=b(), drs=64, dw=b(), n=100, m=400, K=64)
    a.update(change)
    return L.groot_routed_sum_backward(a["dtype"], a["d"], a["dstr"], a["R"], a["rs"], a["p"], a["w"], a["k"], a["dR"], a["drs"], a["dw"], a["n"], a["m"],
                                       a["K"], None)


def norm(**change):
    b = Buffers()
    a = dict(dtype=1, X=b(), xs=64, r=b(), rs=64, g=b(), eps=1e-6, H=b(), hs=64, Y=b(), ys=64, Q=b(), qs=64, sc=b(), rstd=b(), n=100, K=64)
    a.update(change)
    return L.groot_rms_norm(a["dtype"], a["X"], a["xs"], a["r"], a["rs"], a["g"], a["eps"], a["H"], a["hs"], a["Y"], a["ys"], a["Q"], a["qs"], a["sc"],
                            a["rstd"], a["n"], a["K"], None)


def norm_backward(**change):
    b = Buffers()
    a = dict(dtype=1, H=b(), hs=64, rstd=b(), g=b(), dY=b(), dys=64, dH=b(), dhs=64, dX=b(), dxs=64, gd=0, dg=b(), n=100, K=64, ws=b(), wb=MB)
    a.update(change)
    return L.groot_rms_norm_backward(a["dtype"], a["H"], a["hs"], a["rstd"], a["g"], a["dY"], a["dys"], a["dH"], a["dhs"], a["dX"], a["dxs"], a["gd"],
                                     a["dg"], a["n"], a["K"], a["ws"], a["wb"], None)


def at(buffer, more=0):
    return FIRST + buffer * MB + more


NAN, INF = float("nan"), float("inf")
GATE = [dict(dtype=3), dict(dtype=-1), dict(n=-1), dict(E=0), dict(E=1025, ss=2000, dss=2000, sets=1, open=1), dict(k=0), dict(k=33), dict(k=65), dict(gate=2),
        dict(gate=-1), dict(renorm=2), dict(factor=NAN), dict(factor=INF), dict(factor=1e39), dict(s=None), dict(ss=63), dict(s=at(0, 1)), dict(e=None),
        dict(e=at(2, 2)), dict(ss=1 << 62)]
ROUTED = [dict(dtype=7), dict(dtype=-1), dict(n=-1), dict(m=-1), dict(k=0), dict(k=33), dict(K=0), dict(K=65537, xs=70000, rs=70000, os=70000, adds=70000, dstr=70000, drs=70000),
          dict(p=None), dict(p=at(2, 2)), dict(rs=63)]


@pytest.mark.parametrize("call, changes", [
    (route, GATE + [dict(sets=0), dict(sets=7), dict(sets=65, E=65, ss=65, open=1, best=1, k=1), dict(open=0), dict(open=9), dict(best=0), dict(best=3),
                    dict(sets=64, open=64, best=2), dict(open=1, k=9), dict(w=None), dict(p=None), dict(off=None), dict(off=at(5, 4)), dict(bias=at(1, 2)), dict(ws=None),
                    dict(wb=16), dict(ws=at(6, 8)), dict(e=at(0)), dict(w=at(1)), dict(p=at(2)), dict(off=at(0, 8)), dict(ws=at(3)), dict(off=at(4))]),
    (route_backward, GATE + [dict(dw=None), dict(ds=None), dict(dss=63), dict(ds=at(0)), dict(ds=at(1)), dict(ds=at(2)), dict(dw=at(2, 1))]),
    (rows, ROUTED + [dict(X=None), dict(R=None), dict(xs=63), dict(X=at(0, 1)), dict(R=at(0)), dict(R=at(2)), dict(sc=None), dict(rsc=None), dict(rsc=at(0)), dict(R=at(4)),
                     dict(dtype=3, xs=63)]),
    (total, ROUTED + [dict(dtype=3), dict(R=None), dict(out=None), dict(os=63), dict(adds=63), dict(w=at(2, 2)), dict(out=at(0)), dict(out=at(1)), dict(out=at(2)),
                      dict(out=at(3)), dict(out=at(3, 64))]),
    (total_backward, ROUTED + [dict(dtype=3), dict(d=None), dict(dstr=63), dict(R=None), dict(drs=63), dict(dR=None, dw=None), dict(dR=at(0)), dict(dR=at(1)), dict(dR=at(2)),
                               dict(dw=at(3)), dict(dw=at(4)), dict(dw=at(5, 2))]),
    (norm, [dict(dtype=3), dict(n=-1), dict(K=0), dict(K=65537, xs=70000, rs=70000, hs=70000, ys=70000, qs=70000), dict(X=None), dict(xs=63), dict(rs=63), dict(hs=63), dict(ys=63),
            dict(qs=63), dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(eps=1e-50), dict(Q=None), dict(sc=None), dict(g=at(2, 1)), dict(sc=at(6, 2)),
            dict(H=None, Y=None, Q=None, sc=None, rstd=None), dict(H=at(0, 128)), dict(Y=at(1, 128)), dict(Y=at(0), ys=65), dict(H=at(4)), dict(Q=at(0)), dict(Q=at(2)), dict(rstd=at(1)),
            dict(H=at(2)), dict(sc=at(5)), dict(H=at(0), Y=at(0)), dict(n=1 << 41)]),
    (norm_backward, [dict(dtype=4), dict(gd=2), dict(n=-1), dict(K=0), dict(H=None), dict(rstd=None), dict(dY=None), dict(dX=None), dict(hs=63), dict(dys=63), dict(dhs=63),
                     dict(dxs=63), dict(ws=None), dict(wb=64), dict(ws=at(7, 8)), dict(dX=at(0)), dict(dX=at(3)), dict(dX=at(4)), dict(dg=at(2)), dict(dg=at(5)), dict(ws=at(5)),
                     dict(g=at(2, 1)), dict(dg=at(6, 2)), dict(rstd=at(1, 2))]),
])
def test_refused(call, changes):
    for change in changes:
        assert call(**change) == G.GROOT_EINVAL, change
        assert G.groot_last_error().startswith("groot_r"), change


def test_too_many_slots():
    big = dict(n=1 << 30, k=2)
    for call in (route, route_backward, rows, total, total_backward):
        assert call(**big) == G.GROOT_ERANGE
    for call in (rows, total, total_backward):
        assert call(m=1 << 31) == G.GROOT_ERANGE


def test_nothing_to_do():
    none = dict(n=0)
    assert route_backward(**none) == rows(**none) == total(**none) == total_backward(**none) == norm(**none) == G.GROOT_OK
    assert norm_backward(n=0, dg=None) == rows(m=0, R=None, rsc=None) == G.GROOT_OK


def test_workspaces():
    b = ctypes.c_size_t(7)
    assert L.groot_route_workspace(64, 256, 8, ctypes.byref(b)) == G.GROOT_OK
    for n, E, k in ((1, 1, 1), (65, 64, 4), (1 << 20, 1024, 32)):
        size = G.groot_route_workspace(n, E, k)
        assert 0 <= size <= (n // 16 + 2) * E * 4
    for n, K in ((1, 1), (1 << 23, 64), (16384, 4096), (5, 65536)):
        for T in (torch.float32, torch.bfloat16, torch.float16):
            size = G.groot_rms_norm_backward_workspace(n, K, T)
            assert 0 < size <= 64 << 20 or K == 65536, (n, K, size)
    assert G.groot_rms_norm_backward_workspace(0, 64, torch.float32) >= 0
    for call in (lambda: G.groot_route_workspace(1, 0, 1), lambda: G.groot_route_workspace(1, 8, 9), lambda: G.groot_rms_norm_backward_workspace(-1, 8, torch.float32)):
        with pytest.raises(G.GrootError):
            call()
    assert L.groot_route_workspace(64, 256, 8, None) == L.groot_rms_norm_backward_workspace(0, 64, 64, None) == G.GROOT_EINVAL
    with pytest.raises(TypeError):
        G.groot_rms_norm_backward_workspace(1, 8, torch.int8)


def test_tensors_on_the_host_are_refused():
    x, i = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(TypeError):
        G.groot_route(x, None, i, torch.zeros(4, 2), i.clone(), torch.zeros(9, dtype=torch.int64), None)
    with pytest.raises(TypeError):
        G.groot_route_backward(x, i, torch.zeros(4, 2), torch.zeros(4, 8))
    with pytest.raises(TypeError):
        G.groot_routed_rows(x, i, torch.zeros(8, 8))
    with pytest.raises(TypeError):
        G.groot_routed_sum(torch.zeros(8, 8), i, None, None, x)
    with pytest.raises(TypeError):
        G.groot_routed_sum_backward(x, None, i, None, torch.zeros(8, 8), None)
    with pytest.raises(TypeError):
        G.groot_rms_norm(x, None, None, 1e-6, torch.zeros(4, 8))
    with pytest.raises(TypeError):
        G.groot_rms_norm_backward(x, torch.zeros(4), None, x.clone(), x.clone(), None, None)
