"""CPU checks of the calls around the planner: bad arguments are refused on the
host, before any HIP call, and the workspace queries follow their sizes.  No
kernel runs here."""
import ctypes

import pytest
import torch

import paper_2608_03676_amd as taot

P = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first
NAN, INF = float("nan"), float("inf")


def norm(x=P, res=None, w=P, T=4, H=64, dt=0, wdt=0, eps=1e-6, group=0, h=None, y=P, q=None, s=None, r=None):
    return taot.lib().taot_add_rms_norm(x, res, w, T, H, dt, wdt, eps, group, h, y, q, s, r, None)


def norm_backward(dy=P, h=P, r=P, w=P, T=4, H=64, dt=0, wdt=0, dx=P, dw=P, ws=P, n=1 << 40):
    return taot.lib().taot_add_rms_norm_backward(dy, None, h, r, w, T, H, dt, wdt, dx, dw, ws, n, None)


def route(x=P, T=4, E=64, k=8, groups=1, top=1, scale=1.0, flags=0, dt=0, ids=P, w=P):
    return taot.lib().taot_route(x, None, T, E, k, groups, top, scale, flags, dt, ids, w, None)


def route_backward(dw=P, x=P, ids=P, T=4, E=64, k=8, scale=1.0, flags=0, dt=0, out=P):
    return taot.lib().taot_route_backward(dw, x, ids, T, E, k, scale, flags, dt, out, None)


def dispatch_map(ids=P, B=1, rows=1, rank0=0, N=8, home=P, R=4, E=8, K=2, slot=P, X=P, pos=P, off=P, sends=P, ws=P,
                 n=1 << 40):
    return taot.lib().taot_dispatch_map(ids, B, rows, rank0, N, home, R, E, K, slot, X, pos, off, sends, None, ws, n,
                                        None)


def rows(x=P, nb=16, more=None, mb=0, r=1, t=4, k=2, pos=P, out=P, om=None):
    return taot.lib().taot_dispatch_rows(x, nb, more, mb, r, t, k, pos, out, om, None)


def combine(y=P, pos=P, w=None, r=1, t=4, k=2, H=8, dt=0, out=P):
    return taot.lib().taot_combine_rows(y, pos, w, r, t, k, H, dt, out, None)


def combine_backward(d=P, y=P, pos=P, w=P, r=1, t=4, k=2, H=8, dt=0, dy=P, dw=P):
    return taot.lib().taot_combine_rows_backward(d, y, pos, w, r, t, k, H, dt, dy, dw, None)


@pytest.mark.parametrize("call,code,cases", [
    (norm, 1, [dict(T=-1), dict(H=0), dict(dt=3), dict(dt=-1), dict(dt=0, wdt=1), dict(wdt=7), dict(eps=-1.0),
               dict(eps=NAN), dict(eps=INF), dict(group=4), dict(group=24), dict(group=1024), dict(group=-8),
               dict(q=P), dict(s=P), dict(x=None), dict(w=None)]),
    (norm, 2, [dict(H=32769), dict(T=1 << 31)]),
    (norm, 0, [dict(T=0), dict(T=0, x=None)]),
    (norm_backward, 1, [dict(T=-1), dict(H=0), dict(dt=5), dict(wdt=1), dict(dy=None), dict(h=None), dict(r=None),
                        dict(w=None), dict(dx=None), dict(dw=None)]),
    (norm_backward, 2, [dict(H=32769), dict(T=1 << 31)]),
    (norm_backward, 3, [dict(ws=None), dict(n=16)]),
    (route, 1, [dict(T=-1), dict(E=0), dict(k=0), dict(k=65, E=64), dict(groups=0), dict(groups=3), dict(top=0),
                dict(groups=4, top=5), dict(groups=16, top=1), dict(scale=NAN), dict(scale=INF), dict(flags=8),
                dict(dt=3), dict(x=None), dict(ids=None), dict(w=None)]),
    (route, 2, [dict(E=32769), dict(E=100, k=65), dict(E=512, groups=512, top=512), dict(T=1 << 31)]),
    (route, 0, [dict(T=0), dict(T=0, x=None)]),
    (route_backward, 1, [dict(T=-1), dict(E=0), dict(k=0), dict(k=65), dict(scale=NAN), dict(flags=16), dict(dt=3),
                         dict(dw=None), dict(x=None), dict(ids=None), dict(out=None)]),
    (route_backward, 2, [dict(E=32769), dict(E=100, k=65), dict(T=1 << 31)]),
    (route_backward, 0, [dict(T=0)]),
    (dispatch_map, 1, [dict(B=-1), dict(rows=0), dict(rank0=-1), dict(rank0=4), dict(rank0=2, rows=3), dict(N=-1),
                       dict(R=0, rows=0), dict(E=0), dict(K=-1), dict(ids=None), dict(home=None), dict(slot=None),
                       dict(X=None), dict(pos=None), dict(off=None), dict(sends=None)]),
    (dispatch_map, 2, [dict(R=2049), dict(E=32769), dict(K=65), dict(N=1 << 31), dict(B=1 << 29, rows=4)]),
    (dispatch_map, 3, [dict(ws=None), dict(n=64)]),
    (dispatch_map, 0, [dict(B=0)]),
    (rows, 1, [dict(nb=0), dict(mb=-1), dict(mb=4), dict(more=P), dict(mb=4, more=P), dict(r=-1), dict(t=-1),
               dict(k=0), dict(x=None), dict(pos=None), dict(out=None)]),
    (rows, 2, [dict(k=65), dict(t=1 << 31), dict(t=1 << 30), dict(r=1 << 20, t=1 << 20), dict(nb=1 << 31)]),
    (rows, 0, [dict(r=0), dict(t=0)]),
    (combine, 1, [dict(r=-1), dict(t=-1), dict(k=0), dict(H=0), dict(dt=3), dict(y=None), dict(pos=None),
                  dict(out=None)]),
    (combine, 2, [dict(k=65), dict(t=1 << 31), dict(H=(1 << 30) + 1)]),
    (combine, 0, [dict(r=0), dict(t=0)]),
    (combine_backward, 1, [dict(r=-1), dict(t=-1), dict(k=0), dict(H=0), dict(dt=3), dict(d=None), dict(y=None),
                           dict(pos=None), dict(w=None), dict(dy=None), dict(dw=None)]),
    (combine_backward, 2, [dict(k=65), dict(t=1 << 31)]),
    (combine_backward, 0, [dict(r=0), dict(t=0)]),
])
def test_host_validation(call, code, cases):
    for c in cases:
        assert call(**c) == code, (call.__name__, c)


def test_workspace_sizes():
    L = taot.lib()
    size = L.taot_add_rms_norm_backward_workspace_size
    assert size(-1, 8) == 0 and size(4, 0) == 0 and size(8, 64) >= 8 * 64 * 4
    assert size(100000, 4096) == size(1000000, 4096)  # the workers are bounded, not the rows
    size = L.taot_dispatch_map_workspace_size
    assert size(1, 1, 100, 4, 0, 2) == 0 and size(1, 0, 100, 4, 8, 2) == 0 and size(1, 1, -1, 4, 8, 2) == 0
    assert size(2, 4, 5000, 16, 64, 2) > size(1, 4, 5000, 16, 64, 2) > size(1, 1, 5000, 16, 64, 2)


def test_tensors_off_the_gpu_are_refused():
    x = torch.zeros(4, 64)
    ids = torch.zeros(1, 1, 8, dtype=torch.int32)
    with pytest.raises(TypeError):
        taot.add_rms_norm(x, x[0], 1e-6)
    with pytest.raises(TypeError):
        taot.route(x, 8)
    with pytest.raises(TypeError):
        taot.dispatch_map(ids, ids[0, 0], ids[0], ids, 2)
    with pytest.raises(TypeError):
        taot.dispatch_rows(x, ids[0, 0])
    with pytest.raises(TypeError):
        taot.combine_rows(x, ids[0, 0])
