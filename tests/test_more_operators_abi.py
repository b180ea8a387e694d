"""CPU checks of block norm, balance loss, 8-bit rows and their products: bad
arguments are refused on the host, before any HIP call, and the workspace queries
follow their sizes.  No kernel runs here."""
import ctypes

import pytest
import torch

import paper_2608_03676_amd as taot

P = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first
NAN, INF = float("nan"), float("inf")


def block_norm(x=P, r=P, post=P, gate=P, gates=2, w=P, T=4, H=64, dt=0, wdt=0, gdt=0, eps=1e-6, alpha=1.0, h=P, y=P):
    return taot.lib().taot_block_norm(x, r, post, gate, gates, w, T, H, dt, wdt, gdt, eps, alpha, h, y, None, None, None)


def block_norm_backward(dy=P, dh=P, x=P, h=P, rx=P, rh=P, post=P, gate=P, gates=2, w=P, T=4, H=64, dt=0, wdt=0, gdt=0,
                        alpha=1.0, dx=P, dr=P, dw=P, dp=P, dg=P, ws=P, n=1 << 40):
    return taot.lib().taot_block_norm_backward(dy, dh, x, h, rx, rh, post, gate, gates, w, T, H, dt, wdt, gdt, alpha, dx, dr,
                                               dw, dp, dg, ws, n, None)


def balance(x=P, ids=P, m=None, rows=1, tokens=4, E=64, k=8, flags=0, dt=0, loss=P, z=None, c=P, p=P, ws=P, n=1 << 40):
    return taot.lib().taot_balance_loss(x, ids, m, rows, tokens, E, k, flags, dt, loss, z, c, p, None, ws, n, None)


def balance_backward(dl=P, dz=None, x=P, c=P, n=P, rows=1, tokens=4, E=64, flags=0, dt=0, out=P):
    return taot.lib().taot_balance_loss_backward(dl, dz, x, c, n, None, None, rows, tokens, E, flags, dt, out, None)


def quantize(x=P, T=4, H=64, gated=0, dt=0, q=P, s=P):
    return taot.lib().taot_quantize_rows(x, T, H, gated, dt, q, s, None)


def product(x=P, s=P, w=P, ws_=P, off=P, e=P, M=4, N=8, K=16, runs=2, G=2, dt=0, out=P, ws=P, n=1 << 40):
    return taot.lib().taot_matmul_i8(x, s, w, ws_, off, e, M, N, K, runs, G, dt, out, ws, n, None)


@pytest.mark.parametrize("call,code,cases", [
    (block_norm, 1, [dict(T=-1), dict(H=0), dict(dt=3), dict(wdt=1), dict(gdt=1), dict(gdt=7), dict(eps=-1.0), dict(eps=NAN),
                     dict(eps=INF), dict(alpha=NAN), dict(alpha=INF), dict(gates=0), dict(gates=3), dict(gates=-2),
                     dict(w=None), dict(x=None), dict(r=None)]),
    (block_norm, 2, [dict(H=32769), dict(T=1 << 31)]),
    (block_norm, 0, [dict(T=0), dict(T=0, x=None)]),
    (block_norm_backward, 1, [dict(T=-1), dict(H=0), dict(dt=3), dict(wdt=1), dict(gdt=1), dict(alpha=NAN), dict(gates=3),
                              dict(dy=None), dict(h=None), dict(rh=None), dict(rx=None), dict(x=None), dict(dx=None),
                              dict(dr=None), dict(w=None), dict(w=None, dw=None, dh=None), dict(post=None), dict(gate=None)]),
    (block_norm_backward, 2, [dict(H=32769), dict(T=1 << 31)]),
    (block_norm_backward, 3, [dict(ws=None), dict(n=16)]),
    (balance, 1, [dict(rows=-1), dict(tokens=-1), dict(E=0), dict(k=0), dict(flags=2), dict(flags=1, z=P), dict(dt=3),
                  dict(x=None), dict(ids=None), dict(loss=None), dict(c=None), dict(p=None)]),
    (balance, 2, [dict(E=32769), dict(k=65), dict(tokens=1 << 31), dict(rows=1 << 16, tokens=1 << 14)]),
    (balance, 3, [dict(ws=None), dict(n=16)]),
    (balance, 0, [dict(rows=0)]),
    (balance_backward, 1, [dict(rows=-1), dict(tokens=-1), dict(E=0), dict(flags=4), dict(flags=1, dz=P), dict(dt=-1),
                           dict(dl=None), dict(x=None), dict(c=None), dict(n=None), dict(out=None)]),
    (balance_backward, 2, [dict(E=32769), dict(tokens=1 << 31), dict(rows=1 << 16, tokens=1 << 16)]),
    (balance_backward, 0, [dict(rows=0), dict(tokens=0)]),
    (quantize, 1, [dict(T=-1), dict(H=0), dict(gated=2), dict(dt=3), dict(x=None), dict(q=None), dict(s=None)]),
    (quantize, 2, [dict(H=32769), dict(T=1 << 31)]),
    (quantize, 0, [dict(T=0)]),
    (product, 1, [dict(M=-1), dict(N=0), dict(K=0), dict(runs=-1), dict(G=0), dict(dt=3), dict(off=None),
                  dict(off=None, e=None, runs=0), dict(off=None, runs=0, G=1), dict(x=None), dict(s=None), dict(w=None),
                  dict(ws_=None), dict(out=None)]),
    (product, 2, [dict(K=131072), dict(M=(1 << 30) + 1), dict(N=(1 << 30) + 1), dict(runs=(1 << 30) + 1)]),
    (product, 3, [dict(ws=None), dict(n=16)]),
    (product, 0, [dict(M=0)]),
])
def test_host_validation(call, code, cases):
    for c in cases:
        assert call(**c) == code, (call.__name__, c)


def test_workspace_sizes():
    L = taot.lib()
    size = L.taot_block_norm_backward_workspace_size
    assert size(0, 64, 1) == 0 and size(4, 0, 1) == 0 and size(5, 64, 2) == 0 and size(8, 64, 0) >= 2 * 8 * 64 * 4
    assert size(100000, 4096, 1) == size(1000000, 4096, 1)  # the workers are bounded, not the rows
    assert size(1 << 20, 64, 1 << 20) <= 2 * 4 * 64 * 4096 + 512  # nor by the gates
    size = L.taot_balance_loss_workspace_size
    assert size(0, 4, 8) == 0 and size(1, -1, 8) == 0 and size(1, 0, 8) > 0
    assert size(1, 1 << 20, 256) == size(1, 1 << 24, 256) and size(1 << 20, 1, 32) <= size(4096, 1, 32)
    size = L.taot_matmul_i8_workspace_size
    assert size(-1, 2) == 0 and size(4, -1) == 0 and size(4096, 64) > size(64, 64) > 0


def test_tensors_off_the_gpu_are_refused():
    x, one = torch.zeros(4, 64), torch.zeros(4)
    ids = torch.zeros(4, 2, dtype=torch.int32)
    i8 = x.to(torch.int8)
    for call in (lambda: taot.block_norm(x, x, x[0], 1e-6), lambda: taot.block_norm_backward(x, x, x, one, x[0]),
                 lambda: taot.balance_loss(x, ids), lambda: taot.balance_loss_backward(one, x, ids, ids),
                 lambda: taot.quantize_rows(x), lambda: taot.matmul_i8(i8, one, i8, one)):
        with pytest.raises(TypeError):
            call()
