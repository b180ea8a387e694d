"""The calls around the planner at sizes between those of the other tests: widths, numbers of experts and lengths whose
kernels those do not reach.  The checks and their tolerances are the other tests'."""
import pytest
import torch

import paper_2608_03676_amd as taot
import test_gpu_dispatch as dispatch
import test_gpu_norm as norm
import test_gpu_route as route
import test_gpu_route_groups as route_groups

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _gradients(gpu, T, H, dtype):
    g = torch.Generator().manual_seed(T + H)
    return [torch.randn(T, H, generator=g).to(dtype).to(gpu) for _ in range(2)]


# two chunks of columns a lane from 8193 columns on, four from 16385; more rows than workers; outputs past the caches
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H", [(1, 8193), (3, 12000), (700, 8200), (300, 16384), (700, 16385), (1100, 16384), (600, 30011)])
def test_norm_of_wide_rows_and_its_gradient(gpu, dtype, T, H):
    print(f"[norm] {dtype} {T} x {H}", flush=True)
    x, r, w = norm._inputs(gpu, T, H, dtype)
    n = taot.add_rms_norm(x, w, 1e-6, residual=r, group=256)
    norm._check_forward(n, x, r, w, 1e-6, 256)
    dy, dh = _gradients(gpu, T, H, dtype)
    norm._check_backward(taot.add_rms_norm_backward(dy, n.h, n.rstd, w, dh=dh), dy, dh, n.h, n.rstd, w)
    norm._check_backward(taot.add_rms_norm_backward(dy, n.h, n.rstd, w), dy, None, n.h, n.rstd, w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H", [(20000, 1000), (5000, 4089), (5000, 7681)])
def test_norm_of_many_rows(gpu, dtype, T, H):
    x, r, w = norm._inputs(gpu, T, H, dtype)
    norm._check_forward(taot.add_rms_norm(x, w, 1e-6, residual=r, group=0), x, r, w, 1e-6, 0)
    dy, dh = _gradients(gpu, T, H, dtype)
    s = (x.float().square().mean(1) + 1e-6).rsqrt()
    norm._check_backward(taot.add_rms_norm_backward(dy, x, s, w, dh=dh), dy, dh, x, s, w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,groups,k", [(512, 8, 8), (300, 4, 5), (512, 2, 1), (400, 16, 8), (129, 1, 3)])
def test_biased_choices_of_up_to_512_experts(gpu, dtype, E, groups, k):
    x = route._logits(70, E, dtype, seed=E, step=1 / 64)
    for flags in (route.SIG | route.REN, route.SIG | route.REN | route.TWO):
        route_groups._check(gpu, x, k, groups, max(1, groups // 2), flags, bias=route._bias(E, E))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E", [513, 777, 1024])
def test_gradient_of_up_to_1024_experts(gpu, dtype, E):
    route.test_backward(gpu, dtype, 9, E, 8, 0)
    route.test_backward(gpu, dtype, 9, E, 8, route.SIG | route.REN)


# (R, E, K, N): tables too long for a wave's ids, of up to 6, 8, 9 and 12 bits an expert; short rows of 12 bits
@pytest.mark.parametrize("R,E,K,N", [(1024, 40, 4, 300), (1024, 200, 4, 700), (1024, 400, 4, 900), (1024, 4000, 4, 9000),
                                     (16, 600, 2, 100), (16, 1500, 2, 1), (8, 1000, 3, 3000)])
@pytest.mark.parametrize("wild", [False, True])
def test_map_of_many_slots_and_experts(gpu, R, E, K, N, wild):
    print(f"[map] R = {R}, E = {E}, K = {K}, N = {N}", flush=True)
    ids, home, slot, X = dispatch._instance(1, R, 2, E, K, N, seed=E, bad=0.05 if wild else 0.0, wild=wild)
    dispatch._check_map(gpu, ids, home, slot, X, K, rank0=R - 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,k,H", [(5000, 8, 1000), (2100, 4, 4100)])
def test_gradient_of_the_way_back_past_the_caches(gpu, dtype, tokens, k, H):
    pos = torch.from_numpy(dispatch._positions(1, tokens * k, seed=k, dropped=0.1)).to(gpu)
    g = torch.Generator(gpu).manual_seed(H)
    y, d, w = (torch.randn(s, generator=g, device=gpu) for s in ((1, tokens * k, H), (1, tokens, H), (1, tokens * k)))
    y, d = y.to(dtype), d.to(dtype)
    c = taot.combine_rows_backward(d, y, pos, w)
    there = (pos[0] >= 0).nonzero().flatten()
    at = pos[0][there].long()
    D, Y, W = d[0][there // k].double(), y[0][at].double(), w[0][there].double()
    dots, size = (D * Y).sum(1), (D * Y).abs().sum(1)
    assert ((c.dweights[0][there].double() - dots).abs() <= (H / 64 + 10) * 2.0 ** -24 * size).all()
    want = W[:, None] * D
    lim = (dispatch.U[dtype] + 2.0 ** -24) * want.abs() + dispatch.LOW[dtype]
    assert ((c.dy[0][at].double() - want).abs() <= lim).all()
    gone = (pos[0] < 0).nonzero().flatten()
    assert len(gone) and not c.dy[0][~pos[0][gone].long()].any() and not c.dweights[0][gone].any()


# 256 MiB of output and more: past the caches, with one, two and four chunks of columns a lane
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H", [(140000, 1000), (16400, 8192), (9000, 16000), (4500, 30011)])
def test_norm_past_the_caches(gpu, dtype, T, H):
    print(f"[norm] {dtype} {T} x {H}", flush=True)
    T = T // (2 if dtype == torch.float32 else 1)
    x, r, w = norm._inputs(gpu, T, H, dtype)
    n = taot.add_rms_norm(x, w, 1e-6, residual=r, group=256)
    h, s, y = norm._reference(x, r, w, 1e-6)
    del h
    assert ((n.rstd.double() - s).abs() <= norm.FP * s).all()
    slack = 2.0 ** -23 * (x.double().abs() + r.double().abs()) * s[:, None] * w.double().abs()
    assert ((n.y.double() - y).abs() <= (norm.U[dtype] + norm.FP) * y.abs() + norm.LOW[dtype] + slack).all()
    some = slice(T - 700, T)  # the last rows of all outputs, and that a call on them alone gives the same
    part = taot.add_rms_norm(x[some], w, 1e-6, residual=r[some], group=256)
    norm._check_forward(part, x[some], r[some], w, 1e-6, 256)
    for name in ("h", "y", "q", "scale", "rstd"):
        assert torch.equal(getattr(n, name)[some].view(torch.uint8), getattr(part, name).view(torch.uint8))
    del y, slack, part
    dy, dh = (torch.randn(T, H, generator=torch.Generator(gpu).manual_seed(i), device=gpu).to(dtype) for i in (1, 2))
    d = taot.add_rms_norm_backward(dy, n.h, n.rstd, w, dh=dh)
    part = taot.add_rms_norm_backward(dy[some], n.h[some], n.rstd[some], w, dh=dh[some])
    norm._check_backward(part, dy[some], dh[some], n.h[some], n.rstd[some], w)
    assert torch.equal(d.dx[some], part.dx)
    want = (dy.double() * n.h.double() * n.rstd.double()[:, None])
    size = want.abs().sum(0)
    assert ((d.dweight.double() - want.sum(0)).abs() <= (T / 512 + 52) * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,k,H", [(17000, 8, 1000), (8300, 4, 4100)])
def test_there_and_back_past_the_caches(gpu, dtype, tokens, k, H):
    test_gradient_of_the_way_back_past_the_caches(gpu, dtype, tokens, k, H)
    pos = torch.from_numpy(dispatch._positions(1, tokens * k, seed=H, dropped=0.1)).to(gpu)
    x = torch.randn(1, tokens, H, generator=torch.Generator(gpu).manual_seed(k), device=gpu).to(dtype)
    out = taot.dispatch_rows(x, pos)
    there = (pos[0] >= 0).nonzero().flatten()
    assert torch.equal(out[0][pos[0][there].long()], x[0][there // k])
    assert not out[0][~pos[0][pos[0] < 0].long()].any()
