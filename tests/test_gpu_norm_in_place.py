"""add_rms_norm and the gradients with outputs in their inputs' memory: the same
bits as with memory of their own."""
import pytest
import torch

import paper_2608_03676_amd as taot

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
# one, two and four chunks of eight columns a lane, one wave a row and several; rows that end inside a chunk
SHAPES = [(9, 100), (5, 512), (7, 2049), (6, 4096), (3, 5003), (3, 16384), (2, 20001), (2, 32768), (4200, 4096)]


def _random(gpu, *shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(gpu).manual_seed(seed), device=gpu).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H", SHAPES)
def test_norm(gpu, dtype, T, H):
    print(f"[norm in place] {dtype} {T} x {H}", flush=True)
    x, r, w = (_random(gpu, *s, dtype=dtype, seed=H + i) for i, s in enumerate([(T, H), (T, H), (H,)]))
    for group in (None, 0, 64):
        want = taot.add_rms_norm(x, w, 1e-6, residual=r, group=group)
        plain = taot.add_rms_norm(x, w, 1e-6, group=group)
        for h_at, y_at in (("r", None), ("x", None), (None, "x"), (None, "r"), ("x", "r"), ("r", "x")):
            m = dict(x=x.clone(), r=r.clone())
            n = taot.add_rms_norm(m["x"], w, 1e-6, residual=m["r"], group=group,
                                  out=taot.Norm(h=m.get(h_at), y=m.get(y_at)))
            assert (h_at is None or n.h is m[h_at]) and (y_at is None or n.y is m[y_at])
            for name in ("h", "y", "rstd") + (("q", "scale") if group is not None else ()):
                a, b = getattr(n, name), getattr(want, name)
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (group, h_at, y_at, name)
        m = x.clone()
        n = taot.add_rms_norm(m, w, 1e-6, group=group, out=taot.Norm(y=m))
        assert n.y is m and torch.equal(m, plain.y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H", SHAPES + [(1500, 512), (700, 9000)])
def test_gradient(gpu, dtype, T, H):
    """dx in the memory of what it is made from; rows enough that workers take several."""
    print(f"[norm's gradient in place] {dtype} {T} x {H}", flush=True)
    h, dy, dh, w = (_random(gpu, *s, dtype=dtype, seed=H + i) for i, s in enumerate([(T, H)] * 3 + [(H,)]))
    s = torch.rand(T, device=gpu, generator=torch.Generator(gpu).manual_seed(T)) + 0.5
    for d in (dh, None):
        want = taot.add_rms_norm_backward(dy, h, s, w, dh=d)
        for at in ("h", "dy") + (("dh",) if d is not None else ()):
            m = dict(h=h.clone(), dy=dy.clone(), dh=None if d is None else d.clone())
            got = taot.add_rms_norm_backward(m["dy"], m["h"], s, w, dh=m["dh"], out=taot.NormGrad(dx=m[at]))
            assert got.dx is m[at] and torch.equal(got.dx, want.dx) and torch.equal(got.dweight, want.dweight), at


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E", [(9, 8), (5, 60), (20000, 384), (70, 777), (33, 4096), (9, 4104), (3, 9001)])
@pytest.mark.parametrize("flags", [0, taot.ROUTE_RENORM, taot.ROUTE_SIGMOID, taot.ROUTE_SIGMOID | taot.ROUTE_RENORM])
def test_gradient_of_routing(gpu, dtype, T, E, flags):
    x = _random(gpu, T, E, dtype=dtype, seed=E)
    r = taot.route(x, 8, flags=flags)
    dw = _random(gpu, T, 8, dtype=torch.float32, seed=T)
    want = taot.route_backward(dw, x, r.ids, flags=flags)
    m = x.clone()
    assert taot.route_backward(dw, m, r.ids, flags=flags, out=m) is m and torch.equal(m, want)
