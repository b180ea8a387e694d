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
