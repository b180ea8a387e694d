"""Calls with more work than one launch takes: the same as calls on parts of it."""
import torch
import pytest

import paper_2608_03676_amd as taot

pytestmark = pytest.mark.gpu


def _same(a, b):
    assert torch.equal(a.view(torch.uint8) if a.dtype == torch.float8_e4m3fn else a,
                       b.view(torch.uint8) if b.dtype == torch.float8_e4m3fn else b)


def test_norm(gpu):
    T, H, cut = (1 << 23) + 5, 8, 5_000_001
    x = torch.randn(T, H, device=gpu, generator=torch.Generator(gpu).manual_seed(1)).bfloat16()
    w = torch.rand(H, device=gpu)
    whole = taot.add_rms_norm(x, w, 1e-6, residual=x, group=0)
    for rows in (slice(0, cut), slice(cut, T)):
        part = taot.add_rms_norm(x[rows], w, 1e-6, residual=x[rows], group=0)
        for name in ("h", "y", "q", "scale", "rstd"):
            _same(getattr(whole, name)[rows], getattr(part, name))


def test_route(gpu):
    T, E, cut = (1 << 22) + 7, 8, 3_000_001
    x = torch.randn(T, E, device=gpu, generator=torch.Generator(gpu).manual_seed(2)).bfloat16()
    whole = taot.route(x, 2)
    for rows in (slice(0, cut), slice(cut, T)):
        part = taot.route(x[rows], 2)
        _same(whole.ids[rows], part.ids)
        _same(whole.weights[rows], part.weights)


def test_rows_and_the_way_back(gpu):
    tokens, H = (1 << 23) + 3, 8
    g = torch.Generator(gpu).manual_seed(3)
    x = torch.randn(tokens, H, device=gpu, generator=g).half()
    to = torch.randperm(tokens, device=gpu, generator=g)
    pos, w = to.int().view(1, tokens), torch.rand(1, tokens, device=gpu, generator=g)
    out = taot.dispatch_rows(x.view(1, tokens, H), pos)
    out = out[0] if isinstance(out, tuple) else out
    _same(out.view(tokens, H)[to], x)
    back = taot.combine_rows(out, pos)
    _same(back.view(tokens, H), x)
    grad = taot.combine_rows_backward(x.view(1, tokens, H), out, pos, w)
    _same(grad.dy.view(tokens, H)[to], (x.float() * w.view(-1, 1)).half())


def test_map(gpu):
    B, E, N, cut = 4101, 32768, 5, 2000
    g = torch.Generator(gpu).manual_seed(4)
    ids = torch.randint(E, (B, 1, N), device=gpu, generator=g, dtype=torch.int32)
    home = torch.zeros(E, dtype=torch.int32, device=gpu)
    slot = torch.randint(E, (B, 2), device=gpu, generator=g, dtype=torch.int32)
    slot[:, 0] = ids[:, 0, 0]
    X = torch.ones(B, 1, 2, dtype=torch.int32, device=gpu)
    whole = taot.dispatch_map(ids, home, slot, X, 2)
    assert not whole.status.any()
    for some in (slice(0, cut), slice(cut, B)):
        part = taot.dispatch_map(ids[some], home, slot[some], X[some], 2)
        for name in ("pos", "offsets", "sends", "status"):
            _same(getattr(whole, name)[some], getattr(part, name))
