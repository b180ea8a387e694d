"""add_rms_norm and its gradient against the formulas in 64 bits.

Tolerances.  u: half a unit in the last place of the output's type, relative
(bf16 2^-8, f16 2^-11, f32 2^-24; f16 also 2^-25 absolute, below its normal
range).  A row's sum of squares passes through at most 32 + 6 + 16 additions a
value, all of one sign, so the norm is within 60 * 2^-24 < 4e-6 of its value
after the square root, the division and the products.  8 bits: half a unit of
e4m3 is 2^-4 of a normal value and 2^-10 of the scale below that."""
import numpy as np
import pytest
import torch

import paper_2608_03676_amd as taot

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LOW = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
FP = 4e-6
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _at_odd_address(t):
    """The same values in memory that begins one element behind a 16-byte boundary."""
    room = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    room[1:] = t.reshape(-1)
    return room[1:].view(t.shape)


def _inputs(gpu, T, H, dtype, seed=0, residual=True, w_dtype=None):
    g = torch.Generator().manual_seed(seed + 7919 * T + H)
    x = torch.randn(T, H, generator=g).to(dtype)
    r = (3 * torch.randn(T, H, generator=g)).to(dtype) if residual else None
    w = (1 + 0.3 * torch.randn(H, generator=g)).to(w_dtype or dtype)
    return [None if t is None else t.to(gpu) for t in (x, r, w)]


def _reference(x, r, w, eps):
    h = x.double() if r is None else x.double() + r.double()
    s = (h.square().mean(-1) + eps).rsqrt()
    return h, s, h * s[..., None] * w.double()


def _check_forward(n, x, r, w, eps, group):
    h, s, y = _reference(x, r, w, eps)
    dt = x.dtype
    assert ((n.rstd.double() - s).abs() <= FP * s).all()
    if r is None:
        assert n.h is x
    else:
        assert ((n.h.double() - h).abs() <= (U[dt] + 2.0 ** -23) * h.abs() + LOW[dt] + 2.0 ** -23 * r.double().abs()).all()
    # the sum itself is rounded to 32 bits: relative to the larger addend
    slack = 2.0 ** -23 * (x.double().abs() + (0 if r is None else r.double().abs())) * s[..., None] * w.double().abs()
    assert ((n.y.double() - y).abs() <= (U[dt] + FP) * y.abs() + LOW[dt] + slack).all()
    if group is None:
        return
    T, H = x.shape
    G = group or H
    q, scale = n.q.double(), n.scale.double()
    assert scale.shape == (T, -(-H // G))
    for i, lo in enumerate(range(0, H, G)):
        part = y[:, lo:lo + G]
        a = part.abs().amax(1).clamp(min=1e-30)
        top = slack[:, lo:lo + G].amax(1)
        assert ((scale[:, i] * 448 - a).abs() <= FP * a + top).all(), i
        got = q[:, lo:lo + G] * scale[:, i:i + 1]
        lim = torch.maximum(part.abs() * 2.0 ** -4, scale[:, i:i + 1] * 2.0 ** -10) * (1 + 1e-4) + slack[:, lo:lo + G]
        assert ((got - part).abs() <= lim + FP * part.abs()).all(), i


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H", [(1, 1), (3, 7), (5, 8), (2, 9), (4, 100), (3, 512), (3, 513), (4, 2048), (2, 2049),
                                 (3, 5003), (2, 8192), (2, 16400), (2, 32768)])
def test_forward_widths(gpu, dtype, T, H):
    x, r, w = _inputs(gpu, T, H, dtype)
    print(f"[norm] {dtype} {T} x {H}", flush=True)
    for group in (None, 0, 128):
        n = taot.add_rms_norm(x, w, 1e-6, residual=r, group=group)
        _check_forward(n, x, r, w, 1e-6, group)
    n = taot.add_rms_norm(x, w, 1e-6, group=8)
    _check_forward(n, x, None, w, 1e-6, 8)


@pytest.mark.parametrize("T,H", [(4096, 1), (4100, 64), (4097, 520), (4099, 1031), (4098, 4096), (4096, 4104)])
def test_forward_many_rows(gpu, T, H):
    x, r, w = _inputs(gpu, T, H, torch.bfloat16)
    n = taot.add_rms_norm(x, w, 1e-5, residual=r, group=128)
    _check_forward(n, x, r, w, 1e-5, 128)


def test_forward_wide_rows_many(gpu):
    x, r, w = _inputs(gpu, 4096, 16392, torch.float16)
    n = taot.add_rms_norm(x, w, 1e-5, residual=r, group=512)
    _check_forward(n, x, r, w, 1e-5, 512)


@pytest.mark.parametrize("group", [8, 16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("H", [520, 1500])
def test_groups(gpu, group, H):
    x, r, w = _inputs(gpu, 5, H, torch.bfloat16, w_dtype=torch.float32)
    n = taot.add_rms_norm(x, w, 1e-6, residual=r, group=group)
    _check_forward(n, x, r, w, 1e-6, group)


@pytest.mark.parametrize("dtype", TYPES)
def test_odd_addresses(gpu, dtype):
    x, r, w = (_at_odd_address(t) for t in _inputs(gpu, 6, 264, dtype))
    assert x.data_ptr() % 16 != 0
    out = taot.Norm(y=_at_odd_address(x), h=_at_odd_address(x))
    n = taot.add_rms_norm(x, w, 1e-6, residual=r, group=32, out=out)
    _check_forward(n, x, r, w, 1e-6, 32)
    dy = _at_odd_address(x * 0.5)
    d = taot.add_rms_norm_backward(dy, n.h, n.rstd, w, dh=r)
    _check_backward(d, dy, r, n.h, n.rstd, w)


def test_leading_dimensions_and_empty(gpu):
    x, r, w = _inputs(gpu, 6, 40, torch.float16)
    n = taot.add_rms_norm(x.view(2, 3, 40), w, 1e-6, residual=r.view(2, 3, 40), group=16)
    assert n.y.shape == (2, 3, 40) and n.scale.shape == (2, 3, 3) and n.rstd.shape == (2, 3)
    m = taot.add_rms_norm(x, w, 1e-6, residual=r, group=16)
    assert torch.equal(n.y.view(6, 40), m.y) and torch.equal(n.scale.view(6, 3), m.scale)
    e = taot.add_rms_norm(x[:0], w, 1e-6, group=0)
    assert e.y.shape == (0, 40) and e.scale.shape == (0, 1)
    d = taot.add_rms_norm_backward(x[:0], x[:0], torch.empty(0, device=gpu), w)
    assert d.dx.shape == (0, 40) and not d.dweight.any()


def test_zeros_and_what_is_not_finite(gpu):
    x = torch.zeros(4, 256, device=gpu, dtype=torch.bfloat16)
    x[1, 3] = float("inf")
    x[2, 200] = float("nan")
    x[3] = 1.0
    w = torch.ones(256, device=gpu, dtype=torch.bfloat16)
    n = taot.add_rms_norm(x, w, 0.0, group=128)
    y = n.y.float().cpu()
    assert torch.isnan(y[0]).all()                  # 0 / 0 without an epsilon
    assert torch.isnan(y[1, 3]) and not y[1, :3].any()  # infinity / infinity; the rest 0
    assert torch.isnan(y[2]).all()
    n = taot.add_rms_norm(x, w, 1e-6, group=128)
    q, s = n.q.float().cpu(), n.scale.cpu()
    assert not n.y[0].any() and not q[0].any() and (s[0] > 0).all() and (s[0] < 1e-30).all()
    assert (q[3] == 448).all() and torch.allclose(s[3] * 448, torch.ones(2), rtol=FP)


def _check_backward(d, dy, dh, h, rstd, w):
    dt = h.dtype
    T, H = h.shape
    D, X, s, W = dy.double(), h.double(), rstd.double()[:, None], w.double()
    g = D * W
    mean = (g * X).mean(1, keepdim=True)
    dx = s * (g - X * s * s * mean)
    terms = s * (g.abs() + X.abs() * s * s * mean.abs())
    if dh is not None:
        dx = dx + dh.double()
        terms = terms + dh.double().abs()
    # the dot product's rounding: up to 60 additions a term
    dot = s * X.abs() * s * s * (g * X).abs().mean(1, keepdim=True) * 64 * 2.0 ** -24
    assert ((d.dx.double() - dx).abs() <= U[dt] * dx.abs() + LOW[dt] + 8 * 2.0 ** -24 * terms + dot).all()
    dw, size = (D * X * s).sum(0), (D * X * s).abs().sum(0)
    adds = T / 512 + 1 + 16 + 32 + 3
    assert ((d.dweight.double() - dw).abs() <= adds * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H", [(1, 1), (3, 7), (5, 8), (7, 100), (3, 513), (600, 64), (520, 2049), (3, 8192),
                                 (2, 16400), (3, 32768), (4097, 40), (4099, 1032), (4096, 4104)])
def test_backward(gpu, dtype, T, H):
    print(f"[norm backward] {dtype} {T} x {H}", flush=True)
    x, r, w = _inputs(gpu, T, H, dtype)
    g = torch.Generator().manual_seed(T + H)
    dy, dh = (torch.randn(T, H, generator=g).to(dtype).to(gpu) for _ in range(2))
    rstd = (x.float().square().mean(1) + 1e-6).rsqrt()
    d = taot.add_rms_norm_backward(dy, x, rstd, w, dh=dh)
    _check_backward(d, dy, dh, x, rstd, w)
    d2 = taot.add_rms_norm_backward(dy, x, rstd, w.float())
    _check_backward(d2, dy, None, x, rstd, w)
    d3 = taot.add_rms_norm_backward(dy, x, rstd, w, dh=dh)
    assert torch.equal(d.dweight, d3.dweight) and torch.equal(d.dx, d3.dx)


def test_backward_against_differences(gpu):
    """The directional derivative of sum(a y + b h) in 64 bits, by central differences (error about 1e-9 here)."""
    T, H, eps = 9, 130, 1e-5
    x, r, w = _inputs(gpu, T, H, torch.float32)
    g = torch.Generator().manual_seed(5)
    a, b, vx, vw = (torch.randn(s, generator=g).to(gpu) for s in ((T, H), (T, H), (T, H), (H,)))
    n = taot.add_rms_norm(x, w, eps, residual=r)
    d = taot.add_rms_norm_backward(a, n.h, n.rstd, w, dh=b)

    def value(step):
        h, s, y = _reference(x.double() + step * vx.double(), r, w.double() + step * vw.double(), eps)
        return (a.double() * y + b.double() * h).sum()

    want = (value(1e-5) - value(-1e-5)) / 2e-5
    got = (d.dx.double() * vx.double()).sum() + (d.dweight.double() * vw.double()).sum()
    size = (d.dx.double() * vx.double()).abs().sum() + (d.dweight.double() * vw.double()).abs().sum()
    assert abs(want - got) <= 1e-5 * size


def test_another_stream(gpu):
    x, r, w = _inputs(gpu, 300, 2048, torch.bfloat16)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    n = taot.add_rms_norm(x, w, 1e-6, residual=r, group=128, stream=s)
    d = taot.add_rms_norm_backward(x, n.h, n.rstd, w, stream=s)
    s.synchronize()
    _check_forward(n, x, r, w, 1e-6, 128)
    _check_backward(d, x, None, n.h, n.rstd, w)


def test_refusals(gpu):
    x, r, w = _inputs(gpu, 4, 64, torch.bfloat16)
    with pytest.raises(TypeError):
        taot.add_rms_norm(x.double(), w, 1e-6)
    with pytest.raises(TypeError):
        taot.add_rms_norm(x, w.half(), 1e-6)
    with pytest.raises(TypeError):
        taot.add_rms_norm(x.cpu(), w, 1e-6)
    with pytest.raises(TypeError):
        taot.add_rms_norm(x, w, 1e-6, residual=r.float())
    with pytest.raises(ValueError):
        taot.add_rms_norm(x.t(), w, 1e-6)
    with pytest.raises(ValueError):
        taot.add_rms_norm(x, w[:-1], 1e-6)
    with pytest.raises(ValueError):
        taot.add_rms_norm(x, w, 1e-6, residual=r[:2])
    with pytest.raises(ValueError):
        taot.add_rms_norm_backward(x, x, torch.ones(3, device=gpu), w)
    for group in (4, 24, 1024, -8):
        with pytest.raises(taot.TaotError):
            taot.add_rms_norm(x, w, 1e-6, group=group)
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(taot.TaotError):
            taot.add_rms_norm(x, w, eps)
    wide = torch.zeros(1, 32769, device=gpu)
    with pytest.raises(taot.TaotError) as e:
        taot.add_rms_norm(wide, wide[0], 1e-6)
    assert e.value.code == 2

def test_a_result_used_again_leaves_an_earlier_input_alone(gpu):
    """A call without a residual gives its x as h; the next one, with a residual, writes its sum elsewhere."""
    x, r, w = _inputs(gpu, 5, 96, torch.bfloat16)
    before = x.clone()
    n = taot.add_rms_norm(x, w, 1e-6)
    n = taot.add_rms_norm(r, w, 1e-6, residual=x, out=n)
    assert torch.equal(x, before)
    _check_forward(n, r, x, w, 1e-6, None)
    h, y = n.h, n.y
    n = taot.add_rms_norm(x, w, 1e-6, residual=r, out=n)
    assert n.h is h and n.y is y
    _check_forward(n, x, r, w, 1e-6, None)


def test_a_result_used_again_keeps_nothing_of_an_earlier_call(gpu):
    """Without an 8-bit output there is none beside the new y; a refused call leaves the result as it was."""
    x, r, w = _inputs(gpu, 5, 96, torch.bfloat16)
    n = taot.add_rms_norm(x, w, 1e-6, residual=r, group=32)
    n = taot.add_rms_norm(r, w, 1e-6, residual=x, out=n)
    assert n.q is None and n.scale is None
    _check_forward(n, r, x, w, 1e-6, None)
    n = taot.add_rms_norm(x, w, 1e-6, residual=r, group=32, out=n)
    _check_forward(n, x, r, w, 1e-6, 32)
    h, y = n.h, n.y
    with pytest.raises(ValueError):  # another number of scales
        taot.add_rms_norm(r, w, 1e-6, group=8, out=n)
    with pytest.raises(taot.TaotError):
        taot.add_rms_norm(r, w, -1.0, out=n)
    assert n.h is h and n.y is y and not n.h_is_x
    _check_forward(n, x, r, w, 1e-6, 32)
