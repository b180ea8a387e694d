"""Block norm, its gradient, 8-bit rows and the balance gradient where their outputs go past the caches (256 MiB and
more) and where their work is more than one launch takes."""
import pytest
import torch

import paper_2608_03676_amd as taot
from test_gpu_balance import SIGMOID, _grad_check
from test_gpu_block_norm import _check_backward, _check_forward

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
FAR = 256 << 20


def _case(gpu, T, H, dtype, gates, post=True):
    g = torch.Generator(gpu).manual_seed(T + H)

    def new(*shape, scale=1.0, shift=0.0):
        return (shift + scale * torch.randn(shape, generator=g, device=gpu)).to(dtype)

    return dict(x=new(T, H), residual=new(T, H, scale=2.0), dy=new(T, H), dh=new(T, H), weight=new(H, scale=0.3, shift=1.0),
                post=new(H, scale=0.3, shift=0.7) if post else None, gate=new(gates, H, scale=0.5) if gates else None)


def _forward(c, **kw):
    return taot.block_norm(c["x"], c["residual"], c["weight"], 1e-6, post=c["post"], gate=c["gate"], **kw)


@pytest.mark.parametrize("T,H,dtype,gates,post", [
    (16400, 4096, BF16, 4, True), (16400, 4097, F16, 1, True), (33000, 2045, BF16, 0, False), (8200, 4096, F32, 8200, True),
    (4200, 8191, F32, 2, False), (2100, 32768, BF16, 1, True), (135000, 500, F16, 3, True)])
def test_block_norm_past_the_caches(gpu, T, H, dtype, gates, post):
    print(f"[block norm, far] {dtype} {T} x {H}", flush=True)
    c = _case(gpu, T, H, dtype, gates, post)
    o = _forward(c)
    assert 2 * o.y.numel() * o.y.element_size() >= FAR
    _check_forward(o, c, 1e-6, 1.0)
    for over in ("residual", "x"):
        was = c[over].clone()
        s = _forward(c, out=taot.BlockNorm(h=c[over]))
        assert torch.equal(s.h, o.h) and torch.equal(s.y, o.y) and torch.equal(s.rstd_h, o.rstd_h)
        c[over].copy_(was)


def test_block_norm_in_several_launches(gpu):
    """2^23 rows of one wave each are a launch; the gates of the rows behind them are counted from the first row on."""
    c = _case(gpu, 4 * (1 << 21) + 20, 8, BF16, 4)
    o = _forward(c)
    _check_forward(o, c, 1e-6, 1.0)
    T = 2 * (1 << 21) + 10  # the last two gates' rows by themselves
    part = dict(c, x=c["x"][T:], residual=c["residual"][T:], gate=c["gate"][2:].contiguous())
    p = _forward(part)
    for n in ("h", "y", "rstd_x", "rstd_h"):
        assert torch.equal(getattr(o, n)[T:], getattr(p, n)), n


@pytest.mark.parametrize("T,H,dtype,gates,post", [
    (16400, 4096, BF16, 4, True), (16400, 4097, F16, 1, True), (16400, 4096, F16, 8200, True), (33000, 2045, BF16, 33000, False),
    (8200, 4104, F32, 2, True), (8200, 8200, BF16, 4, True), (8200, 8200, BF16, 1640, True), (1050, 32767, F32, 0, True)])
def test_block_norm_gradient_past_the_caches(gpu, T, H, dtype, gates, post):
    print(f"[block norm backward, far] {dtype} {T} x {H}, {gates} gates", flush=True)
    c = _case(gpu, T, H, dtype, gates, post)
    o = _forward(c)

    def back(**kw):
        return taot.block_norm_backward(c["dy"], c["x"], o.h, o.rstd_h, c["weight"], rstd_x=o.rstd_x, post=c["post"],
                                        gate=c["gate"], dh=c["dh"], **kw)

    got = back()
    assert 2 * got.dx.numel() * got.dx.element_size() >= FAR
    _check_backward(got, c, o, 1.0)
    again = back(out=taot.BlockNormGrad(dx=c["dy"], dresidual=c["dh"]))  # over the inputs
    for n in ("dx", "dresidual", "dweight", "dpost", "dgate"):
        a, b = getattr(got, n), getattr(again, n)
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b)), n


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,H", [(65600, 4096), (65600, 4099), (400000, 700), (8400, 32768)])
def test_rows_past_the_caches(gpu, dtype, T, H):
    g = torch.Generator(gpu).manual_seed(T)
    for gated in (False, True):
        print(f"[rows, far] {dtype} {T} x {H} {gated}", flush=True)
        x = torch.randn(T, H * (1 + gated), generator=g, device=gpu, dtype=F32).to(dtype)
        q, scale = taot.quantize_rows(x, gated=gated)
        assert q.numel() >= FAR
        cut = T // 3
        for rows in (slice(0, cut), slice(cut, 2 * cut), slice(2 * cut, T)):  # through the caches
            p = taot.quantize_rows(x[rows], gated=gated)
            assert torch.equal(q[rows], p.q) and torch.equal(scale[rows], p.scale)


def test_rows_in_several_launches(gpu):
    T, cut = (1 << 23) + 5, 5_000_001
    x = torch.randn(T, 16, device=gpu, generator=torch.Generator(gpu).manual_seed(5)).half()
    for gated in (False, True):
        q, scale = taot.quantize_rows(x, gated=gated)
        for rows in (slice(0, cut), slice(cut, T)):
            p = taot.quantize_rows(x[rows], gated=gated)
            assert torch.equal(q[rows], p.q) and torch.equal(scale[rows], p.scale)


@pytest.mark.parametrize("flags", [0, SIGMOID])
@pytest.mark.parametrize("rows,tokens,experts", [(2500, 5, 16), (4100, 3, 40), (2050, 2, 600), (2049, 2, 3000)])
def test_balance_gradient_in_several_launches(gpu, rows, tokens, experts, flags):
    g = torch.Generator(gpu).manual_seed(rows)
    x = torch.randn(rows, tokens, experts, device=gpu, generator=g).bfloat16()
    ids = torch.randint(experts, (rows, tokens, 2), device=gpu, generator=g, dtype=torch.int32)
    mask = torch.rand(rows, tokens, device=gpu, generator=g) < 0.8
    add = (torch.randn(x.shape, device=gpu, generator=g) / experts).bfloat16()
    dloss, dz = (torch.randn(rows, device=gpu, generator=g) for _ in range(2))
    dz = None if flags else dz
    b = taot.balance_loss(x, ids, mask=mask, flags=flags)
    got = taot.balance_loss_backward(dloss, x, b.counts, b.tokens, mask=mask, dz=dz, add=add, flags=flags)
    _grad_check(got, x, ids, b.counts, b.tokens, mask, dloss, dz, add, flags != 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gates_of_rows_far_below_zero(gpu, dtype):
    """silu of a value below -88 is less than 1e-36, whatever the value."""
    low = [torch.finfo(dtype).min, -1e38, -1e30, -1e5, -200.0, -100.0, -89.0, -88.0, -87.5, -80.0]
    x = torch.zeros(3, 2, 64, device=gpu)
    x[0, 0, :10], x[0, 0, 20] = torch.tensor(low, device=gpu), 127.0
    x[0, 1] = 1.0
    x[1, 0, 3], x[1, 1, 3] = float("-inf"), 1.0  # the product is no number
    x[2, 0, 5], x[2, 1, 5] = 5.0, float("inf")
    q, scale = taot.quantize_rows(x.to(dtype).view(3, 128), gated=True)
    want = torch.zeros(64, dtype=torch.int8, device=gpu)
    want[20] = 127
    assert torch.equal(q[0], want) and abs(float(scale[0]) - 1) < 16 * 2.0 ** -24
    assert torch.isnan(scale[1:]).all() and not q[1:].any()
