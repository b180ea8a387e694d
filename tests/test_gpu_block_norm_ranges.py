"""block_norm_backward for rows far from 1 in size, whose intermediate products leave 32 bits if their factors meet in
another order than the formula's results need: b = 1 / rms(h) is up to 1e18 here, its cube is no float.

Tolerances are those of the gradient's test, of one row's sums: 150 * 2^-24 relative to the magnitudes a result is made
of, which the two norms' rounded products h b and x a (one rounding each) do not change.  Results below the smallest
normal float are not asked for: the smallest here, a gradient divided by both sizes, is 1e-33."""
import pytest
import torch

import paper_2608_03676_amd as taot
from test_gpu_block_norm import _check_backward

pytestmark = pytest.mark.gpu

# sizes of a row's h and x; 8192 squares of 3e16 are summed without leaving 32 bits
SIZES = [(1, 1), (1e-12, 1), (1e-14, 1), (1e-15, 2), (1e-18, 1), (1e14, 1), (1e16, 3), (3e16, 1), (1, 1e-18), (1, 1e-14), (2, 1e15),
         (1, 3e16), (1e-16, 1e-18), (3e16, 1e16), (1e-14, 1e14), (1e15, 1e-15)]


def _gradient(gpu, H, dtype, sizes, eps, gates, post, dh):
    g = torch.Generator().manual_seed(H)

    def new(*shape, scale=1.0):
        return (scale * torch.randn(shape, generator=g)).to(dtype).to(gpu)

    T = len(sizes)
    of_h, of_x = (torch.tensor([s[i] for s in sizes], dtype=torch.float64)[:, None] for i in (0, 1))
    c = dict(x=(of_x * torch.randn((T, H), generator=g)).to(dtype).to(gpu), residual=None, dy=new(T, H),
             dh=new(T, H) if dh else None, weight=1 + new(H, scale=0.3), post=1 + new(H, scale=0.3) if post else None,
             gate=new(gates, H, scale=0.5) if gates else None)
    h = (of_h * torch.randn((T, H), generator=g)).to(dtype).to(gpu)
    o = taot.BlockNorm(h=h, rstd_h=(h.double().square().mean(1) + eps).rsqrt().float())
    if post:
        o.rstd_x = (c["x"].double().square().mean(1) + eps).rsqrt().float()
    got = taot.block_norm_backward(c["dy"], c["x"], h, o.rstd_h, c["weight"], rstd_x=o.rstd_x, post=c["post"],
                                   gate=c["gate"], dh=c["dh"])
    return got, c, o


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [5, 40, 515, 4096, 8191, 8192, 8200, 16384])  # up to 8192 columns in registers, but for 5
def test_rows_of_all_sizes(gpu, dtype, H):
    for gates, post, dh in ((1, True, False), (16, True, True), (4, True, False), (0, False, True), (0, True, False)):
        print(f"[block norm ranges] {dtype} {H} columns, {gates} gates, post {post}, dh {dh}", flush=True)
        got, c, o = _gradient(gpu, H, dtype, SIZES, 0.0, gates, post, dh)
        for v in (got.dx, got.dresidual, got.dweight):
            assert torch.isfinite(v).all()
        _check_backward(got, c, o, 1.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [5, 40, 515, 8192, 8200])
def test_rows_whose_squares_are_hardly_floats(gpu, dtype, H):
    """b = 1e21, whose square is no float."""
    for gates, post in ((1, True), (4, True), (0, False)):
        got, c, o = _gradient(gpu, H, dtype, [(1e-20, 1), (1e-21, 1), (1, 1e-21), (1, 1e-20)], 0.0, gates, post, False)
        _check_backward(got, c, o, 1.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [5, 40, 4096, 8192, 8200])
def test_rows_of_zeros_with_a_small_eps(gpu, dtype, H):
    """b = 1e15, h = 0: dresidual is b dy w + dh, nothing of it is lost in a product of b's cube and 0."""
    for gates, post in ((1, True), (4, True), (0, False)):
        print(f"[block norm ranges] zeros, {dtype} {H} columns, {gates} gates, post {post}", flush=True)
        got, c, o = _gradient(gpu, H, dtype, [(0, 1), (1, 0), (1, 1), (0, 0)], 1e-30, gates, post, True)
        for n in ("dx", "dresidual", "dweight", "dpost", "dgate"):
            v = getattr(got, n)
            assert v is None or torch.isfinite(v).all(), n
        _check_backward(got, c, o, 1.0)
