"""Gradients that reach balance_loss from outside its usual range.  One that is not finite has to be seen in what leaves:
the step that it belongs to is not to be taken.  A large one whose results are finite may not leave 32 bits on the way."""
import pytest
import torch

import paper_2608_03676_amd as taot
from test_gpu_balance import E, SIGMOID, TYPES, _case, _grad_check, _scores

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
EXPERTS = [16, 40, 64, 160, 600, 2048, 3000]  # 2, 8 and 16 lanes, a wave and a block for a token


def _formula(x, counts, tokens, dloss, dz):
    p, lse = _scores(x.double(), False)
    n = x.shape[2]
    a = (dloss.double() * n / (counts.sum(1).clamp(min=1) * tokens.clamp(min=1)))[:, None, None] * counts[:, None, :].double()
    return p * (a - (a * p).sum(-1, keepdim=True) + (2 * dz.double() / tokens.clamp(min=1))[:, None, None] * lse[..., None])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("experts", EXPERTS)
def test_dz_that_is_not_finite(gpu, dtype, experts):
    print(f"[balance incoming] {dtype} {experts}", flush=True)
    x, ids, mask = _case(gpu, 5, 21, experts, 2, dtype, True)
    x[:, :, 3] = -INF  # an expert of p = 0: its gradient is 0 times what is not finite
    b = taot.balance_loss(x, ids, mask=mask)
    one = torch.ones(5, device=gpu)
    add = torch.randn(x.shape, device=gpu, generator=torch.Generator(gpu).manual_seed(1)).to(dtype)
    usual = taot.balance_loss_backward(one, x, b.counts, b.tokens, mask=mask, dz=one, add=add)
    assert torch.isfinite(usual).all()
    dz = torch.tensor([1.0, NAN, INF, -INF, 1.0], device=gpu)
    for more in (add, None):
        got = taot.balance_loss_backward(one, x, b.counts, b.tokens, mask=mask, dz=dz, add=more)
        want = _formula(x, b.counts, b.tokens, one, dz)
        for r in (1, 2, 3):
            g, w = got[r][mask[r]].double(), want[r][mask[r]]
            assert not torch.isfinite(w).any() and torch.equal(torch.isnan(g), torch.isnan(w))
            assert torch.equal(torch.nan_to_num(g), torch.nan_to_num(w))  # the infinities' signs
            assert torch.equal(got[r][~mask[r]], torch.zeros_like(got[r][~mask[r]]) if more is None else more[r][~mask[r]])
        if more is not None:
            assert torch.equal(got[[0, 4]], usual[[0, 4]])


@pytest.mark.parametrize("flags", [0, SIGMOID])
@pytest.mark.parametrize("experts", EXPERTS)
def test_dloss_that_is_not_finite(gpu, experts, flags):
    x, ids, mask = _case(gpu, 4, 21, experts, 2, torch.float32, True)
    b = taot.balance_loss(x, ids, mask=mask, flags=flags)
    usual = taot.balance_loss_backward(torch.ones(4, device=gpu), x, b.counts, b.tokens, mask=mask, flags=flags)
    dloss = torch.tensor([1.0, NAN, INF, -INF], device=gpu)
    got = taot.balance_loss_backward(dloss, x, b.counts, b.tokens, mask=mask, flags=flags)
    assert torch.equal(got[0], usual[0])
    for r in (1, 2, 3):
        assert not torch.isfinite(got[r][mask[r]]).any() and not got[r][~mask[r]].any()


def test_a_logit_of_infinity_with_a_finite_dz(gpu):
    """It counts as the largest float, and so does its logarithm: the gradient is finite, that of all others 0."""
    top = torch.finfo(torch.float32).max
    for experts in EXPERTS:
        x, ids, _ = _case(gpu, 2, 20, experts, 2, torch.float32)
        x[0, 9, 4], x[1, 7, 5] = INF, INF
        b = taot.balance_loss(x, ids)
        dz = torch.tensor([3.0, -500.0], device=gpu)
        got = taot.balance_loss_backward(torch.ones(2, device=gpu), x, b.counts, b.tokens, dz=dz)
        assert torch.isfinite(got).all()
        assert abs(float(got[0, 9, 4]) / (0.3 * top) - 1) < 16 * E and got[1, 7, 5] == -top  # 50 times the largest float
        for r, t in ((0, 9), (1, 7)):
            assert (got[r, t] != 0).sum() == 1


@pytest.mark.parametrize("flags", [0, SIGMOID])
@pytest.mark.parametrize("experts,size", [(16, 3e37), (160, 5e36), (600, 3e36), (4096, 3e36)])
def test_large_incoming_gradients(gpu, experts, size, flags):
    """dloss E is no float, dloss E / n is; 2 dz is none, 2 dz / n is."""
    x, ids, _ = _case(gpu, 3, 64, experts, 8, torch.float32)
    x *= 0.3
    b = taot.balance_loss(x, ids, flags=flags)
    dloss = torch.tensor([size, -size, 1.0], device=gpu)
    dz = None if flags else torch.tensor([2e38, -2e38, 1.0], device=gpu)
    got = taot.balance_loss_backward(dloss, x, b.counts, b.tokens, dz=dz, flags=flags)
    assert torch.isfinite(got).all()
    _grad_check(got, x, ids, b.counts.double(), b.tokens.double(), None, dloss, dz, None, flags != 0)
