"""route by groups of experts, against the definition in 64 bits: what a group
counts as, and groups of which little or nothing can be chosen.

Without a bias the keys of single experts are their logits; a group counts as its
largest key, or by two as the sum of its two best scores (and biases).  Tokens on
which a sum comes within 2e-6 of another, relative (a score in 32 bits is within 3
units of 2^-24 for its exponential, 2 for its sum and division, and 2^-24 times the
logits' spread, below 16 here), are left out, and are few; the sums of equal logits
are equal.  Weights are allowed what tests of single experts allow them: 1.5e-5, and
3e-6 where only the chosen enter."""
import numpy as np
import pytest
import torch

import paper_2608_03676_amd as taot

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
SIG, REN, TWO = taot.ROUTE_SIGMOID, taot.ROUTE_RENORM, taot.ROUTE_GROUP_TWO
NEAR = 2e-6


def oracle(x, k, bias, groups, top_groups, flags):
    """ids [T][k], weights [T][k], sure [T]."""
    T, E = x.shape
    ids, weights, sure = np.full((T, k), -1), np.zeros((T, k)), np.ones(T, bool)
    for t in range(T):
        z = np.where(x[t] > -np.inf, np.minimum(x[t], 3.402823466e38), -np.inf)
        ok = z > -np.inf
        if not ok.any():
            continue
        with np.errstate(over="ignore"):
            s = np.where(ok, 1 / (1 + np.exp(-z)) if flags & SIG else np.exp(z - z[ok].max()), 0)
        if not flags & SIG:
            s = s / s.sum()
        score = s if bias is None else s + bias
        key = z if bias is None else score
        ok &= key > -np.inf
        key = np.where(ok, key, -np.inf)
        by = key.reshape(groups, -1)
        order = np.argsort(-by, axis=1, kind="stable")[:, :2]
        value = by.max(1)
        if flags & TWO:
            there = np.take_along_axis(ok.reshape(groups, -1), order, 1)
            two = np.where(there, np.take_along_axis(score.reshape(groups, -1), order, 1), 0)
            value = np.where(there[:, 0], two.sum(1), -np.inf)
        rank = np.lexsort((np.arange(groups), -value))
        last, rest = value[rank[top_groups - 1]], value[rank[top_groups:]]
        if len(rest) and rest[0] > -np.inf and last != rest[0]:
            sure[t] = last - rest[0] > NEAR * (abs(last) if flags & TWO else 1)
        key.reshape(groups, -1)[rank[top_groups:]] = -np.inf
        best = np.lexsort((np.arange(E), -key))[:k + 1]
        gaps = -np.diff(key[best][key[best] > -np.inf])
        if (gaps > 0).any():
            sure[t] &= bias is None or gaps[gaps > 0].min() > NEAR
        pick = [e for e in best[:k] if key[e] > -np.inf]
        w = s[pick]
        if flags & REN and pick:
            if flags & SIG:
                w = w / (w.sum() + 1e-20)
            else:
                w = np.exp(z[pick] - z[pick].max())
                w = w / w.sum()
        ids[t, :len(pick)], weights[t, :len(pick)] = pick, w
    return ids, weights, sure


def _logits(T, E, dtype, seed, step):
    x = torch.randn(T, E, generator=torch.Generator().manual_seed(seed)) * 1.5
    return ((x / step).round() * step).to(dtype)  # exact in every type


def _check(gpu, x, k, groups, top_groups, flags, bias=None):
    r = taot.route(x.to(gpu), k, bias=None if bias is None else bias.to(gpu), groups=groups, top_groups=top_groups,
                   flags=flags)
    ids, weights, sure = oracle(x.double().numpy(), k, None if bias is None else bias.double().numpy(), groups,
                                top_groups, flags)
    assert sure.mean() > 0.8, sure.mean()
    got_ids, got_w = r.ids.cpu().numpy(), r.weights.double().cpu().numpy()
    wrong = sure & (got_ids != ids).any(1)
    assert not wrong.any(), (np.flatnonzero(wrong), got_ids[wrong][:3], ids[wrong][:3])
    tol = 3e-6 if flags & (SIG | REN) else 1.5e-5
    assert (np.abs(got_w - weights)[sure] <= tol * np.abs(weights[sure]) + 1e-30).all()
    return r, sure


# (experts, groups): up to 512 experts a few lanes a token, up to 4096 a wave, above a block
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,groups", [(16, 4), (64, 8), (256, 8), (384, 16), (512, 4), (520, 4), (1024, 16), (6000, 4)])
@pytest.mark.parametrize("flags", [0, TWO, REN | TWO, SIG | TWO])
def test_a_group_of_lowest_values_comes_before_a_masked_one(gpu, dtype, E, groups, flags):
    """The type's lowest value can be chosen, -infinity cannot, though two of the one may add up to the other."""
    low, gs = torch.finfo(dtype).min, E // groups
    x = torch.full((4, E), low, dtype=dtype)
    x[0, :gs] = -np.inf               # a masked group before those of lowest values
    x[1, : E - gs] = -np.inf          # all masked but the last
    x[2, gs:2 * gs] = -np.inf
    x[2, gs - 1] = 0.0                # one value above the lowest, and a masked group behind it
    x[3, :gs] = -np.inf
    x[3, gs:] = float("nan")
    x[3, -1] = low                    # one expert in all
    for k in (1, min(3, gs)):
        r, _ = _check(gpu, x, k, groups, 1, flags)
        assert (r.ids[:3] >= 0).all() and (r.ids[3, 0] == E - 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,groups,k", [(16, 1, 8), (16, 4, 4), (64, 8, 6), (256, 8, 8), (256, 1, 8), (384, 16, 12),
                                        (512, 4, 8), (512, 1, 16), (520, 8, 8), (4096, 16, 8)])
@pytest.mark.parametrize("flags", [0, REN, SIG, SIG | REN])
def test_masked_rows_of_every_type(gpu, dtype, E, groups, k, flags):
    x = _logits(9, E, dtype, seed=E + k, step=1 / 64)
    low = torch.finfo(dtype).min
    x[0] = -np.inf                    # a row that is masked altogether
    x[1, 3:] = -np.inf                # fewer experts than choices
    x[2] = low
    x[2, 5] = 0.0
    x[3, ::2] = float("nan")
    x[4, 7] = float("inf")
    x[5] = float("nan")
    x[6, 1:] = low
    x[7, : E // 2] = -np.inf
    x[8, :] = low
    r, _ = _check(gpu, x, k, groups, max(1, groups // 2), flags)
    assert (r.ids[0] == -1).all() and not r.weights[0].any() and not torch.isnan(r.weights).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_two_logits_are_not_added(gpu, dtype):
    """10 + 0 is more than 4 + 4, but sigmoid(10) + sigmoid(0) = 1.50 is less than 2 sigmoid(4) = 1.96."""
    x = torch.tensor([[10.0, 0.0, 4.0, 4.0]], dtype=dtype)
    r, _ = _check(gpu, x, 1, 2, 1, SIG | TWO)
    assert r.ids.tolist() == [[2]]
    # 3 - 9 is less than 0.5 + 0.5, but e^3 + e^-9 = 20.1 is more than 2 e^0.5 = 3.3
    x = torch.tensor([[3.0, -9.0, 0.5, 0.5]], dtype=dtype)
    r, _ = _check(gpu, x, 2, 2, 1, TWO)
    assert r.ids.tolist() == [[0, 1]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,groups,top_groups,k", [(16, 4, 2, 4), (60, 3, 2, 6), (64, 64, 20, 8), (64, 4, 2, 6),
                                                   (160, 8, 4, 6), (256, 8, 4, 8), (256, 16, 5, 8), (384, 8, 3, 12),
                                                   (500, 5, 2, 8), (512, 32, 7, 8), (520, 4, 2, 8), (1000, 8, 4, 8),
                                                   (4096, 16, 8, 8), (4096, 8, 3, 16), (1000, 4, 2, 20),
                                                   (256, 128, 30, 8), (6000, 4, 2, 8), (9000, 8, 3, 8)])
@pytest.mark.parametrize("flags", [TWO, REN | TWO, SIG | TWO, SIG | REN | TWO])
def test_groups_by_two_scores(gpu, dtype, E, groups, top_groups, k, flags):
    """By the sum of two scores, without a bias and with one; a bias of zeros chooses as none does."""
    x = _logits(43, E, dtype, seed=E + groups, step=1 / 64)
    r, sure = _check(gpu, x, k, groups, top_groups, flags)
    z, sure_z = _check(gpu, x, k, groups, top_groups, flags, bias=torch.zeros(E))
    both = torch.from_numpy(sure & sure_z)
    assert torch.equal(r.ids.cpu()[both], z.ids.cpu()[both])
    b = torch.randint(-20, 21, (E,), generator=torch.Generator().manual_seed(E)).float() / 256
    _check(gpu, x, k, groups, top_groups, flags, bias=b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,groups", [(64, 4), (256, 8), (512, 16), (1000, 8), (4096, 16), (6000, 4)])
@pytest.mark.parametrize("flags", [TWO, REN | TWO, SIG | TWO])
def test_equal_groups_and_few_experts_by_two(gpu, dtype, E, groups, flags):
    """Equal sums: the lower group; a group with one expert counts as its score; infinities and NaN."""
    gs = E // groups
    x = _logits(6, E, dtype, seed=E, step=1 / 8)
    x[0] = x[0, :gs].repeat(groups)              # groups that are alike
    x[1] = -np.inf
    x[1, ::gs] = x[2, ::gs]                      # one expert a group
    x[2, gs + 1:2 * gs] = -np.inf
    x[3, 3 * gs - 1] = float("inf")
    x[4, ::3] = float("nan")
    x[5] = x[5].abs().neg() - 9                  # all far below zero
    _check(gpu, x, 2, groups, groups // 2, flags)
