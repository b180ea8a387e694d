"""Tokens of which each has to count in balance_loss, with a bound on its sums that does not grow with their number."""
import pytest
import torch

import paper_2608_03676_amd as taot
from test_gpu_balance import E, SIGMOID, _case, _reference

pytestmark = pytest.mark.gpu


# A value's additions: a lane's tokens (at most 5 at these sizes), its wave's, 16 waves, up to 16 blocks a thread of the
# last sum and 32 of those: under 160, whatever the number of tokens.
@pytest.mark.parametrize("flags", [0, SIGMOID])
@pytest.mark.parametrize("rows,tokens,experts", [(1, 70001, 16), (1, 70000, 64), (1, 65537, 256), (4, 8191, 160), (1, 4099, 600),
                                                 (1, 6001, 4096)])
def test_each_token_counts(gpu, rows, tokens, experts, flags):
    """Each of many experts has nearly all its score from one token, the first, the last, or one that others decide by
    lot: a token left out would leave its expert nothing."""
    print(f"[balance tokens] {rows} x {tokens} x {experts}", flush=True)
    x, ids, _ = _case(gpu, rows, tokens, experts, 2, torch.float32)
    g = torch.Generator().manual_seed(tokens)
    n = experts - 4
    for r in range(rows):
        at = torch.randperm(tokens, generator=g)[:n]
        at[0], at[1], at[2] = tokens - 1, 0, tokens - 2
        x[r, :, :n] = -30.0 + 0.1 * x[r, :, :n]
        x[r, at.to(gpu), torch.arange(n, device=gpu)] = 3.0
    b = taot.balance_loss(x, ids, flags=flags)
    prob = _reference(x, ids, None, flags != 0)[3]
    alone = prob[:, :n] * tokens
    assert (alone > 1e-3).all() and (alone < 1.5).all()
    R = float(x.max() - x.min())
    assert ((b.prob.double() - prob).abs() <= (R + 64 + 160) * E * prob).all()
