"""The example layer: norm, router, planner, dispatch, experts and the way back
together, against a dense layer that knows no ranks, in 64 bits.

What the example rounds to 16 bits (the norm's output, the experts' rows, the
sums) the dense layer does not: 2^-8 each, a few of them in a row; the 8-bit rows
are taken from the example.  Gradients of the dense layer are autograd's, with
the 8-bit rounding as the identity."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _rel(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("R,E,tokens,H,k", [(4, 16, 60, 256, 4), (16, 64, 33, 128, 8), (3, 7, 50, 200, 2)])
def test_layer_against_a_dense_one(gpu, R, E, tokens, H, k):
    import moe_layer as M
    layer = M.make_layer(R, E, H, top_k=k, seed=R)
    layer.bias[layer.home == 0] += 0.3
    g = torch.Generator(device="cuda").manual_seed(R)
    x, res, dout = (torch.randn((R, tokens, H), generator=g, device="cuda").bfloat16() for _ in range(3))
    out, s = M.forward(layer, x, res)
    grads = M.backward(layer, s, dout)
    assert int(s["plan"].schedule.X.sum()) > 0, "the plan moves nothing: the test would not see replicas"
    assert int(s["d"].sends.sum()) == R * tokens * k

    w, gate, experts = (t.double().requires_grad_() for t in (layer.norm, layer.gate, layer.experts))
    X = x.double().requires_grad_()
    h = X + res.double()
    y = h * (h.square().mean(-1, keepdim=True) + layer.eps).rsqrt() * w
    n, ids = s["n"], s["r"].ids[0].long()
    value = n.q.double() * n.scale.double().repeat_interleave(M.GROUP, -1)[..., :H]
    assert _rel(value, y.detach()) < 2.0 ** -4  # half a unit of the 8-bit format
    sent = y + (value - y).detach()             # its value, and the identity's gradient
    p = torch.sigmoid(y.reshape(-1, H) @ gate.t()).view(R, tokens, E).gather(2, ids)
    p = p / p.sum(-1, keepdim=True)
    want = h.clone()
    for e in range(E):
        mine = (p * (ids == e)).sum(-1, keepdim=True)
        want = want + mine * (sent.reshape(-1, H) @ experts[e]).view(R, tokens, H)
    assert _rel(out, want.detach()) < 3 * 2.0 ** -8
    dx, dw, dgate, dexperts = torch.autograd.grad(want, (X, w, gate, experts), dout.double())
    for name, ref in (("x", dx), ("norm", dw), ("gate", dgate), ("experts", dexperts)):
        assert _rel(grads[name], ref) < 4 * 2.0 ** -8, name


def test_the_plan_evens_the_loads(gpu):
    import moe_layer as M
    layer = M.make_layer(16, 64, 128)
    layer.bias[layer.home == 3] += 0.5
    g = torch.Generator(device="cuda").manual_seed(2)
    x, res = (torch.randn((16, 200, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    _, s = M.forward(layer, x, res)
    before, after = s["plan"].loads.load_r[0], s["d"].sends[0].sum(0)
    assert int(after.sum()) == int(before.sum())
    assert int(after.max()) < int(before.max())
