"""Block norm, balance loss, 8-bit rows and their products together, as a layer uses
them: the serving example against a dense layer in 64 bits, a router's loss and
choices with their gradients, and captured graphs.

Tolerance of the example: its first product's result is rounded to bfloat16 (2^-9 of a
value on average at most), and what is made of it, 2^-8 or so, moves an 8-bit step of
about 1/30 of the rows' size to its neighbour in as many cases as it is parts of a step:
sqrt(2^-8 / 30) = 0.011 of the size at most.  The next product and the sum keep that, and
round to bfloat16 once each: 2^-6 in all."""
import os
import sys

import pytest
import torch

import paper_2608_03676_amd as taot

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _rel(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("R,E,tokens,H,F,k", [(4, 16, 60, 256, 128, 4), (8, 32, 33, 136, 72, 2), (3, 7, 50, 201, 51, 2)])
def test_serving_layer(gpu, R, E, tokens, H, F, k):
    import moe_serving as M
    layer = M.make_layer(R, E, H, F, top_k=k, seed=R)
    layer.router[layer.home == 0] += 0.3 * H ** -0.5  # a rank that receives more than others
    g = torch.Generator(device="cuda").manual_seed(R)
    x, res = (torch.randn((R, tokens, H), generator=g, device="cuda").bfloat16() for _ in range(2))
    h, out, s = M.forward(layer, x, res)
    assert int(s["plan"].schedule.X.sum()) > 0, "the plan moves nothing: the test would not see replicas"
    rows = (s["q"].q.double() * s["q"].scale.double()).view(-1, H)
    # a row's 8-bit values: within half a step of the norm's output
    assert ((rows - s["n"].y.double().view(-1, H)).abs() <= s["q"].scale.double().view(-1, 1) * (0.5 + 1e-4)).all()
    up, down = layer.up.double() * layer.up_scale.double()[..., None], layer.down.double() * layer.down_scale.double()[..., None]
    ids, w = s["r"].ids.view(-1, k).long(), s["r"].weights.view(-1, k).double()
    want = torch.zeros_like(rows)
    for e in range(E):
        both = rows @ up[e].t().contiguous()
        v = both[:, :F] * torch.sigmoid(both[:, :F]) * both[:, F:]
        a = v.abs().amax(1, keepdim=True).clamp(min=1e-30)
        v = torch.round(v / a * 127) * a / 127
        want += (w * (ids == e)).sum(1, keepdim=True) * (v @ down[e].t().contiguous())
    assert _rel(out.view(-1, H), want) < 2.0 ** -6
    d = dict(x=x.double().view(-1, H), res=res.double().view(-1, H))
    n = d["x"] * (d["x"].square().mean(1, keepdim=True) + layer.eps).rsqrt() * layer.post.double() * layer.gate.double()
    assert _rel(h.view(-1, H), layer.alpha * d["res"] + n) < 2.0 ** -8
    h2, out2, _ = M.forward(layer, out, h)  # a layer's results are the next one's inputs
    assert torch.isfinite(h2).all() and torch.isfinite(out2).all()


def test_choices_losses_and_gradients_of_a_router(gpu):
    """dlogits of weights and both losses together, and on through the norms, against 64-bit automatic gradients of the
    formulas.  Each call rounds to 32 bits a few times a value; sums of at most 70 terms of either sign: 1e-4 of the
    size of all is 20 times what they add up to."""
    T, H, E, k = 70, 96, 24, 4
    g = torch.Generator().manual_seed(11)
    x, res, dy, router = (torch.randn(s, generator=g).to(gpu) for s in ((T, H), (T, H), (T, H), (E, H)))
    post, gate, weight = (1 + 0.2 * torch.randn(s, generator=g).to(gpu) for s in ((H,), (2, H), (H,)))
    mask = (torch.rand(T, generator=g) < 0.8).to(gpu)
    dw = torch.randn(T, k, generator=g).to(gpu)
    n = taot.block_norm(x, res, weight, 1e-6, post=post, gate=gate, alpha=0.7)
    logits = n.y @ router.t()
    r = taot.route(logits, k, flags=taot.ROUTE_RENORM)
    b = taot.balance_loss(logits, r.ids, mask=mask)
    cl, cz = torch.tensor(2.0, device=gpu), torch.tensor(0.3, device=gpu)
    dl = taot.route_backward(dw, logits, r.ids, flags=taot.ROUTE_RENORM)
    dl = taot.balance_loss_backward(cl, logits, b.counts, b.tokens, mask=mask, dz=cz, add=dl, out=dl)
    d = taot.block_norm_backward((dy.double() + dl.double() @ router.double()).float(), x, n.h, n.rstd_h, weight,
                                 rstd_x=n.rstd_x, post=post, gate=gate, alpha=0.7)
    X, P, G, W, S = (t.double().requires_grad_() for t in (x, post, gate, weight, res))
    a = X * (X.square().mean(1, keepdim=True) + 1e-6).rsqrt() * P * G.repeat_interleave(T // 2, 0)
    h = 0.7 * S + a
    y = h * (h.square().mean(1, keepdim=True) + 1e-6).rsqrt() * W
    L = y @ router.double().t()
    ids = r.ids.long()
    chosen = torch.softmax(L.gather(1, ids), 1)
    m = mask.double()
    prob = (torch.softmax(L, 1) * m[:, None]).sum(0) / m.sum()
    hits = torch.bincount(ids[mask].flatten(), minlength=E).double()
    loss = E * (hits / hits.sum() * prob).sum()
    z = (torch.logsumexp(L, 1).square() * m).sum() / m.sum()
    assert abs(float(b.loss) - float(loss)) < 1e-5 * float(loss) and abs(float(b.z) - float(z)) < 1e-5 * float(z)
    total = (dy.double() * y).sum() + (dw.double() * chosen).sum() + 2.0 * loss + 0.3 * z
    for name, got, ref in zip(("x", "post", "gate", "weight", "residual"), (d.dx, d.dpost, d.dgate, d.dweight, d.dresidual),
                              torch.autograd.grad(total, (X, P, G, W, S))):
        assert _rel(got, ref) < 1e-4, name


@pytest.mark.parametrize("tokens", [24, 1100])
def test_replays_equal_eager_calls(gpu, tokens):
    """Outputs and workspaces kept, inputs changed in place, several replays with eager work between them; two graphs share
    the workspaces."""
    H, F, E, k, rows = 264, 136, 32, 4, 2
    g = torch.Generator(device="cuda").manual_seed(tokens)

    def new(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    x, res, dy, dh = (new(tokens, H) for _ in range(4))
    post, weight, gate = new(H), new(H), new(4, H)
    logits, mask = new(rows, tokens // rows, E), torch.rand((rows, tokens // rows), generator=g, device="cuda") < 0.9
    ids = torch.randint(0, E, (rows, tokens // rows, k), generator=g, device="cuda").int()
    one = torch.ones(rows, device="cuda")
    up = taot.quantize_rows(new(E, 2 * F, H))
    sizes = torch.multinomial(torch.ones(E, device="cuda"), tokens, replacement=True, generator=g).bincount(minlength=E)
    offsets = torch.cat([torch.zeros(1, device="cuda"), sizes.cumsum(0)]).int()
    experts = torch.randperm(E, generator=g, device="cuda").int()
    L = taot.lib()
    room = {n: torch.empty(s, dtype=torch.uint8, device="cuda") for n, s in dict(
        norm=L.taot_block_norm_backward_workspace_size(tokens, H, 4),
        balance=L.taot_balance_loss_workspace_size(rows, tokens // rows, E),
        product=L.taot_matmul_i8_workspace_size(tokens, E)).items()}

    def new_outputs():
        return dict(n=taot.BlockNorm(), d=taot.BlockNormGrad(), b=taot.Balance(), q=taot.Rows8(), a=taot.Rows8(), up=None, dl=None)

    def step(o, ws):
        n = taot.block_norm(x, res, weight, 1e-6, post=post, gate=gate, out=o["n"])
        q = taot.quantize_rows(n.y, out=o["q"])
        o["up"] = taot.matmul_i8(q.q, q.scale, up.q, up.scale[..., 0], offsets=offsets, experts=experts, out=o["up"],
                                 workspace=ws.get("product"))
        a = taot.quantize_rows(o["up"], gated=True, out=o["a"])
        b = taot.balance_loss(logits, ids, mask=mask, out=o["b"], workspace=ws.get("balance"))
        o["dl"] = taot.balance_loss_backward(one, logits, b.counts, b.tokens, mask=mask, dz=one, out=o["dl"])
        d = taot.block_norm_backward(dy, x, n.h, n.rstd_h, weight, rstd_x=n.rstd_x, post=post, gate=gate, dh=dh, out=o["d"],
                                     workspace=ws.get("norm"))
        return [n.y, n.h, n.rstd_x, n.rstd_h, q.q, q.scale, o["up"], a.q, a.scale, b.loss, b.z, b.counts, b.prob, b.tokens,
                o["dl"], d.dx, d.dresidual, d.dweight, d.dpost, d.dgate]

    graphs = []
    for _ in range(2):
        kept = new_outputs()
        step(kept, room)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = step(kept, room)
        graphs.append((graph, captured))
    for replay in range(4):
        for t in (x, res, logits):
            t.copy_(new(*t.shape))
        offsets[1:-1] = offsets[1:-1].roll(replay).sort().values
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        eager = step(new_outputs(), {})
        torch.cuda.synchronize()
        for which, (_, captured) in enumerate(graphs):
            for i, (a, b) in enumerate(zip(captured, eager)):
                assert torch.equal(a, b), (replay, which, i)


def test_two_streams_at_once(gpu):
    """Calls with workspaces of their own run beside one another."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = torch.randint(-128, 128, (2000, 512), generator=g, device="cuda").to(torch.int8), \
        torch.randint(-128, 128, (8, 384, 512), generator=g, device="cuda").to(torch.int8)
    sx, sw = torch.rand(2000, generator=g, device="cuda"), torch.rand((8, 384), generator=g, device="cuda")
    offsets = torch.arange(0, 2001, 250, device="cuda").int()
    logits = torch.randn((1, 4000, 256), generator=g, device="cuda")
    ids = torch.randint(0, 256, (1, 4000, 8), generator=g, device="cuda").int()
    want, loss = taot.matmul_i8(x, sx, w, sw, offsets=offsets), taot.balance_loss(logits, ids).loss
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [(taot.matmul_i8(x, sx, w, sw, offsets=offsets, stream=s), taot.balance_loss(logits, ids, stream=s).loss)
           for _ in range(5) for s in streams]
    for s in streams:
        s.synchronize()
    for out, l in got:
        assert torch.equal(out, want) and torch.equal(l, loss)
