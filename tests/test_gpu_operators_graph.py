"""The calls around the planner under HIP graph capture: outputs and workspaces
kept by the caller, inputs changed in place, several replays with eager work in
between, each equal to the eager calls."""
import pytest
import torch

import paper_2608_03676_amd as taot

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [40, 3000])  # a short row in one launch, and the launches of a long one
def test_replays_equal_eager_calls(gpu, tokens):
    R, E, H, k, K = 8, 32, 264, 4, 2
    flags = taot.ROUTE_SIGMOID | taot.ROUTE_RENORM
    g = torch.Generator(device="cuda").manual_seed(tokens)

    def new(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    x, res, logits = new(1, tokens, H).bfloat16(), new(1, tokens, H).bfloat16(), new(1, 1, tokens, E)
    w, bias = new(H).bfloat16(), 0.01 * new(E)
    home = (torch.arange(E, device="cuda") // (E // R)).int()
    slot = torch.randint(-1, E, (1, R * K), generator=g, device="cuda").int()
    X = torch.randint(0, tokens // 8, (1, R, R * K), generator=g, device="cuda").int()
    N = tokens * k
    n, r, d, ng, cg = taot.Norm(), taot.Routing(), taot.Dispatch(), taot.NormGrad(), taot.CombineGrad()
    kept = {}

    def step(keep):
        o = (n, r, d, ng, cg) if keep else (taot.Norm(), taot.Routing(), taot.Dispatch(), taot.NormGrad(), taot.CombineGrad())
        b = kept if keep else {}
        a = taot.add_rms_norm(x, w, 1e-6, residual=res, group=128, out=o[0])
        c = taot.route(logits, k, bias=bias, groups=4, top_groups=2, flags=flags, out=o[1])
        m = taot.dispatch_map(c.ids.view(1, 1, N), home, slot, X, K, rank0=3, out=o[2], workspace=b.get("map"))
        rows, scale = taot.dispatch_rows(a.q.view(1, 1, tokens, H), m.pos, scale=a.scale.view(1, 1, tokens, -1),
                                         out=b.get("rows"), out_scale=b.get("scale"))
        y = taot.dispatch_rows(a.y.view(1, 1, tokens, H), m.pos, out=b.get("y"))
        back = taot.combine_rows(y, m.pos, weights=c.weights.view(1, 1, N), top_k=k, out=b.get("back"))
        cb = taot.combine_rows_backward(back, y, m.pos, c.weights.view(1, 1, N), out=o[4])
        dl = taot.route_backward(cb.dweights.view(c.weights.shape), logits, c.ids, flags=flags, out=b.get("dl"))
        db = taot.add_rms_norm_backward(back.view(1, tokens, H), a.h, a.rstd, w, out=o[3], workspace=b.get("norm"))
        b.update(rows=rows, scale=scale, y=y, back=back, dl=dl)
        return [a.y, a.q.view(torch.uint8), a.scale, a.h, c.ids, c.weights, m.pos, m.offsets, m.sends, m.status,
                rows.view(torch.uint8), scale, back, cb.dy, cb.dweights, dl, db.dx, db.dweight]

    L = taot.lib()
    kept["map"] = torch.empty(L.taot_dispatch_map_workspace_size(1, 1, N, R, E, K), dtype=torch.uint8, device="cuda")
    kept["norm"] = torch.empty(L.taot_add_rms_norm_backward_workspace_size(tokens, H), dtype=torch.uint8, device="cuda")
    step(True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(True)
    for replay in range(4):
        x.copy_(new(1, tokens, H))
        logits.copy_(new(1, 1, tokens, E))
        graph.replay()
        torch.cuda.synchronize()
        eager = step(False)
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(captured, eager)):
            assert torch.equal(a, b), (replay, i)
