"""One mixture-of-experts layer in service, with experts in 8-bit integers, all R ranks as data on one GPU.

    block's output, residual -> norms, gate, new residual -> 8-bit rows -> router -> planner -> dispatch by the plan
        -> up product -> gated activation as 8-bit rows -> down product -> weighted sum

Weights are rounded once, a scale for each channel; rows travel as 8-bit integers and a scale.  The products take
each run of rows that the plan sends to an expert's instance with that expert's weight, without a copy to the host.

    python examples/moe_serving.py [--tokens 64] [--width 512] [--inner 256] [--ranks 8] [--experts 32]
"""
import argparse
import dataclasses
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_03676_amd as taot  # noqa: E402

FLAGS = taot.ROUTE_SIGMOID | taot.ROUTE_RENORM


@dataclasses.dataclass
class Layer:
    norm: torch.Tensor        # [H] of the norm before the router and the experts
    post: torch.Tensor        # [H] of the norm behind the block before
    gate: torch.Tensor        # [H] gate of that block's output
    router: torch.Tensor      # [E][H]
    up: torch.Tensor          # [E][2 F][H] int8: gate and up projection
    up_scale: torch.Tensor    # [E][2 F]
    down: torch.Tensor        # [E][H][F] int8
    down_scale: torch.Tensor  # [E][H]
    home: torch.Tensor        # [E] int32 home rank
    cost: torch.Tensor        # [R][R] topology cost
    K: int = 2                # guest slots of a rank
    top_k: int = 4
    eps: float = 1e-6
    alpha: float = 1.0        # scale of the residual


def make_layer(R, E, H, F, top_k=4, device="cuda", seed=0) -> Layer:
    g = torch.Generator().manual_seed(seed)

    def new(*shape, scale=1.0, shift=0.0):
        return (shift + scale * torch.randn(shape, generator=g)).to(device)

    r = torch.arange(R)
    cost = 1.0 + 3.0 * (r[:, None] // 8 != r[None, :] // 8).float()  # nodes of eight ranks
    cost.fill_diagonal_(0.0)
    up, down = taot.quantize_rows(new(E, 2 * F, H, scale=H ** -0.5)), taot.quantize_rows(new(E, H, F, scale=F ** -0.5))
    return Layer(norm=new(H, scale=0.1, shift=1.0).bfloat16(), post=new(H, scale=0.1, shift=0.7).bfloat16(),
                 gate=new(H, scale=0.3).bfloat16(), router=new(E, H, scale=H ** -0.5), up=up.q, up_scale=up.scale[..., 0],
                 down=down.q, down_scale=down.scale[..., 0], home=(torch.arange(E) * R // E).int().to(device),
                 cost=cost.to(device), top_k=top_k)


def runs(layer: Layer, d, slot_expert: torch.Tensor):
    """(offsets, experts) of the runs of all send buffers [R][N]: for each the instances in send order, by rank its own
    experts, then its guest slots, and behind them what is sent nowhere (expert -1)."""
    E, R, K, N = layer.home.numel(), layer.cost.shape[0], layer.K, d.pos.shape[-1]
    dev = layer.home.device
    rank = torch.cat([2 * layer.home, 2 * (torch.arange(R * K, device=dev) // K).int() + 1])
    expert = torch.cat([torch.arange(E, device=dev).int(), slot_expert])
    order = torch.cat([expert[rank.sort(stable=True).indices], torch.full((1,), -1, device=dev, dtype=torch.int32)])
    first = d.offsets[0] + N * torch.arange(R, device=dev, dtype=torch.int32)[:, None]
    end = torch.full((1,), R * N, device=dev, dtype=torch.int32)
    return torch.cat([first.reshape(-1), end]), order.repeat(R)


def forward(layer: Layer, x: torch.Tensor, residual: torch.Tensor):
    """x (the block's output before), residual [R][tokens][H] -> (new residual, the experts' output), the next layer's
    residual and x, and what was on the way."""
    R, tokens, H = x.shape
    E, k = layer.router.shape[0], layer.top_k
    n = taot.block_norm(x, residual, layer.norm, layer.eps, post=layer.post, gate=layer.gate, alpha=layer.alpha)
    q = taot.quantize_rows(n.y)
    r = taot.route((n.y.view(-1, H).float() @ layer.router.t()).view(1, R, tokens, E), k, flags=FLAGS)
    ids = r.ids.view(1, R, tokens * k)
    plan = taot.plan_step(ids, layer.home, layer.cost, E, eps=0.2, iters=200, K=layer.K)
    d = taot.dispatch_map(ids, layer.home, plan.schedule.slot_expert, plan.schedule.X, layer.K)
    rows, scales = taot.dispatch_rows(q.q[None], d.pos, scale=q.scale[None])
    offsets, experts = runs(layer, d, plan.schedule.slot_expert[0])
    both = taot.matmul_i8(rows.view(-1, H), scales, layer.up, layer.up_scale, offsets=offsets, experts=experts)
    act = taot.quantize_rows(both, gated=True)
    back = taot.matmul_i8(act.q, act.scale, layer.down, layer.down_scale, offsets=offsets, experts=experts)
    out = taot.combine_rows(back.view(1, R, tokens * k, H), d.pos, weights=r.weights.view(1, R, -1), top_k=k)
    return n.h, out[0], dict(n=n, q=q, r=r, plan=plan, d=d)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--ranks", type=int, default=8)
    ap.add_argument("--experts", type=int, default=32)
    ap.add_argument("--tokens", type=int, default=64, help="tokens of a rank")
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--inner", type=int, default=256)
    a = ap.parse_args()
    layer = make_layer(a.ranks, a.experts, a.width, a.inner)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, h = (torch.randn((a.ranks, a.tokens, a.width), generator=g, device="cuda").bfloat16() for _ in range(2))
    for i in range(3):
        h, x, saved = forward(layer, x, h)
        print(f"layer {i}: residual {h.float().norm():.4g}, output {x.float().norm():.4g}, "
              f"copies to guests {int(saved['plan'].schedule.X.sum())}")


if __name__ == "__main__":
    main()
