"""One mixture-of-experts layer with a planned step, forward and backward, all R ranks as data on one GPU.

    residual + x -> norm (and its 8-bit form) -> router -> planner -> dispatch by the plan
        -> experts, each at the rank that the plan sends its tokens to -> weighted sum -> new residual

The products with the router's and the experts' weights are torch's; everything between them is this
package's.  On a cluster each rank calls the same functions with its own row (dispatch_map with rank0 = its
number), and an all-to-all with `sends` lies between dispatch_rows and the experts, and before combine_rows.

    python examples/moe_layer.py [--tokens 256] [--width 512] [--ranks 16] [--experts 64] [--hot 0.5]
"""
import argparse
import dataclasses
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_03676_amd as taot  # noqa: E402

FLAGS = taot.ROUTE_SIGMOID | taot.ROUTE_RENORM
GROUP = 128  # columns that share a scale in the 8-bit rows


@dataclasses.dataclass
class Layer:
    norm: torch.Tensor     # [H] weight of the norm
    gate: torch.Tensor     # [E][H] router
    bias: torch.Tensor     # [E] balance bias of the router
    experts: torch.Tensor  # [E][H][H]
    home: torch.Tensor     # [E] int32 home rank
    cost: torch.Tensor     # [R][R] topology cost
    K: int = 2             # guest slots of a rank
    top_k: int = 8
    eps: float = 1e-6


def make_layer(R, E, H, top_k=8, device="cuda", seed=0) -> Layer:
    g = torch.Generator().manual_seed(seed)
    r = torch.arange(R)
    cost = 1.0 + 3.0 * (r[:, None] // 8 != r[None, :] // 8).float()  # nodes of eight ranks
    cost.fill_diagonal_(0.0)
    layer = Layer(norm=1 + 0.1 * torch.randn(H, generator=g), gate=torch.randn(E, H, generator=g) * H ** -0.5,
                  bias=torch.zeros(E), experts=torch.randn(E, H, H, generator=g) * H ** -0.5,
                  home=(torch.arange(E) * R // E).int(), cost=cost, top_k=top_k)
    for f in ("norm", "gate", "bias", "experts", "home", "cost"):
        setattr(layer, f, getattr(layer, f).to(device))
    return layer


def _instances(layer: Layer, slot_expert: torch.Tensor):
    """The expert of each instance in send order: by rank, its own experts, then its guest slots (-1: empty)."""
    R, K = layer.cost.shape[0], layer.K
    home, slots = layer.home.tolist(), slot_expert.tolist()
    out = []
    for r in range(R):
        out += [e for e in range(len(home)) if home[e] == r] + slots[r * K:(r + 1) * K]
    return out


def _runs(layer: Layer, plan, d):
    """(source rank, expert, first row, end) of every instance that receives rows."""
    experts = _instances(layer, plan.schedule.slot_expert[0])
    offsets = d.offsets[0].tolist()
    return [(r, e, off[i], off[i + 1]) for r, off in enumerate(offsets) for i, e in enumerate(experts)
            if off[i + 1] > off[i]]


def forward(layer: Layer, x: torch.Tensor, residual: torch.Tensor):
    """x, residual [R][tokens][H] -> (new residual [R][tokens][H], what the backward pass needs)."""
    R, tokens, H = x.shape
    E, k = layer.gate.shape[0], layer.top_k
    n = taot.add_rms_norm(x, layer.norm, layer.eps, residual=residual, group=GROUP)
    logits = (n.y.view(-1, H).float() @ layer.gate.t()).view(1, R, tokens, E)
    r = taot.route(logits, k, bias=layer.bias, flags=FLAGS)
    ids = r.ids.view(1, R, tokens * k)
    plan = taot.plan_step(ids, layer.home, layer.cost, E, eps=0.2, iters=200, K=layer.K)
    d = taot.dispatch_map(ids, layer.home, plan.schedule.slot_expert, plan.schedule.X, layer.K)
    rows, scales = taot.dispatch_rows(n.q[None], d.pos, scale=n.scale[None])
    # the experts, wherever their rows went: values of the 8-bit rows times the expert's weight
    sent = rows.float() * scales.repeat_interleave(GROUP, -1)[..., :H]
    back = torch.zeros((1, R, tokens * k, H), dtype=x.dtype, device=x.device)
    for rank, e, lo, hi in _runs(layer, plan, d):
        back[0, rank, lo:hi] = (sent[0, rank, lo:hi] @ layer.experts[e]).to(x.dtype)
    out = taot.combine_rows(back, d.pos, weights=r.weights.view(1, R, -1), top_k=k)
    return n.h + out[0], dict(n=n, logits=logits, r=r, plan=plan, d=d, sent=sent, back=back)


def backward(layer: Layer, saved, dout: torch.Tensor):
    """Gradients by x (and the residual alike), the norm's weight, the router and the experts."""
    n, r, d = saved["n"], saved["r"], saved["d"]
    R, tokens, H = dout.shape
    k = layer.top_k
    c = taot.combine_rows_backward(dout[None], saved["back"], d.pos, r.weights.view(1, R, -1))
    drows = torch.zeros_like(c.dy)
    dexperts = torch.zeros_like(layer.experts)
    for rank, e, lo, hi in _runs(layer, saved["plan"], d):
        dy = c.dy[0, rank, lo:hi].float()
        drows[0, rank, lo:hi] = (dy @ layer.experts[e].t()).to(drows.dtype)
        dexperts[e] += saved["sent"][0, rank, lo:hi].t() @ dy
    dy = taot.combine_rows(drows, d.pos, top_k=k)[0].float()  # dispatch_rows' gradient
    dlogits = taot.route_backward(c.dweights.view(r.weights.shape), saved["logits"], r.ids, flags=FLAGS)
    dlogits = dlogits.view(-1, layer.gate.shape[0])
    dgate = dlogits.t() @ n.y.view(-1, H).float()
    dy = (dy.view(-1, H) + dlogits @ layer.gate).view(R, tokens, H).to(n.h.dtype)
    g = taot.add_rms_norm_backward(dy, n.h, n.rstd, layer.norm, dh=dout)
    return dict(x=g.dx, norm=g.dweight, gate=dgate, experts=dexperts)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--ranks", type=int, default=16)
    ap.add_argument("--experts", type=int, default=64)
    ap.add_argument("--tokens", type=int, default=256, help="tokens of a rank")
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hot", type=float, default=0.5, help="how far the first rank's experts are preferred")
    a = ap.parse_args()
    layer = make_layer(a.ranks, a.experts, a.width)
    layer.bias[layer.home == 0] += a.hot  # a rank that receives more than it can take
    g = torch.Generator(device="cuda").manual_seed(1)
    x, res, dout = (torch.randn((a.ranks, a.tokens, a.width), generator=g, device="cuda").bfloat16() for _ in range(3))
    out, saved = forward(layer, x, res)
    grads = backward(layer, saved, dout)
    load, sends = saved["plan"].loads.load_r[0], saved["d"].sends[0].sum(0)
    print(f"{a.ranks} ranks, {a.experts} experts, {a.tokens} tokens of {a.width} a rank, top {layer.top_k}")
    print(f"largest rank load {int(load.max())} of a mean {float(load.float().mean()):.0f}; with the plan {int(sends.max())}")
    print("norms: out %.4g, " % out.float().norm() + ", ".join(f"d{n} {v.float().norm():.4g}" for n, v in grads.items()))


if __name__ == "__main__":
    main()
