"""Cases of the operators around the planner: what makes the routing ids, and what carries a plan out.

  norm      add_rms_norm             residual addition, root-mean-square norm, 8-bit output with scales
  norm_bwd  add_rms_norm_backward
  route     route                    logits -> experts and weights of each token (plan_loads reads the ids)
  route_bwd route_backward
  map       dispatch_map             each routed copy's place in its source rank's send buffer, as the schedule splits them
  rows      dispatch_rows            8-bit rows and their scales into the send buffer
  combine   combine_rows             weighted sum of the rows that came back
  combine_bwd  combine_rows_backward

`own` chooses between the package's kernels and the plain form in elementary tensor operations.
Ranks, experts, tokens and choices are those of the benchmark's configurations; row widths are generic.
"""
import math

import torch

own = False

SIGMOID, RENORM, GROUP_TWO = 0x1, 0x2, 0x4  # flags of route
F8_MAX = 448.0   # largest finite value of the 8-bit format (e4m3)
F8_FLOOR = 1e-30  # smallest magnitude that a scale is made for
TINY = 1e-20     # added to a sum of chosen scores before it divides

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # a few sequences in generation: one token each, all latency
        dict(name="norm_decode", kind="norm", T=4, H=2048, dtype="bf16", residual=True, group=128),
        # one rank's tokens of a long-sequence step, 8-bit payload in groups of 128
        dict(name="norm_step", kind="norm", T=16384, H=4096, dtype="bf16", residual=True, group=128),
        # ragged: a width that no vector divides, one scale a row, no residual
        dict(name="norm_odd", kind="norm", T=1237, H=5003, dtype="f16", residual=False, group=0),
        dict(name="norm_bwd_step", kind="norm_bwd", T=8192, H=5120, dtype="bf16", residual=True),
        # the benchmark's smallest layer: 16 tokens in generation, 128 experts
        dict(name="route_decode", kind="route", T=16, E=128, k=8, dtype="bf16", sigmoid=False, renorm=True, groups=1,
             top_groups=1, bias=False, two=False),
        # four micro-batches of 16384 tokens, 256 experts in 8 groups, scores with a balance bias
        dict(name="route_groups", kind="route", T=65536, E=256, k=8, dtype="f32", sigmoid=True, renorm=True, groups=8,
             top_groups=4, bias=True, two=True),
        # the stress configuration's 4096 experts
        dict(name="route_wide", kind="route", T=8192, E=4096, k=8, dtype="bf16", sigmoid=False, renorm=False, groups=1,
             top_groups=1, bias=False, two=False),
        dict(name="route_bwd_step", kind="route_bwd", T=32768, E=384, k=8, dtype="bf16", sigmoid=False, renorm=False),
        # one source rank of 256 in one layer: what a rank does for itself
        dict(name="map_rank", kind="map", B=1, R=256, rows=1, E=384, tokens=8192, k=8, K=2, zipf=1.3),
        # all 64 source ranks of a layer
        dict(name="map_layer", kind="map", B=1, R=64, rows=64, E=256, tokens=16384, k=8, K=2, zipf=1.2),
        dict(name="rows_step", kind="rows", rows=1, tokens=8192, k=8, H=4096, group=128),
        dict(name="combine_bwd_step", kind="combine_bwd", rows=1, tokens=8192, k=8, H=2048, dtype="bf16"),
    ]


def _size(rng, lo, hi):
    """A size spread over the logarithm of lo..hi: odd, or a multiple of ten."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))
    return n if n < 16 else n | 1 if rng.random() < 0.5 else n // 10 * 10


def _width(rng):
    return rng.choice([64, 256, 512, 1024, 2048, 2560, 4096, 5120, 8192]) + rng.choice([0, 0, 0, 0, 8, 4, -1, 3])


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "route", "route", "route_bwd", "map", "map", "rows", "combine", "combine_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("norm", "norm_bwd"):
        H = _width(rng)
        c = dict(kind=kind, T=_size(rng, 1, min(32768, (1 << 25) // H)), H=H, dtype=dtype, residual=rng.random() < 0.7)
        if kind == "norm":
            c["group"] = rng.choice([0, 32, 64, 128, 128, 128])
        return c
    if kind in ("route", "route_bwd"):
        sigmoid = rng.random() < 0.5
        k = rng.choice([1, 2, 4, 6, 8, 8])
        groups = rng.choice([1, 1, 4, 8])
        E = rng.choice([16, 64, 128, 160, 256, 384, 512, 1000, 4096])
        c = dict(kind=kind, T=_size(rng, 1, (1 << 25) // E // 2), E=E, k=k, dtype=dtype, sigmoid=sigmoid,
                 renorm=rng.random() < 0.7)
        if kind == "route":
            c.update(groups=groups, top_groups=max(1, groups // 2), bias=sigmoid, two=sigmoid and groups > 1)
        return c
    tokens, k = _size(rng, 1, 16384), rng.choice([1, 2, 4, 6, 8])
    if kind == "map":
        R = rng.choice([4, 16, 24, 64, 256])
        rows = rng.choice([1, R])
        if rows * tokens * k > 1 << 22:
            rows = 1
        return dict(kind=kind, B=rng.choice([1, 1, 2]), R=R, rows=rows, E=R * rng.choice([1, 2, 4]) + rng.choice([0, 0, 1]),
                    tokens=tokens, k=k, K=rng.choice([1, 2, 4]), zipf=round(rng.uniform(0.8, 1.5), 2))
    H = _width(rng)
    c = dict(kind=kind, rows=rng.choice([1, 1, 3]), tokens=0, k=k, H=H)
    c["tokens"] = min(tokens, max(1, (1 << 26) // (c["rows"] * k * H)))
    if kind == "rows":
        return dict(c, group=rng.choice([32, 64, 128, 128]))
    return dict(c, dtype=dtype)


# ---- inputs -----------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _routing(g, rows, tokens, k, E, zipf):
    """[rows][tokens * k] int32 expert ids under a Zipf law over a seeded permutation."""
    p = torch.arange(1, E + 1, device="cuda", dtype=torch.float64) ** -zipf
    p = p[torch.randperm(E, generator=g, device="cuda")]
    cdf = (p / p.sum()).cumsum(0).float()
    x = torch.rand((rows, tokens * k), generator=g, device="cuda")
    return torch.searchsorted(cdf, x, right=True, out_int32=True).clamp_(max=E - 1)


def _positions(g, rows, N):
    """[rows][N] int32: an order of the copies as a dispatch gives it (grouped by 64 destinations, stable)."""
    dest = torch.randint(64, (rows, N), generator=g, device="cuda")
    order = dest.sort(dim=1, stable=True).indices
    at = torch.arange(N, device="cuda", dtype=torch.int32).expand(rows, N).contiguous()
    return torch.empty((rows, N), dtype=torch.int32, device="cuda").scatter_(1, order, at)


def _plan(c, g, ids):
    """A schedule of the kind the planner gives: the hottest experts copied to guest slots, each copy an
    equal share of every source rank's tokens (one slot in eight stays empty)."""
    B, R, E, S = c["B"], c["R"], c["E"], c["R"] * c["K"]
    x = torch.zeros((B, E), dtype=torch.int64, device="cuda")
    x.scatter_add_(1, ids.view(B, -1).long(), torch.ones_like(ids.view(B, -1), dtype=torch.int64))
    hot = x.sort(dim=1, descending=True, stable=True).indices[:, :max(1, E // 8)]
    pick = (torch.rand((B, S), generator=g, device="cuda").square() * hot.shape[1]).long().clamp_(max=hot.shape[1] - 1)
    slot = hot.gather(1, pick).int()
    slot = torch.where(torch.rand((B, S), generator=g, device="cuda") < 0.125, torch.full_like(slot, -1), slot)
    copies = torch.zeros((B, E + 1), dtype=torch.int64, device="cuda")
    copies.scatter_add_(1, slot.long() % (E + 1), torch.ones_like(slot, dtype=torch.int64))
    share = (x[:, :E] // (c["rows"] * (copies[:, :E] + 1))).gather(1, slot.long().clamp(min=0))
    share = torch.where(slot >= 0, share, torch.zeros_like(share))
    jitter = torch.rand((B, R, S), generator=g, device="cuda") * 0.4 + 0.7
    return slot.contiguous(), (share[:, None, :] * jitter).int().contiguous()


def prepare(case, seed):
    c, g = case, _gen(seed)
    kind = c["kind"]
    s = dict(case=c)
    if kind in ("norm", "norm_bwd"):
        T, H, dt = c["T"], c["H"], DTYPES[c["dtype"]]
        wide = 1 + 7 * (torch.rand(H, generator=g, device="cuda") < 0.01).float()  # a few channels far above the rest
        s["weight"] = (1 + 0.2 * _randn(g, H)).to(dt)
        if kind == "norm":
            s["x"] = _randn(g, T, H, dtype=dt)
            s["residual"] = (_randn(g, T, H) * 2 * wide).to(dt) if c["residual"] else None
        else:
            h = _randn(g, T, H) * 2 * wide
            s["h"] = h.to(dt)
            s["rstd"] = (s["h"].float().square().mean(1) + 1e-6).rsqrt()
            s["dy"] = (0.01 * _randn(g, T, H)).to(dt)
            s["dh"] = (0.01 * _randn(g, T, H)).to(dt) if c["residual"] else None
    elif kind in ("route", "route_bwd"):
        T, E, dt = c["T"], c["E"], DTYPES[c["dtype"]]
        s["logits"] = (1.2 * _randn(g, T, E) + 0.7 * _randn(g, E)).to(dt)
        if kind == "route":
            steps = torch.randint(-40, 41, (E,), generator=g, device="cuda")  # the bias moves in steps of a thousandth
            s["bias"] = steps.float() * 0.001 if c["bias"] else None
        else:
            s["ids"] = s["logits"].float().sort(dim=1, descending=True, stable=True).indices[:, :c["k"]].int().contiguous()
            s["dweights"] = _randn(g, T, c["k"])
    elif kind == "map":
        E, R = c["E"], c["R"]
        e = torch.arange(E, device="cuda", dtype=torch.int32)
        s["home"] = e // (E // R) if E % R == 0 else e % R
        s["ids"] = _routing(g, c["B"] * c["rows"], c["tokens"], c["k"], E, c["zipf"]).view(c["B"], c["rows"], -1)
        s["slot_expert"], s["X"] = _plan(c, g, s["ids"])
        s["rank0"] = 0 if c["rows"] == R else seed % R
    else:
        rows, tokens, N, H = c["rows"], c["tokens"], c["tokens"] * c["k"], c["H"]
        s["pos"] = _positions(g, rows, N)
        if kind == "rows":
            s["x"] = _randn(g, rows, tokens, H).mul_(60).clamp_(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn)
            s["scale"] = _randn(g, rows, tokens, -(-H // c["group"])).abs_() * 0.01 + 1e-4
        else:
            w = torch.rand((rows, N), generator=g, device="cuda").view(rows, tokens, -1) + 0.1
            s["weights"] = (w / w.sum(2, keepdim=True)).view(rows, N)
            s["y"] = _randn(g, rows, N, H, dtype=DTYPES[c["dtype"]])
            if kind == "combine_bwd":
                s["dout"] = (0.01 * _randn(g, rows, tokens, H)).to(DTYPES[c["dtype"]])
    return s


# ---- one pass ---------------------------------------------------------------

def run(s):
    return _kernels(s) if own else _plain(s)


def _flags(c):
    return (SIGMOID if c["sigmoid"] else 0) | (RENORM if c["renorm"] else 0) | (GROUP_TWO if c.get("two") else 0)


def _kernels(s):
    import paper_2608_03676_amd as taot
    c = s["case"]
    kind = c["kind"]
    if kind == "norm":
        n = taot.add_rms_norm(s["x"], s["weight"], 1e-6, residual=s["residual"], group=c["group"])
        return [n.y, n.q, n.scale, n.rstd, n.h if c["residual"] else None]
    if kind == "norm_bwd":
        d = taot.add_rms_norm_backward(s["dy"], s["h"], s["rstd"], s["weight"], dh=s["dh"])
        return [d.dx, d.dweight]
    if kind == "route":
        r = taot.route(s["logits"], c["k"], bias=s["bias"], groups=c["groups"], top_groups=c["top_groups"],
                       scale=2.5, flags=_flags(c))
        return [r.ids, r.weights]
    if kind == "route_bwd":
        return taot.route_backward(s["dweights"], s["logits"], s["ids"], scale=2.5, flags=_flags(c))
    if kind == "map":
        m = taot.dispatch_map(s["ids"], s["home"], s["slot_expert"], s["X"], c["K"], rank0=s["rank0"])
        return [m.pos, m.offsets, m.sends]
    if kind == "rows":
        return list(taot.dispatch_rows(s["x"], s["pos"], scale=s["scale"]))
    if kind == "combine":
        return taot.combine_rows(s["y"], s["pos"], weights=s["weights"], top_k=c["k"])
    return list(taot.combine_rows_backward(s["dout"], s["y"], s["pos"], s["weights"]))


def _plain(s):
    return {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "route": _plain_route, "route_bwd": _plain_route_bwd,
            "map": _plain_map, "rows": _plain_rows, "combine": _plain_combine,
            "combine_bwd": _plain_combine_bwd}[s["case"]["kind"]](s)


def _plain_norm(s):
    x, w, r = s["x"], s["weight"], s["residual"]
    T, H = x.shape
    G = s["case"]["group"] or H
    h = x.float() if r is None else x.float() + r.float()
    rstd = 1 / torch.sqrt(h.square().mean(1) + 1e-6)
    y = h * rstd[:, None] * w.float()
    n = -(-H // G)
    p = y if n * G == H else torch.cat([y, y.new_zeros((T, n * G - H))], 1)
    p = p.view(T, n, G)
    amax = p.abs().amax(2).clamp(min=F8_FLOOR)
    q = (p * (F8_MAX / amax)[:, :, None]).view(T, -1)[:, :H].to(torch.float8_e4m3fn)
    return [y.to(x.dtype), q, amax / F8_MAX, rstd, None if r is None else h.to(x.dtype)]


def _plain_norm_bwd(s):
    h, rstd, w = s["h"].float(), s["rstd"][:, None], s["weight"].float()
    dy = s["dy"].float()
    g = dy * w
    dx = rstd * (g - h * (rstd * rstd * (g * h).mean(1, keepdim=True)))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return [dx.to(s["h"].dtype), (dy * h * rstd).sum(0)]


def _best(keys, k):
    """The k largest of each row in descending order, the lower index first among equals."""
    v, i = keys.sort(dim=-1, descending=True, stable=True)
    return v[..., :k], i[..., :k]


def _plain_route(s):
    c, x = s["case"], s["logits"].float()
    T, E = x.shape
    score = 1 / (1 + torch.exp(-x)) if c["sigmoid"] else x
    key = score if s["bias"] is None else score + s["bias"]
    if c["groups"] > 1:
        by = key.view(T, c["groups"], -1)
        if c["two"]:
            top = _best(by, 2)[0]
            value = top[..., 0] + top[..., 1]
        else:
            value = by.amax(2)
        keep = torch.zeros_like(value, dtype=torch.bool).scatter_(1, _best(value, c["top_groups"])[1], True)
        key = torch.where(keep[:, :, None], by, torch.full_like(by, -math.inf)).view(T, E)
    ids = _best(key, c["k"])[1]
    if c["sigmoid"]:
        w = score.gather(1, ids)
        w = w / (w.sum(1, keepdim=True) + TINY) if c["renorm"] else w
    else:
        p = (x - x.amax(1, keepdim=True)).exp()
        w = p.gather(1, ids)
        w = w / (w.sum(1, keepdim=True) if c["renorm"] else p.sum(1, keepdim=True))
    return [ids.int(), w * 2.5]


def _plain_route_bwd(s):
    c, x, ids, dw = s["case"], s["logits"].float(), s["ids"].long(), 2.5 * s["dweights"]
    if c["sigmoid"]:
        p = 1 / (1 + torch.exp(-x.gather(1, ids)))
        if c["renorm"]:
            total = p.sum(1, keepdim=True) + TINY
            dw = (dw - (dw * p).sum(1, keepdim=True) / total) / total
        dx = torch.zeros_like(x).scatter_(1, ids, dw * p * (1 - p))
    else:
        p = (x - x.amax(1, keepdim=True)).exp()
        if c["renorm"]:
            v = p.gather(1, ids)
            v = v / v.sum(1, keepdim=True)
            dx = torch.zeros_like(x).scatter_(1, ids, v * (dw - (dw * v).sum(1, keepdim=True)))
        else:
            p = p / p.sum(1, keepdim=True)
            dp = torch.zeros_like(x).scatter_(1, ids, dw)
            dx = p * (dp - (dp * p).sum(1, keepdim=True))
    return dx.to(s["logits"].dtype)


def _plain_map(s):
    c, ids, home, slot, X, K = s["case"], s["ids"], s["home"].long(), s["slot_expert"].long(), s["X"], s["case"]["K"]
    B, rows, N = ids.shape
    E, S, R = home.numel(), slot.shape[1], X.shape[1]
    e = ids.long()
    # which occurrence of its expert each copy is, in its row
    by, order = e.sort(dim=2, stable=True)
    experts = torch.arange(E + 1, device=e.device)
    start = torch.searchsorted(by, experts.expand(B, rows, E + 1).contiguous())
    at = torch.arange(N, device=e.device)
    occ = torch.empty_like(e).scatter_(2, order, at - start.gather(2, by))
    # the slots of each expert in ascending order, and how many copies go to those before it
    se, perm = torch.where(slot >= 0, slot, torch.full_like(slot, E)).sort(dim=1, stable=True)
    first = torch.searchsorted(se, experts.expand(B, E + 1).contiguous())
    share = X[:, s["rank0"]:s["rank0"] + rows].long().gather(2, perm[:, None].expand(B, rows, S))
    upto = share.cumsum(2)
    before = torch.cat([torch.zeros_like(upto[..., :1]), upto], 2).gather(2, first[:, None].expand(B, rows, E + 1))
    idx = torch.searchsorted(upto, before.gather(2, e) + occ, right=True)
    guest = idx < first[:, None].expand(B, rows, E + 1).gather(2, e + 1)
    # instances in send order: rank by rank, its own experts, then its guest slots
    ranked = home.sort(dim=0, stable=True)
    own_at = torch.empty_like(home).scatter_(0, ranked.indices, torch.arange(E, device=e.device)) + K * home
    upto_rank = torch.searchsorted(ranked.values, torch.arange(R + 1, device=e.device))
    s_all = torch.arange(S, device=e.device)
    guest_at = s_all + upto_rank[s_all // K + 1]
    chosen = perm[:, None].expand(B, rows, S).gather(2, idx.clamp(max=S - 1))
    inst = torch.where(guest, guest_at[chosen], own_at[e])
    by, order = inst.sort(dim=2, stable=True)
    pos = torch.empty_like(inst).scatter_(2, order, at.expand(B, rows, N))
    every = torch.arange(E + S + 1, device=e.device)
    offsets = torch.searchsorted(by, every.expand(B, rows, E + S + 1).contiguous())
    edge = offsets[..., upto_rank + K * torch.arange(R + 1, device=e.device)]
    return [pos.int(), offsets.int(), (edge[..., 1:] - edge[..., :-1]).int()]


def _gathered(s):
    """Rows of y in the tokens' order, [rows][tokens][k][H] in 32 bits."""
    y, pos, c = s["y"], s["pos"].long(), s["case"]
    row = torch.arange(c["rows"], device=pos.device)[:, None]
    return y[row, pos].float().view(c["rows"], c["tokens"], c["k"], c["H"])


def _spread(x, pos, k):
    """out[row][pos[i]] = x[row][i / k]."""
    rows, N = pos.shape
    src = torch.empty_like(pos, dtype=torch.int64).scatter_(1, pos.long(), torch.arange(N, device=pos.device).expand(rows, N))
    return x[torch.arange(rows, device=pos.device)[:, None], src // k]


def _plain_rows(s):
    k = s["case"]["k"]
    return [_spread(s["x"].view(torch.uint8), s["pos"], k).view(torch.float8_e4m3fn), _spread(s["scale"], s["pos"], k)]


def _plain_combine(s):
    c = s["case"]
    w = s["weights"].view(c["rows"], c["tokens"], c["k"], 1)
    return (w * _gathered(s)).sum(2).to(s["y"].dtype)


def _plain_combine_bwd(s):
    c = s["case"]
    d = s["dout"].float()[:, :, None, :]
    w = s["weights"].view(c["rows"], c["tokens"], c["k"], 1)
    dw = (d * _gathered(s)).sum(3).view(c["rows"], -1)
    at = s["pos"].long()[:, :, None].expand(-1, -1, c["H"])
    dy = torch.empty_like(s["y"], dtype=torch.float32).scatter_(1, at, (w * d).reshape(c["rows"], -1, c["H"]))
    return [dy.to(s["y"].dtype), dw]


# ---- the definitions in 64 bits ----------------------------------------------

def exact(case, seed):
    c = case
    if c["kind"] == "map":
        return None  # whole numbers
    s = prepare(c, seed)
    f64 = {n: v.double() for n, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if c["kind"] == "norm":
        h = f64["x"] + f64["residual"] if c["residual"] else f64["x"]
        rstd = (h.pow(2).sum(1) / c["H"] + 1e-6).pow(-0.5)
        y = f64["weight"] * h * rstd[:, None]
        G = c["group"] or c["H"]
        part = [y[:, lo:lo + G] for lo in range(0, c["H"], G)]
        scale = torch.stack([p.abs().max(1).values for p in part], 1) / F8_MAX
        q = torch.cat([p / scale[:, i:i + 1] for i, p in enumerate(part)], 1)
        return [y, q, scale, rstd, h if c["residual"] else None]
    if c["kind"] == "norm_bwd":
        h, rstd, dy = f64["h"], f64["rstd"][:, None], f64["dy"]
        n = h * rstd
        dn = dy * f64["weight"]
        dx = rstd * (dn - n * (dn * n).sum(1, keepdim=True) / c["H"])
        return [dx + f64["dh"] if c["residual"] else dx, (dy * n).sum(0)]
    if c["kind"] == "route":
        x = f64["logits"]
        p = torch.sigmoid(x) if c["sigmoid"] else torch.softmax(x, 1)
        key = p + f64["bias"] if c["bias"] else p
        if c["groups"] > 1:
            g = key.view(c["T"], c["groups"], -1)
            best = g.topk(2 if c["two"] else 1, 2).values.sum(2)
            least = best.topk(c["top_groups"], 1).values[:, -1:]
            key = g.masked_fill((best < least)[:, :, None], -math.inf).view(c["T"], -1)
        w = p.gather(1, key.sort(dim=1, descending=True, stable=True).indices[:, :c["k"]])
        w = w / w.sum(1, keepdim=True) if c["renorm"] else w
        return [None, 2.5 * w]
    if c["kind"] == "route_bwd":
        x = f64["logits"].requires_grad_()
        w = (torch.sigmoid(x) if c["sigmoid"] else torch.softmax(x, 1)).gather(1, s["ids"].long())
        w = w / w.sum(1, keepdim=True) if c["renorm"] else w
        return torch.autograd.grad(2.5 * w, x, f64["dweights"])[0]
    rows, tokens, k, H = c["rows"], c["tokens"], c["k"], c["H"]
    token = torch.arange(tokens * k, device="cuda") // k
    if c["kind"] == "rows":
        out, sc = torch.empty_like(f64["x"].repeat(1, k, 1)), torch.empty_like(f64["scale"].repeat(1, k, 1))
        for r in range(rows):
            out[r, s["pos"][r].long()] = f64["x"][r, token]
            sc[r, s["pos"][r].long()] = f64["scale"][r, token]
        return [out, sc]
    y, pos = f64["y"], s["pos"].long().view(rows, tokens, k)
    w = f64["weights"].view(rows, tokens, k, 1)
    if c["kind"] == "combine":
        out = torch.zeros((rows, tokens, H), dtype=torch.float64, device="cuda")
        for r in range(rows):
            for j in range(k):
                out[r] += w[r, :, j] * y[r, pos[r, :, j]]
        return out
    dy, dw = torch.empty_like(y), torch.empty((rows, tokens, k), dtype=torch.float64, device="cuda")
    for r in range(rows):
        for j in range(k):
            dy[r, pos[r, :, j]] = w[r, :, j] * f64["dout"][r]
            dw[r, :, j] = (f64["dout"][r] * y[r, pos[r, :, j]]).sum(1)
    return [dy, dw.view(rows, -1)]


def work(case):
    """Each input read once, each output written once; sums, products and exponentials as operations."""
    c = case
    kind = c["kind"]
    z = SIZE.get(c.get("dtype"), 1)
    if kind == "norm":
        n = c["T"] * c["H"]
        r = 2 * n * z if c["residual"] else 0
        return {"bytes": 2 * n * z + r + n + 4 * c["T"] * (1 + -(-c["H"] // (c["group"] or c["H"]))) + c["H"] * z, "flops": 8 * n}
    if kind == "norm_bwd":
        n = c["T"] * c["H"]
        return {"bytes": n * z * (4 if c["residual"] else 3) + 4 * c["T"] + c["H"] * (z + 4), "flops": 12 * n}
    if kind == "route":
        n = c["T"] * c["E"]
        return {"bytes": n * z + 8 * c["T"] * c["k"], "flops": 4 * n}
    if kind == "route_bwd":
        n = c["T"] * c["E"]
        dense = not c["sigmoid"] and not c["renorm"]  # else only the chosen logits matter
        return {"bytes": n * z * (2 if dense else 1) + c["T"] * c["k"] * (8 if dense else 8 + z), "flops": 6 * n}
    if kind == "map":
        rows, S = c["B"] * c["rows"], c["R"] * c["K"]
        return {"bytes": rows * (8 * c["tokens"] * c["k"] + 4 * S + 4 * (c["E"] + S) + 4 * c["R"]) + 4 * (c["E"] + c["B"] * S), "flops": 0}
    n, N = c["rows"] * c["tokens"] * c["H"], c["rows"] * c["tokens"] * c["k"]
    if kind == "rows":
        g = 4 * c["rows"] * c["tokens"] * -(-c["H"] // c["group"])
        return {"bytes": (n + g) * (1 + c["k"]) + 4 * N, "flops": 0}
    if kind == "combine":
        return {"bytes": n * z * (1 + c["k"]) + 8 * N, "flops": 2 * n * c["k"]}
    return {"bytes": n * z * (1 + 2 * c["k"]) + 12 * N, "flops": 3 * n * c["k"]}
