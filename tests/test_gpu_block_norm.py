"""block_norm and its gradient against the formulas in 64 bits.

Tolerances.  U: half a step of the output's type, relative (f16 also 2^-25
absolute, below its normal range).  A row's sum of squares passes through at most
8 * 4 + 6 + 16 additions a value, all of one sign, so 1 / rms is within
60 * 2^-24 < 4e-6 of its value after the square root and the division; the
products behind it round at 2^-24 each.  The sum h is rounded relative to its
larger addend, and what is taken of it after (y, both gradients) carries that."""
import pytest
import torch

import paper_2608_03676_amd as taot

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LOW = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
TYPES = [torch.bfloat16, torch.float16, torch.float32]
FP = 4e-6
E = 2.0 ** -24


def _case(gpu, T, H, dtype, post=True, gates=1, weight=True, wide=None, gate_wide=None, seed=0):
    g = torch.Generator().manual_seed(seed + 7919 * T + H)

    def new(*shape, to=dtype, scale=1.0, shift=0.0):
        return (shift + scale * torch.randn(shape, generator=g)).to(to).to(gpu)

    c = dict(x=new(T, H), residual=new(T, H, scale=2.0), dy=new(T, H), dh=new(T, H), weight=None, post=None, gate=None)
    if weight:
        c["weight"] = new(H, to=wide or dtype, scale=0.3, shift=1.0)
    if post:
        c["post"] = new(H, to=wide or dtype, scale=0.3, shift=0.7)
    if gates:
        c["gate"] = new(gates, H, to=gate_wide or dtype, scale=0.5)
    return c


def _wide(c):
    return {n: None if v is None else v.double() for n, v in c.items()}


def _rows(gate, T):
    return 1.0 if gate is None else gate.repeat_interleave(T // gate.shape[0], 0)


def _forward(c, eps, alpha):
    d = _wide(c)
    x, T = d["x"], c["x"].shape[0]
    a, n = None, x
    if c["post"] is not None:
        a = (x.square().mean(1) + eps).rsqrt()
        n = x * a[:, None] * d["post"]
    n = n * _rows(d["gate"], T)
    h = alpha * d["residual"] + n
    size = abs(alpha) * d["residual"].abs() + n.abs()
    b = (h.square().mean(1) + eps).rsqrt()
    y = None if c["weight"] is None else h * b[:, None] * d["weight"]
    return a, h, size, b, y


def _check_forward(o, c, eps, alpha):
    dt = c["x"].dtype
    a, h, size, b, y = _forward(c, eps, alpha)
    off = (FP + 4 * E) * size  # of the sum in 32 bits: n carries a's error and three products'
    if a is not None:
        assert ((o.rstd_x.double() - a).abs() <= FP * a).all()
    assert ((o.h.double() - h).abs() <= U[dt] * h.abs() + LOW[dt] + off * (1 + U[dt])).all()
    if y is None:
        assert o.y is None and o.rstd_h is None
        return
    # b: the sum of squares carries 2 sum |h| off
    slip = b ** 2 * (h.abs() * off).mean(1)
    assert ((o.rstd_h.double() - b).abs() <= (FP + slip) * b).all()
    w = c["weight"].double().abs()
    assert ((o.y.double() - y).abs() <= (U[dt] + FP + slip[:, None]) * y.abs() + LOW[dt]
            + off * b[:, None] * w * (1 + U[dt])).all()


WIDTHS = [(1, 1), (3, 7), (5, 8), (2, 9), (4, 100), (3, 512), (3, 513), (4, 2048), (3, 5003), (2, 8192), (2, 8193),
          (2, 16400), (2, 32768)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H", WIDTHS)
def test_forward(gpu, dtype, T, H):
    print(f"[block norm] {dtype} {T} x {H}", flush=True)
    for post, gates, weight, alpha in ((True, 1, True, 1.0), (False, 0, True, 0.5), (True, T, False, -2.0),
                                       (False, T, True, 1.0), (True, 0, True, 0.0)):
        c = _case(gpu, T, H, dtype, post, gates, weight)
        o = taot.block_norm(c["x"], c["residual"], c["weight"], 1e-6, post=c["post"], gate=c["gate"], alpha=alpha)
        _check_forward(o, c, 1e-6, alpha)


@pytest.mark.parametrize("T,H,gates", [(4100, 64, 4), (4098, 520, 3), (4096, 4104, 4096), (600, 1031, 30)])
def test_forward_many_rows(gpu, T, H, gates):
    c = _case(gpu, T, H, torch.bfloat16, gates=gates, wide=torch.float32, gate_wide=torch.float32)
    o = taot.block_norm(c["x"], c["residual"], c["weight"], 1e-5, post=c["post"], gate=c["gate"], alpha=1.0)
    _check_forward(o, c, 1e-5, 1.0)


def _backward(c, h, a, b, alpha):
    """Gradients of the formulas, and for each a sum of the magnitudes of what it is made of."""
    d = _wide(c)
    x, T, H = d["x"], *c["x"].shape
    g = _rows(d["gate"], T)
    D, size, dw, dw_size = torch.zeros_like(x), torch.zeros_like(x), None, None
    if c["weight"] is not None:
        h, b = h.double(), b.double()[:, None]
        u = d["dy"] * d["weight"]
        D = b * (u - h * (b * b * (u * h).mean(1, keepdim=True)))
        # the mean's terms are of either sign: its error is relative to their magnitudes
        size = b * (u.abs() + h.abs() * (b * b * (u * h).abs().mean(1, keepdim=True)))
        dw, dw_size = (d["dy"] * h * b).sum(0), (d["dy"] * h * b).abs().sum(0)
    if c["dh"] is not None:
        D, size = D + d["dh"], size + d["dh"].abs()
    t, t_size = g * D, abs(g) * size
    n, S = x, None
    dx, dx_size = t, t_size
    dpost = dgate = None
    if c["post"] is not None:
        a = a.double()[:, None]
        S = x * a
        n = S * d["post"]
        dpost = ((t * S).sum(0), (t_size * S.abs()).sum(0))
        p, p_size = t * d["post"], t_size * d["post"].abs()
        dx = a * (p - x * (a * a * (p * x).mean(1, keepdim=True)))
        dx_size = a * (p_size + x.abs() * (a * a * (p_size * x.abs()).mean(1, keepdim=True)))
    if c["gate"] is not None:
        k = c["gate"].shape[0]
        dgate = ((D * n).view(k, -1, H).sum(1), (size * n.abs()).view(k, -1, H).sum(1))
    return dict(dx=(dx, dx_size), dresidual=(alpha * D, abs(alpha) * size), dweight=(dw, dw_size), dpost=dpost, dgate=dgate)


def _check_backward(got, c, o, alpha):
    """A row's result is of sums of at most 54 additions and ten operations, twice over: 150 E relative to the terms.
    A sum over T rows: a worker's rows one after the other (16 waves and 256 units share T), then 32 threads and theirs."""
    dt = c["x"].dtype
    T = c["x"].shape[0]
    want = _backward(c, o.h, o.rstd_x, o.rstd_h, alpha)
    for name, w in want.items():
        v = getattr(got, name)
        if w is None or w[0] is None:
            assert v is None, name
            continue
        ref, size = w
        v = v.double().view(ref.shape)
        if name in ("dx", "dresidual"):
            assert ((v - ref).abs() <= U[dt] * ref.abs() + LOW[dt] + 150 * E * size).all(), name
        else:
            adds = T / 256 + 4096 / 32 + 64
            assert ((v - ref).abs() <= (150 + adds) * E * size).all(), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H", WIDTHS + [(600, 64), (520, 2049), (4098, 40)])
def test_backward(gpu, dtype, T, H):
    print(f"[block norm backward] {dtype} {T} x {H}", flush=True)
    for post, gates, weight, dh, alpha in ((True, 1, True, True, 1.0), (False, 0, True, False, 0.5),
                                           (True, T, False, True, -2.0), (False, T, True, True, 1.0),
                                           (True, 0, True, False, 1.0), (False, 1, False, True, 3.0)):
        c = _case(gpu, T, H, dtype, post, gates, weight)
        if not dh:
            c["dh"] = None
        o = taot.block_norm(c["x"], c["residual"], c["weight"], 1e-6, post=c["post"], gate=c["gate"], alpha=alpha)
        args = (c["dy"] if weight else None, c["x"], o.h if weight else None, o.rstd_h, c["weight"])
        kw = dict(rstd_x=o.rstd_x, post=c["post"], gate=c["gate"], alpha=alpha, dh=c["dh"])
        got = taot.block_norm_backward(*args, **kw)
        _check_backward(got, c, o, alpha)
        again = taot.block_norm_backward(*args, **kw)
        for f in ("dx", "dresidual", "dweight", "dpost", "dgate"):
            a, b = getattr(got, f), getattr(again, f)
            assert (a is None) == (b is None) and (a is None or torch.equal(a, b)), f


@pytest.mark.parametrize("T,H,gates", [(12, 64, 3), (4096, 100, 4), (4098, 520, 3), (900, 1031, 300), (1200, 4104, 600),
                                       (4097 * 2, 64, 4097), (4097, 40, 4097), (768, 8200, 256), (600, 8200, 300),
                                       (24, 9000, 2)])
def test_backward_of_gates(gpu, T, H, gates):
    print(f"[block norm backward] {T} x {H}, {gates} gates", flush=True)
    c = _case(gpu, T, H, torch.bfloat16, gates=gates, wide=torch.float32, gate_wide=torch.float32)
    for post in (True, False):
        c["post"] = c["post"] if post else None
        o = taot.block_norm(c["x"], c["residual"], c["weight"], 1e-6, post=c["post"], gate=c["gate"])
        got = taot.block_norm_backward(c["dy"], c["x"], o.h, o.rstd_h, c["weight"], rstd_x=o.rstd_x, post=c["post"],
                                       gate=c["gate"], dh=c["dh"])
        _check_backward(got, c, o, 1.0)


def test_against_differences(gpu):
    """The directional derivative of sum(p y + q h) in 64 bits by central differences (error about 1e-9 here)."""
    T, H, eps, alpha = 12, 130, 1e-5, 1.5
    c = _case(gpu, T, H, torch.float32, gates=3)
    o = taot.block_norm(c["x"], c["residual"], c["weight"], eps, post=c["post"], gate=c["gate"], alpha=alpha)
    got = taot.block_norm_backward(c["dy"], c["x"], o.h, o.rstd_h, c["weight"], rstd_x=o.rstd_x, post=c["post"],
                                   gate=c["gate"], alpha=alpha, dh=c["dh"])
    g = torch.Generator().manual_seed(3)
    v = {n: torch.randn(c[n].shape, generator=g).to(gpu) for n in ("x", "residual", "weight", "post", "gate")}

    def value(step):
        m = dict(_wide(c), **{n: c[n].double() + step * t.double() for n, t in v.items()})
        _, h, _, _, y = _forward(m, eps, alpha)
        return (c["dy"].double() * y + c["dh"].double() * h).sum()

    want = (value(1e-5) - value(-1e-5)) / 2e-5
    parts = [getattr(got, "d" + n).double() * t.double() for n, t in v.items()]
    assert abs(want - sum(p.sum() for p in parts)) <= 1e-5 * sum(p.abs().sum() for p in parts)


@pytest.mark.parametrize("dtype", TYPES)
def test_odd_addresses_and_in_place(gpu, dtype):
    def shifted(t):
        room = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
        room[1:] = t.reshape(-1)
        return room[1:].view(t.shape)

    c = _case(gpu, 40, 264, dtype, gates=4)
    want = taot.block_norm(c["x"], c["residual"], c["weight"], 1e-6, post=c["post"], gate=c["gate"])
    s = {n: shifted(v) for n, v in c.items()}
    assert s["x"].data_ptr() % 16 != 0
    o = taot.block_norm(s["x"], s["residual"], s["weight"], 1e-6, post=s["post"], gate=s["gate"],
                        out=taot.BlockNorm(h=s["residual"]))
    assert torch.equal(o.y, want.y) and o.h is s["residual"] and torch.equal(o.h, want.h)
    kw = dict(post=c["post"], gate=c["gate"])
    a = taot.block_norm_backward(c["dy"], c["x"], want.h, want.rstd_h, c["weight"], rstd_x=want.rstd_x, dh=c["dh"], **kw)
    b = taot.block_norm_backward(s["dy"], s["x"], o.h, o.rstd_h, s["weight"], rstd_x=o.rstd_x, post=s["post"],
                                 gate=s["gate"], dh=s["dh"], out=taot.BlockNormGrad(dx=s["x"], dresidual=s["dh"]))
    for f in ("dx", "dresidual", "dweight", "dpost", "dgate"):
        assert torch.equal(getattr(a, f), getattr(b, f)), f
    for H in (520, 9000):  # in place in the kernels that read a row ahead, and more than once
        c = _case(gpu, 600, H, dtype, gates=2)
        o = taot.block_norm(c["x"], c["residual"], c["weight"], 1e-6, post=c["post"], gate=c["gate"])
        args = dict(rstd_x=o.rstd_x, post=c["post"], gate=c["gate"], dh=c["dh"])
        a = taot.block_norm_backward(c["dy"], c["x"], o.h, o.rstd_h, c["weight"], **args)
        b = taot.block_norm_backward(c["dy"], c["x"], o.h, o.rstd_h, c["weight"], **args,
                                     out=taot.BlockNormGrad(dx=c["dy"], dresidual=c["dh"]))
        assert torch.equal(a.dx, b.dx) and torch.equal(a.dresidual, b.dresidual) and torch.equal(a.dgate, b.dgate)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H", [9, 513, 1025, 1031, 2049, 4097, 5003, 8191])
def test_odd_widths_in_place(gpu, dtype, H):  # the end of a row is read by two lanes, of two waves at some of these
    c = _case(gpu, 700, H, dtype, gates=700)
    for post in (None, c["post"]):
        args = (c["weight"], 1e-6)
        want = taot.block_norm(c["x"], c["residual"], *args, post=post, gate=c["gate"])
        for over in ("x", "residual"):
            v = {n: c[n].clone() for n in ("x", "residual")}
            o = taot.block_norm(v["x"], v["residual"], *args, post=post, gate=c["gate"], out=taot.BlockNorm(h=v[over]))
            assert torch.equal(o.h, want.h) and torch.equal(o.y, want.y)
        kw = dict(rstd_x=want.rstd_x, post=post, gate=c["gate"])
        a = taot.block_norm_backward(c["dy"], c["x"], want.h, want.rstd_h, c["weight"], dh=c["dh"], **kw)
        dy, dh = c["dy"].clone(), c["dh"].clone()
        b = taot.block_norm_backward(dy, c["x"], want.h, want.rstd_h, c["weight"], dh=dh, **kw,
                                     out=taot.BlockNormGrad(dx=dy, dresidual=dh))
        for f in ("dx", "dresidual", "dweight", "dgate"):
            assert torch.equal(getattr(a, f), getattr(b, f)), f


def test_shapes_of_gates_and_empty(gpu):
    c = _case(gpu, 24, 40, torch.float16, gates=4)
    flat = taot.block_norm(c["x"], c["residual"], c["weight"], 1e-6, post=c["post"], gate=c["gate"])
    x, r = c["x"].view(4, 6, 40), c["residual"].view(4, 6, 40)
    for gate in (c["gate"], c["gate"].view(4, 1, 40)):
        o = taot.block_norm(x, r, c["weight"], 1e-6, post=c["post"], gate=gate)
        assert o.y.shape == x.shape and o.rstd_x.shape == (4, 6) and torch.equal(o.y.view(24, 40), flat.y)
        d = taot.block_norm_backward(x, x, o.h, o.rstd_h, c["weight"], rstd_x=o.rstd_x, post=c["post"], gate=gate)
        assert d.dgate.shape == gate.shape
    one = taot.block_norm(x, r, c["weight"], 1e-6, gate=c["gate"][0].contiguous())
    assert torch.equal(one.y, taot.block_norm(x, r, c["weight"], 1e-6, gate=c["gate"][:1].expand(4, 40).contiguous()).y)
    for bad in (c["gate"][:3].contiguous(), torch.zeros(6, 40, device=gpu), torch.zeros(4, 3, 40, device=gpu),
                torch.zeros(41, device=gpu), torch.zeros((), device=gpu)):
        with pytest.raises(ValueError):
            taot.block_norm(x, r, c["weight"], 1e-6, gate=bad)
    with pytest.raises(ValueError):  # 5 gates do not divide 24 rows
        taot.block_norm(c["x"], c["residual"], c["weight"], 1e-6, gate=torch.zeros(5, 40, device=gpu))
    e = c["x"][:0]
    o = taot.block_norm(e, e, c["weight"], 1e-6, post=c["post"], gate=c["gate"][0].contiguous())
    assert o.y.shape == (0, 40)
    d = taot.block_norm_backward(e, e, e, torch.empty(0, device=gpu), c["weight"], rstd_x=torch.empty(0, device=gpu),
                                 post=c["post"], gate=c["gate"][0].contiguous())
    assert not d.dweight.any() and not d.dpost.any() and not d.dgate.any()


def test_not_finite_rows_stay_by_themselves(gpu):
    c = _case(gpu, 5, 700, torch.float32)
    clean = taot.block_norm(c["x"], c["residual"], c["weight"], 1e-6, post=c["post"], gate=c["gate"])
    x = c["x"].clone()
    x[1, 3], x[3, 600] = float("nan"), float("inf")
    o = taot.block_norm(x, c["residual"], c["weight"], 1e-6, post=c["post"], gate=c["gate"])
    assert torch.isnan(o.y[1]).all() and torch.isnan(o.y[3]).all()
    assert torch.equal(o.y[[0, 2, 4]], clean.y[[0, 2, 4]])
    zero = torch.zeros_like(c["x"])
    o = taot.block_norm(zero, zero, c["weight"], 1e-6, post=c["post"], gate=c["gate"])
    assert not o.y.any() and not o.h.any()


def test_another_stream_and_a_result_used_again(gpu):
    c = _case(gpu, 300, 2048, torch.bfloat16)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    o = taot.block_norm(c["x"], c["residual"], c["weight"], 1e-6, post=c["post"], gate=c["gate"], stream=s)
    d = taot.block_norm_backward(c["dy"], c["x"], o.h, o.rstd_h, c["weight"], rstd_x=o.rstd_x, post=c["post"],
                                 gate=c["gate"], dh=c["dh"], stream=s)
    s.synchronize()
    _check_forward(o, c, 1e-6, 1.0)
    _check_backward(d, c, o, 1.0)
    y, h = o.y, o.h
    o = taot.block_norm(c["residual"], c["x"], c["weight"], 1e-6, out=o)
    assert o.y is y and o.h is h and o.rstd_x is None
    _check_forward(o, dict(c, x=c["residual"], residual=c["x"], post=None, gate=None), 1e-6, 1.0)


def test_refusals(gpu):
    c = _case(gpu, 4, 64, torch.bfloat16)
    x, r, w, p, g = (c[n] for n in ("x", "residual", "weight", "post", "gate"))
    with pytest.raises(TypeError):
        taot.block_norm(x.double(), r, w, 1e-6)
    with pytest.raises(TypeError):
        taot.block_norm(x, r.float(), w, 1e-6)
    with pytest.raises(TypeError):  # vectors of two types
        taot.block_norm(x, r, w.float(), 1e-6, post=p)
    with pytest.raises(TypeError):
        taot.block_norm(x, r, w, 1e-6, gate=g.half())
    with pytest.raises(ValueError):
        taot.block_norm(x, r[:2], w, 1e-6)
    with pytest.raises(ValueError):
        taot.block_norm(x.t(), r, w, 1e-6)
    for eps, alpha in ((-1.0, 1.0), (float("nan"), 1.0), (1e-6, float("inf"))):
        with pytest.raises(taot.TaotError):
            taot.block_norm(x, r, w, eps, alpha=alpha)
    one = torch.ones(4, device=gpu)
    with pytest.raises(ValueError):
        taot.block_norm_backward(None, x, None, None, None)
    with pytest.raises(TypeError):
        taot.block_norm_backward(x, x, x, None, w)
    with pytest.raises(ValueError):
        taot.block_norm_backward(x, x, x, one, w, rstd_x=one)
    with pytest.raises(TypeError):
        taot.block_norm_backward(x, x, x, one, w, post=p)
    with pytest.raises(taot.TaotError) as e:
        taot.block_norm_backward(x, x, x, one, w, workspace=torch.empty(8, dtype=torch.uint8, device=gpu))
    assert e.value.code == 3
    with pytest.raises(RuntimeError, match="gate"):
        taot.block_norm(x, r, w, 1e-6, gate=g.clone().requires_grad_())
