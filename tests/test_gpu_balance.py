"""balance_loss and its gradient against the formulas in 64 bits.

Tolerances, E = 2^-24.  A softmax score is an exponential of a difference that is
rounded (E times its magnitude, at most the logits' span R), over a sum of at most
60 additions of one sign: within (R + 64) E of its value.  Sums over tokens are of
one sign too and add at most their number of additions."""
import pytest
import torch

import paper_2608_03676_amd as taot

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LOW = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
TYPES = [torch.bfloat16, torch.float16, torch.float32]
SIGMOID = taot.ROUTE_SIGMOID


def _case(gpu, rows, tokens, experts, k, dtype, masked=False, seed=0):
    g = torch.Generator().manual_seed(seed + 31 * tokens + experts)
    x = (1.5 * torch.randn(rows, tokens, experts, generator=g) + torch.randn(experts, generator=g)).to(dtype)
    ids = torch.randint(-1, experts + 1, (rows, tokens, k), generator=g).int()  # some are no expert
    mask = torch.rand(rows, tokens, generator=g) < 0.7 if masked else None
    return x.to(gpu), ids.to(gpu), None if mask is None else mask.to(gpu)


def _scores(x, sigmoid):
    """(p, log-sum-exp) in 64 bits, of the definition's values for what is not finite."""
    x = torch.where(torch.isnan(x), torch.full_like(x, float("-inf")), x.clamp(max=torch.finfo(torch.float32).max))
    if sigmoid:
        s = torch.sigmoid(x)
        return s / (s.sum(-1, keepdim=True) + 1e-20), torch.zeros_like(x[..., 0])
    lse = torch.logsumexp(x, -1)
    none = torch.isinf(lse)
    return torch.where(none[..., None], torch.zeros_like(x), torch.softmax(x, -1)), torch.where(none, torch.zeros_like(lse), lse)


def _reference(x, ids, mask, sigmoid):
    rows, tokens, n = x.shape
    p, lse = _scores(x.double(), sigmoid)
    keep = torch.ones((rows, tokens), device=x.device).double() if mask is None else mask.double()
    count = keep.sum(1)
    each = count.clamp(min=1)
    hits = torch.stack([torch.bincount(i[(i >= 0) & (i < n)].long(), minlength=n) for i in
                        (ids[r][keep[r] > 0] for r in range(rows))])
    prob = (p * keep[..., None]).sum(1) / each[:, None]
    loss = n * (hits.double() * prob).sum(1) / hits.sum(1).clamp(min=1)
    return loss, (lse.square() * keep).sum(1) / each, hits, prob, count, lse, keep


def _check(b, x, ids, mask, sigmoid):
    loss, z, hits, prob, count, lse, keep = _reference(x, ids, mask, sigmoid)
    n, tokens = x.shape[2], x.shape[1]
    fine = x.float()[torch.isfinite(x)]
    R = float(fine.max() - fine.min()) if fine.numel() else 0.0
    assert torch.equal(b.counts.long(), hits) and torch.equal(b.tokens.double(), count)
    tol = (R + 64 + tokens) * E
    assert ((b.prob.double() - prob).abs() <= tol * prob).all()
    assert ((b.loss.double() - loss).abs() <= (tol + (n / 256 + 16) * E) * loss).all()
    if sigmoid:
        assert b.z is None
        return
    slip = E * (R + 64 + 3 * lse.abs())
    assert ((b.z.double() - z).abs() <= (2 * lse.abs() * slip * keep).sum(1) / count.clamp(min=1) + (tokens + 16) * E * z).all()


SHAPES = [(1, 1, 1, 1), (2, 3, 7, 2), (1, 17, 128, 8), (3, 100, 129, 8), (1, 1000, 256, 8), (2, 77, 257, 6), (1, 500, 512, 4),
          (1, 33, 513, 8), (2, 40, 1024, 8), (1, 50, 1030, 2), (1, 31, 2048, 8), (2, 9, 2049, 8), (1, 20, 4096, 8),
          (1, 5, 8193, 3), (1, 3, 20000, 64), (1, 2, 32768, 8)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(gpu, dtype, shape):
    print(f"[balance] {dtype} {shape}", flush=True)
    for masked in (False, True):
        for flags in (0, SIGMOID):
            x, ids, mask = _case(gpu, *shape, dtype, masked)
            b = taot.balance_loss(x, ids, mask=mask, flags=flags)
            _check(b, x, ids, mask, flags != 0)
            again = taot.balance_loss(x, ids, mask=None if mask is None else mask.byte(), flags=flags)
            assert torch.equal(b.loss, again.loss) and torch.equal(b.prob, again.prob)


def test_many_tokens_and_many_rows(gpu):
    for shape in ((1, 70000, 64, 8), (4, 8191, 160, 8), (3000, 5, 16, 2), (2049, 1, 40, 2)):
        x, ids, mask = _case(gpu, *shape, torch.bfloat16, True)
        _check(taot.balance_loss(x, ids, mask=mask), x, ids, mask, False)


def _grad_check(got, x, ids, counts, tokens, mask, dloss, dz, add, sigmoid):
    rows, T, n = x.shape
    p, lse = _scores(x.double(), sigmoid)
    a = (dloss.double() * n / (counts.sum(1).clamp(min=1) * tokens.clamp(min=1)))[:, None, None] * counts[:, None, :].double()
    dot, dot_size = (a * p).sum(-1, keepdim=True), (a.abs() * p).sum(-1, keepdim=True)
    fine = x.float()[torch.isfinite(x)]
    R = float(fine.max() - fine.min())
    if sigmoid:
        v = torch.nan_to_num(torch.sigmoid(x.double()), nan=0.0)
        V = v.sum(-1, keepdim=True) + 1e-20
        dx, size = (a - dot) / V * v * (1 - v), (a.abs() + dot_size) / V * v  # 1 - v is off by E times 1, not times itself
    else:
        up = 0.0 if dz is None else (2 * dz.double() / tokens.clamp(min=1))[:, None, None] * lse[..., None]
        dx, size = p * (a - dot + up), p * (a.abs() + dot_size + (0.0 if dz is None else up.abs()))
    keep = torch.ones((rows, T, 1), device=x.device).double() if mask is None else mask.double()[..., None]
    dx, size = dx * keep, size * keep
    if add is not None:
        dx, size = dx + add.double(), size + add.double().abs() * 2.0 ** -6  # one addition of them: E, of 64 E here
    dt = x.dtype
    # twice a score's error, the dot product's 60 additions, a dozen operations
    assert ((got.double() - dx).abs() <= U[dt] * dx.abs() + LOW[dt] + (2 * R + 256) * E * size).all()
    if add is not None and mask is not None:
        assert torch.equal(got[~mask], add[~mask])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(gpu, dtype, shape):
    print(f"[balance backward] {dtype} {shape}", flush=True)
    for masked, added, flags in ((False, False, 0), (True, True, 0), (True, False, SIGMOID), (False, True, SIGMOID)):
        x, ids, mask = _case(gpu, *shape, dtype, masked, seed=1)
        b = taot.balance_loss(x, ids, mask=mask, flags=flags)
        g = torch.Generator().manual_seed(4)
        dloss, dz = ((0.5 + torch.rand(shape[0], generator=g)).to(gpu) * shape[1] for _ in range(2))
        dz = None if flags else dz
        add = (torch.randn(x.shape, generator=g) / shape[2]).to(dtype).to(gpu) if added else None
        got = taot.balance_loss_backward(dloss, x, b.counts, b.tokens, mask=mask, dz=dz, add=add, flags=flags)
        _grad_check(got, x, ids, b.counts.double(), b.tokens.double(), mask, dloss, dz, add, flags != 0)
        for into in (x.clone(), None if add is None else add.clone()):  # in place
            if into is not None:
                y = into if add is None or not torch.equal(into, add) else x
                z = into if add is not None and torch.equal(into, add) else add
                r = taot.balance_loss_backward(dloss, y, b.counts, b.tokens, mask=mask, dz=dz, add=z, flags=flags, out=into)
                assert r is into and torch.equal(r, got)


# A token's experts in two lanes (to 16), eight (to 64) or more; rows of few and of many blocks.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 70001, 16, 2), (3, 4000, 9, 1), (2, 3001, 33, 4), (5, 2000, 64, 8), (2, 9000, 8, 2),
                                   (9, 600, 17, 3), (32, 128, 4096, 8), (40, 70, 65, 8)])
def test_few_experts_and_many_blocks(gpu, dtype, shape):
    print(f"[balance] {dtype} {shape}", flush=True)
    x, ids, mask = _case(gpu, *shape, dtype, True)
    for flags in (0, SIGMOID):
        b = taot.balance_loss(x, ids, mask=mask, flags=flags)
        _check(b, x, ids, mask, flags != 0)
        g = torch.Generator(device=gpu).manual_seed(3)
        dloss, dz = (torch.randn(shape[0], device=gpu, generator=g) for _ in range(2))
        add = torch.randn(x.shape, device=gpu, generator=g).to(dtype)
        dz = None if flags else dz
        got = taot.balance_loss_backward(dloss, x, b.counts, b.tokens, mask=mask, dz=dz, add=add, flags=flags)
        _grad_check(got, x, ids, b.counts, b.tokens, mask, dloss, dz, add, flags != 0)


@pytest.mark.parametrize("flags", [0, SIGMOID])
def test_against_differences(gpu, flags):
    """The loss's directional derivative in 64 bits by central differences (error about 1e-9 here)."""
    x, ids, mask = _case(gpu, 2, 30, 40, 4, torch.float32, True)
    b = taot.balance_loss(x, ids, mask=mask, flags=flags)
    g = torch.Generator().manual_seed(9)
    dloss, dz = (torch.randn(2, generator=g).to(gpu) for _ in range(2))
    v = torch.randn(x.shape, generator=g).to(gpu).double()
    got = taot.balance_loss_backward(dloss, x, b.counts, b.tokens, mask=mask, dz=None if flags else dz, flags=flags).double()

    def value(step):
        loss, z, *_ = _reference(x.double() + step * v, ids, mask, flags != 0)
        return (loss * dloss.double()).sum() + (0 if flags else (z * dz.double()).sum())

    want = (value(1e-5) - value(-1e-5)) / 2e-5
    assert abs(want - (got * v).sum()) <= 1e-5 * (got * v).abs().sum()


def test_even_choices_have_a_loss_of_one(gpu):
    x = torch.zeros(1, 64, 16, device=gpu)
    ids = (torch.arange(64 * 2, device=gpu) % 16).int().view(1, 64, 2)
    b = taot.balance_loss(x, ids)
    assert abs(float(b.loss) - 1) < 64 * E and (b.counts == 8).all()
    one = taot.balance_loss(x[0], torch.zeros_like(ids[0]))  # a single set of tokens; all of them at one expert
    assert one.loss.shape == () and abs(float(one.loss) - 1) < 64 * E and int(one.counts[0]) == 128


@pytest.mark.parametrize("flags", [0, SIGMOID])
@pytest.mark.parametrize("experts", [16, 600, 3000])
def test_masked_experts_and_what_is_not_finite(gpu, flags, experts):
    x, ids, _ = _case(gpu, 2, 20, experts, 2, torch.float32)
    x[0, 3, 1:] = float("-inf")       # one expert left
    x[0, 4] = float("-inf")           # none left
    x[0, 5, 2] = float("nan")
    x[1, 6, :3] = float("-inf")
    x[1, 7] = torch.finfo(torch.float32).min  # masked by the type's lowest value: all alike
    x[1, 8, 5] = torch.finfo(torch.float32).min
    b = taot.balance_loss(x, ids, flags=flags)
    assert torch.isfinite(b.loss).all() and torch.isfinite(b.prob).all()
    y = x.clone()
    y[1, 7] = 0.0  # the same scores of a softmax; its logarithm is not
    p = _reference(x if flags else y, ids, None, flags != 0)[3]
    span = 2 * float(x[torch.isfinite(x) & (x.abs() < 1e30)].abs().max()) + 90
    assert ((b.prob.double() - p).abs() <= (span + 84) * E * p + 2.0 ** -126).all()
    got = taot.balance_loss_backward(torch.ones(2, device=gpu), x, b.counts, b.tokens, flags=flags)
    assert torch.isfinite(got).all() and not got[0, 4].any() and not got[0, 5, 2].any() and not got[1, 6, :3].any()
    x[0, 9, 4] = float("inf")
    p = taot.balance_loss(x[:, 9:10].contiguous(), ids[:, 9:10].contiguous(), flags=flags).prob
    assert torch.isfinite(p).all() and (flags or (p[0, 4] == 1 and p[0].sum() == 1))


def test_no_tokens(gpu):
    x, ids, _ = _case(gpu, 2, 6, 32, 2, torch.bfloat16)
    none = torch.zeros(2, 6, dtype=torch.bool, device=gpu)
    b = taot.balance_loss(x, ids, mask=none)
    assert not b.loss.any() and not b.z.any() and not b.counts.any() and not b.prob.any() and not b.tokens.any()
    d = taot.balance_loss_backward(torch.ones(2, device=gpu), x, b.counts, b.tokens, mask=none)
    assert not d.any()
    b = taot.balance_loss(x[:, :0].contiguous(), ids[:, :0].contiguous())
    assert not b.loss.any() and not b.counts.any() and b.counts.shape == (2, 32)
    assert taot.balance_loss_backward(torch.ones(2, device=gpu), x[:, :0].contiguous(), b.counts, b.tokens).shape == (2, 0, 32)
    b = taot.balance_loss(x[:0], ids[:0])
    assert b.loss.shape == (0,) and b.counts.shape == (0, 32)


def test_counts_of_several_ranks(gpu):
    """Gradients with the choices of all ranks are those of one rank that has all tokens, where dloss is scaled by a rank's
    share of them; bfloat16 results of sums in other orders are equal but for a step."""
    x, ids, _ = _case(gpu, 1, 64, 48, 4, torch.float32)
    whole = taot.balance_loss(x, ids)
    one = torch.ones(1, device=gpu)
    want = taot.balance_loss_backward(one, x, whole.counts, whole.tokens)
    for half in (slice(0, 32), slice(32, 64)):
        part = x[:, half].contiguous()
        b = taot.balance_loss(part, ids[:, half].contiguous())
        got = taot.balance_loss_backward(0.5 * one, part, whole.counts, b.tokens)
        assert torch.allclose(got, want[:, half], rtol=8 * E, atol=0)


def test_another_stream(gpu):
    x, ids, mask = _case(gpu, 2, 3000, 256, 8, torch.bfloat16, True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    b = taot.balance_loss(x, ids, mask=mask, stream=s)
    d = taot.balance_loss_backward(torch.ones(2, device=gpu), x, b.counts, b.tokens, mask=mask, stream=s)
    s.synchronize()
    _check(b, x, ids, mask, False)
    _grad_check(d, x, ids, b.counts.double(), b.tokens.double(), mask, torch.ones(2, device=gpu), None, None, False)


def test_refusals(gpu):
    x, ids, mask = _case(gpu, 2, 6, 32, 2, torch.bfloat16, True)
    b = taot.balance_loss(x, ids)
    one = torch.ones(2, device=gpu)
    with pytest.raises(TypeError):
        taot.balance_loss(x.double(), ids)
    with pytest.raises(TypeError):
        taot.balance_loss(x, ids.long())
    with pytest.raises(TypeError):
        taot.balance_loss(x, None)
    with pytest.raises(TypeError):
        taot.balance_loss(x, ids, mask=mask.float())
    for call in (lambda: taot.balance_loss(x[0, 0], ids[0, 0]), lambda: taot.balance_loss(x, ids[:1]),
                 lambda: taot.balance_loss(x, ids, mask=mask[:, :3]), lambda: taot.balance_loss(x.transpose(0, 1), ids),
                 lambda: taot.balance_loss_backward(one[:1], x, b.counts, b.tokens),
                 lambda: taot.balance_loss_backward(one, x, b.counts[:, :5].contiguous(), b.tokens),
                 lambda: taot.balance_loss_backward(one, x, b.counts, b.tokens, add=x[:1])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: taot.balance_loss(x, ids, flags=taot.ROUTE_RENORM), lambda: taot.balance_loss(x, ids[..., :0].contiguous()),
                 lambda: taot.balance_loss_backward(one, x, b.counts, b.tokens, dz=one, flags=SIGMOID)):
        with pytest.raises(taot.TaotError) as e:
            call()
        assert e.value.code == 1
    with pytest.raises(taot.TaotError) as e:
        taot.balance_loss(x, ids, workspace=torch.empty(8, dtype=torch.uint8, device=gpu))
    assert e.value.code == 3
    with pytest.raises(RuntimeError, match="logits"):
        taot.balance_loss(x.clone().requires_grad_(), ids)
