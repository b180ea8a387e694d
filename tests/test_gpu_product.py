"""quantize_rows and matmul_i8 against their definitions in 64 bits.

Tolerances, E = 2^-24: a scale is of one division and one product (4 E with the
maximum's own rounding; a gated value carries 12 E); a quotient lands on the nearest
integer, or where it is within its own error of a half on the other.  A product's
sum is exact; its float, the two scales and the output's rounding are 3 E and half a
step U of the output's type (f16 also 2^-25 absolute)."""
import pytest
import torch

import paper_2608_03676_amd as taot

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LOW = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _shifted(t, by=1):
    room = torch.empty(t.numel() + by, dtype=t.dtype, device=t.device)
    room[by:] = t.reshape(-1)
    return room[by:].view(t.shape)


# ---- rows ----------------------------------------------------------------------

def _check_rows(q, scale, x, gated):
    v = x.double()
    if gated:
        g, u = v.chunk(2, -1)
        v = g * torch.sigmoid(g) * u
    off = (16 if gated else 4) * E
    a = v.abs().amax(-1, keepdim=True).clamp(min=1e-30)
    assert q.dtype == torch.int8 and scale.shape == (*x.shape[:-1], 1)
    assert ((scale.double() * 127 - a).abs() <= off * a).all()
    exact = v / a * 127
    assert ((q.double() - exact).abs() <= 0.5 + 2 * off * 127).all()
    assert q.abs().max() <= 127


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H", [(1, 1), (3, 7), (5, 8), (2, 9), (4, 100), (3, 512), (3, 513), (4, 2048), (3, 5003), (2, 8192),
                                 (2, 8193), (2, 16400), (2, 32768), (4100, 40)])
def test_rows(gpu, dtype, T, H):
    print(f"[rows] {dtype} {T} x {H}", flush=True)
    g = torch.Generator().manual_seed(T + H)
    for gated in (False, True):
        x = torch.randn(T, H * (1 + gated), generator=g).to(dtype).to(gpu)
        q, scale = taot.quantize_rows(x, gated=gated)
        _check_rows(q, scale, x, gated)
        s = taot.quantize_rows(_shifted(x), gated=gated, out=taot.Rows8(q=_shifted(q)))
        assert torch.equal(s.q, q) and torch.equal(s.scale, scale)
    x = torch.randn(T, H, generator=g).to(dtype).to(gpu)
    a = x.float().abs().amax(1, keepdim=True).clamp(min=1e-30)
    q, _ = taot.quantize_rows(x)  # the definition in 32 bits, bit for bit
    assert torch.equal(q, torch.round(x.float() * (torch.full_like(a, 127) / a)).to(torch.int8))


def test_rows_of_zeros_halves_and_what_is_not_finite(gpu):
    x = torch.zeros(6, 300, device=gpu)
    x[1, 0], x[1, 1:5] = 127.0, torch.tensor([0.5, 1.5, 2.5, -0.5], device=gpu)
    x[2, 299], x[2, 3] = float("inf"), 1.0
    x[3, 7] = float("nan")
    x[4, 5] = -1e-38
    x[5, 0], x[5, 1] = torch.finfo(torch.float32).max, -torch.finfo(torch.float32).max
    q, s = taot.quantize_rows(x)
    assert not q[0].any() and s[0] > 0 and s[0] < 1e-30
    assert q[1, :5].tolist() == [127, 0, 2, 2, 0] and s[1] == 1
    assert torch.isnan(s[2:4]).all() and not q[2:4].any()
    assert not q[4].any()  # below the floor
    assert q[5, :2].tolist() == [127, -127]
    e = taot.quantize_rows(x[:0])
    assert e.q.shape == (0, 300) and e.scale.shape == (0, 1)
    lead = taot.quantize_rows(x.view(2, 3, 300), gated=True)
    assert lead.q.shape == (2, 3, 150) and lead.scale.shape == (2, 3, 1)


# ---- products ------------------------------------------------------------------

def _integers(gpu, g, *shape):
    return torch.randint(-128, 128, shape, generator=g).to(torch.int8).to(gpu)


def _operands(gpu, M, N, K, G=None, seed=0):
    g = torch.Generator().manual_seed(seed + M + 3 * N + 7 * K)
    x = _integers(gpu, g, M, K)
    w = _integers(gpu, g, *((N, K) if G is None else (G, N, K)))
    sx = (0.5 + torch.rand(M, 1, generator=g)).to(gpu) * 0.01
    sw = (0.5 + torch.rand(w.shape[:-1], generator=g)).to(gpu) * 0.01
    return x, sx, w, sw


def _near(out, want):
    dt = out.dtype
    return bool(((out.double() - want).abs() <= (U[dt] + 4 * E) * want.abs() + LOW[dt]).all())


def _dense(x, sx, w, sw):
    return (x.double() @ w.double().t().contiguous()) * sx.double().view(-1, 1) * sw.double()


DENSE = [(1, 1, 1), (1, 3, 15), (2, 16, 16), (5, 17, 17), (16, 100, 127), (1, 2048, 2048), (16, 33, 2049), (3, 64, 5003),
         (17, 5, 31), (63, 129, 128), (64, 128, 129), (65, 130, 1000), (100, 257, 640), (127, 64, 64), (128, 256, 128),
         (129, 255, 257), (256, 512, 1024), (300, 300, 300), (511, 1, 100), (1000, 769, 333)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", DENSE)
def test_one_weight(gpu, dtype, M, N, K):
    print(f"[product] {dtype} {M} x {N} x {K}", flush=True)
    x, sx, w, sw = _operands(gpu, M, N, K)
    out = taot.matmul_i8(x, sx, w, sw, dtype=dtype)
    assert out.shape == (M, N) and out.dtype == dtype and _near(out, _dense(x, sx, w, sw))
    odd = taot.matmul_i8(_shifted(x, 3), _shifted(sx), _shifted(w, 5), _shifted(sw), dtype=dtype, out=_shifted(out))
    assert torch.equal(odd, out)


def test_the_largest_sums(gpu):
    """131071 terms of 2^14 each: one more would not fit 32 bits."""
    K = 131071
    for M in (1, 40, 130):
        x, w = torch.full((M, K), -128, dtype=torch.int8, device=gpu), torch.full((3, K), -128, dtype=torch.int8, device=gpu)
        out = taot.matmul_i8(x, torch.ones(M, device=gpu), w, torch.ones(3, device=gpu), dtype=torch.float32)
        assert (out == float(K << 14)).all()  # 2^31 - 2^14: 17 bits of value
    with pytest.raises(taot.TaotError) as e:
        x, w = (torch.zeros((1, K + 1), dtype=torch.int8, device=gpu) for _ in range(2))
        taot.matmul_i8(x, torch.ones(1, device=gpu), w, torch.ones(1, device=gpu))
    assert e.value.code == 2


def _runs(out, x, sx, w, sw, offsets, experts):
    """What the definition says of offsets and experts, run by run."""
    M, G = x.shape[0], w.shape[0]
    want = torch.zeros(out.shape, dtype=torch.float64, device=out.device)
    at = 0
    o = []
    for v in offsets:
        at = max(at, min(max(v, 0), M))
        o.append(at)
    for i in range(len(o) - 1):
        e = i if experts is None else experts[i]
        if 0 <= e < G and o[i] < o[i + 1]:
            r = slice(o[i], o[i + 1])
            want[r] = _dense(x[r], sx[r], w[e], sw[e])
    return want


def _grouped(gpu, M, N, K, G, offsets, experts=None, dtype=torch.bfloat16):
    x, sx, w, sw = _operands(gpu, M, N, K, G)
    out = torch.full((M, N), 7.0, dtype=dtype, device=gpu)
    taot.matmul_i8(x, sx, w, sw, offsets=torch.tensor(offsets, dtype=torch.int32, device=gpu),
                   experts=None if experts is None else torch.tensor(experts, dtype=torch.int32, device=gpu), out=out, dtype=dtype)
    assert _near(out, _runs(out, x, sx, w, sw, offsets, experts))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,N", [(128, 64), (1003, 259), (33, 300)])
def test_runs(gpu, dtype, K, N):
    print(f"[runs] {dtype} K {K} N {N}", flush=True)
    _grouped(gpu, 40, N, K, 4, [0, 1, 1, 30, 40], dtype=dtype)                       # empty, one row, all up to the end
    _grouped(gpu, 40, N, K, 4, [3, 10, 17, 17, 25], dtype=dtype)                     # rows of no run before and behind
    _grouped(gpu, 300, N, K, 3, [0, 64, 129, 129, 200, 290], [2, 0, 1, 2, 2], dtype)  # a weight twice, tiles that end inside
    _grouped(gpu, 1000, N, K, 2, [0, 257, 800, 801], [1, 0, 1], dtype)
    _grouped(gpu, 700, N, K, 3, [0, 256, 512, 700], [1, -1, 0], dtype)               # a run of no expert
    _grouped(gpu, 50, N, K, 2, [0, 20, 50], [2, 1], dtype)                           # an expert that is none
    _grouped(gpu, 5, N, K, 1, [0, 5], None, dtype)


def test_offsets_that_are_wrong(gpu):
    """Taken within [0, M] and each as at least the one before it: no row is read or written outside, none twice."""
    for M in (40, 600):
        _grouped(gpu, M, 70, 100, 4, [-5, 10, 2 * M, 3, M])
        _grouped(gpu, M, 70, 100, 4, [M, 30, 20, 10, 0])
        _grouped(gpu, M, 70, 100, 3, [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0])
        _grouped(gpu, M, 70, 100, 2, [0, 20, 10, 30, M], [0, 1, 0, 2 ** 31 - 1])


# Where rows begin at multiples of 16 bytes, pieces go straight to LDS: tiles of 128 by 128 from 48 rows a run on, and of
# 256 by 256 from 96 rows a run and 176 of them on.
@pytest.mark.parametrize("K", [16, 128, 144, 256, 272, 384, 400, 512, 528, 640, 768, 896, 1024, 2064])
def test_tiles_of_whole_pieces(gpu, K):
    print(f"[pieces] K {K}", flush=True)
    for M, N in ((48, 64), (128, 128), (129, 1000), (700, 300), (257, 2049), (6001, 2305)):
        x, sx, w, sw = _operands(gpu, M, N, K)
        for dtype in TYPES:
            out = torch.full((M + 1, N), 7.0, dtype=dtype, device=gpu)
            taot.matmul_i8(x, sx, w, sw, dtype=dtype, out=out[:M])
            assert _near(out[:M], _dense(x, sx, w, sw)) and (out[M] == 7).all(), (M, N)
            assert torch.equal(taot.matmul_i8(_shifted(x, 3), sx, _shifted(w, 5), sw, dtype=dtype), out[:M]), (M, N)
    _grouped(gpu, 1200, 260, K, 4, [0, 0, 5, 133, 300, 555, 811, 812, 940, 1190], [0, 3, -1, 2, 2, 4, 1, 0, 3])
    sizes = [0, 900, 1, 255, 256, 257, 512, 700, 3, 900]
    offsets = [7]
    for n in sizes:
        offsets.append(offsets[-1] + n)
    _grouped(gpu, offsets[-1] + 9, 3001, K, 3, offsets, [1, 0, 2, 1, -1, 2, 0, 3, 1, 2])


# Tiles of 256 by 256 by way of registers (from 96 of them and 64 rows a run on) where rows begin elsewhere.
@pytest.mark.parametrize("K", [16, 128, 144, 256, 400, 1024, 1, 17, 132, 333])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_tiles_of_many_rows(gpu, K, dtype):
    print(f"[large] {dtype} K {K}", flush=True)
    x, sx, w, sw = _operands(gpu, 4000, 1601, K)
    out = taot.matmul_i8(x, sx, w, sw, dtype=dtype)
    assert _near(out, _dense(x, sx, w, sw))
    assert torch.equal(taot.matmul_i8(_shifted(x, 3), sx, _shifted(w, 5), sw, dtype=dtype), out)
    g = torch.Generator().manual_seed(K)
    sizes = torch.randint(0, 200, (40,), generator=g)
    sizes[7], sizes[8], sizes[9] = 256, 257, 511
    offsets = [3] + (3 + sizes.cumsum(0)).tolist()
    experts = torch.randint(-1, 4, (40,), generator=g).tolist()
    _grouped(gpu, offsets[-1] + 30, 520, K, 3, offsets, experts, dtype)


# Tiles of 64 rows by 128 channels (from 129 of them on), and fewer, whose waves share the inner dimension.
@pytest.mark.parametrize("K", [4, 64, 128, 255, 256, 388, 1024, 1030, 2050, 1, 131])
def test_middling_runs(gpu, K):
    for M, N in ((2000, 600), (2001, 521), (100, 512), (33, 70)):
        for dtype in (torch.bfloat16, torch.float32):
            x, sx, w, sw = _operands(gpu, M, N, K)
            out = taot.matmul_i8(x, sx, w, sw, dtype=dtype)
            assert _near(out, _dense(x, sx, w, sw)), (M, N)
            assert torch.equal(taot.matmul_i8(_shifted(x, 1), sx, _shifted(w, 2), sw, dtype=dtype), out), (M, N)
    _grouped(gpu, 1250, 700, K, 24, [0, 466, 655, 767, 844, 901, 946, 984] + list(range(1000, 1170, 10)))
    _grouped(gpu, 300, 100, K, 2, [10, 150, 290], [1, 0])


def test_wrong_offsets_of_large_runs(gpu):
    M = 9000
    _grouped(gpu, M, 520, 48, 40, [-7, 300, 200, 5000, 4000, 10 ** 9, 5] + [6000 + 75 * i for i in range(34)])


@pytest.mark.parametrize("runs", [1022, 1023, 1024, 1025, 3000])
def test_many_runs(gpu, runs):
    g = torch.Generator().manual_seed(runs)
    sizes = torch.randint(0, 4, (runs,), generator=g)
    sizes[runs // 2] = 100
    offsets = [5] + (5 + sizes.cumsum(0)).tolist()
    _grouped(gpu, offsets[-1] + 3, 20, 48, 7, offsets, torch.randint(-1, 8, (runs,), generator=g).tolist())


def test_no_rows_and_no_runs(gpu):
    x, sx, w, sw = _operands(gpu, 20, 30, 64, 2)
    one = torch.zeros(1, dtype=torch.int32, device=gpu)
    out = taot.matmul_i8(x, sx, w, sw, offsets=one, experts=one[:0])
    assert out.shape == (20, 30) and not out.any()
    assert taot.matmul_i8(x[:0], sx[:0], w, sw, offsets=one, experts=one[:0]).shape == (0, 30)
    assert taot.matmul_i8(x[:0], sx[:0], w[0], sw[0]).shape == (0, 30)


def test_scales_that_are_not_finite(gpu):
    x, sx, w, sw = _operands(gpu, 20, 30, 64)
    clean = taot.matmul_i8(x, sx, w, sw)
    sx[3] = float("nan")
    out = taot.matmul_i8(x, sx, w, sw)
    rest = [i for i in range(20) if i != 3]
    assert torch.isnan(out[3]).all() and torch.equal(out[rest], clean[rest])


def test_offsets_beyond_32_bits(gpu):
    """Inputs and outputs of more than 2^31 values: their last rows."""
    print("[product] large", flush=True)
    M, K = 70000, 32768
    x = torch.zeros((M, K), dtype=torch.int8, device=gpu)
    x[-3:] = 1
    w = torch.ones((20, K), dtype=torch.int8, device=gpu)
    out = taot.matmul_i8(x, torch.ones(M, device=gpu), w, torch.ones(20, device=gpu), dtype=torch.float32)
    assert (out[-3:] == K).all() and not out[:-3].any()
    del x, w, out
    G, N, K = 9, 16384, 16384
    w = torch.zeros((G, N, K), dtype=torch.int8, device=gpu)
    w[-1, -1] = 2
    x = torch.ones((4, K), dtype=torch.int8, device=gpu)
    out = taot.matmul_i8(x, torch.ones(4, device=gpu), w, torch.ones((G, N), device=gpu), dtype=torch.float32,
                         offsets=torch.tensor([0, 2, 4], dtype=torch.int32, device=gpu),
                         experts=torch.tensor([0, 8], dtype=torch.int32, device=gpu))
    assert (out[2:, -1] == 2 * K).all() and not out[:2].any() and not out[:, :-1].any()
    del x, w, out
    M, N, K = 60000, 40000, 16
    x, w = torch.ones((M, K), dtype=torch.int8, device=gpu), torch.ones((N, K), dtype=torch.int8, device=gpu)
    sx = torch.ones(M, device=gpu)
    sx[-1] = 2.0
    out = taot.matmul_i8(x, sx, w, torch.ones(N, device=gpu))
    assert (out[-1] == 2 * K).all() and (out[-2] == K).all() and (out[0] == K).all() and (out[53687] == K).all()


def test_leading_dimensions_and_another_stream(gpu):
    x, sx, w, sw = _operands(gpu, 24, 40, 200)
    want = taot.matmul_i8(x, sx, w, sw)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = taot.matmul_i8(x.view(2, 3, 4, 200), sx.view(2, 3, 4, 1), w, sw, stream=s)
    many = taot.matmul_i8(x, sx, w[None], sw[None], offsets=torch.tensor([0, 24], dtype=torch.int32, device=gpu), stream=s)
    s.synchronize()
    assert out.shape == (2, 3, 4, 40) and torch.equal(out.view(24, 40), want) and torch.equal(many, want)


def test_refusals(gpu):
    x, sx, w, sw = _operands(gpu, 8, 30, 64, 2)
    off = torch.tensor([0, 4, 8], dtype=torch.int32, device=gpu)
    for call in (lambda: taot.matmul_i8(x.float(), sx, w, sw, offsets=off), lambda: taot.matmul_i8(x, sx, w.short(), sw, offsets=off),
                 lambda: taot.matmul_i8(x, sx.half(), w, sw, offsets=off), lambda: taot.matmul_i8(x, sx, w, sw, offsets=off.long()),
                 lambda: taot.matmul_i8(x, sx, w, sw, offsets=off, dtype=torch.float64), lambda: taot.matmul_i8(x.cpu(), sx, w, sw),
                 lambda: taot.quantize_rows(x), lambda: taot.quantize_rows(None)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: taot.matmul_i8(x, sx, w, sw), lambda: taot.matmul_i8(x, sx, w[0], sw[0], offsets=off),
                 lambda: taot.matmul_i8(x[:, :32].contiguous(), sx, w, sw, offsets=off), lambda: taot.matmul_i8(x, sx[:3], w, sw, offsets=off),
                 lambda: taot.matmul_i8(x, sx, w, sw[:1], offsets=off), lambda: taot.matmul_i8(x, sx, w, sw, offsets=off[:2]),
                 lambda: taot.matmul_i8(x, sx, w, sw, offsets=off, experts=off), lambda: taot.matmul_i8(x, sx, w[0], sw[0], experts=off),
                 lambda: taot.matmul_i8(x, sx, w, sw, offsets=off[:0]), lambda: taot.matmul_i8(x, sx, w[0].t(), sw[0]),
                 lambda: taot.quantize_rows(sx.view(8, 1), gated=True)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(taot.TaotError) as e:
        taot.matmul_i8(x, sx, w, sw, offsets=off, workspace=torch.empty(8, dtype=torch.uint8, device=gpu))
    assert e.value.code == 3
    with pytest.raises(taot.TaotError) as e:
        taot.quantize_rows(torch.zeros(1, 32769, device=gpu))
    assert e.value.code == 2
    with pytest.raises(RuntimeError, match="weight_scale"):
        taot.matmul_i8(x, sx, w, sw.clone().requires_grad_(), offsets=off)
