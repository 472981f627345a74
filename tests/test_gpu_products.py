"""The 8-bit and the grouped products and the quantisation of rows against float64.

Tolerances, from the roundings on the way (u = 2^-24 for f32; a second-order term is far below the slack of 1.01):
  8 bits: the sum is exact; to f32 u, product of the two scales u, their product with the sum u, sum with the bias u of the result.
  bf16:   K products, exact in f32, added in some order: K u sum |x w| at most; the bias as above.
  GELU:   its fit is within 2.5194e-5 of the erf form (test_the_gelus_fit evaluates both in float64 over every argument, on the
          CPU), its exp2 and reciprocal within 2^-21 of the value, its slope at most 1.13.
  output in bf16: half a step, 2^-8 of the value."""
import math
import zlib

import pytest

import paper_2006_03031_amd as nb

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FIT = 2.52e-5
EPIS = {"none": nb.EPI_NONE, "bias": nb.EPI_BIAS, "gelu": nb.EPI_BIAS_GELU_ERF}
DTYPES = {nb.BF16: torch.bfloat16, nb.F32: torch.float32}
KEPT = 768.0   # content of rows and of memory that a call has to leave alone


@pytest.fixture(scope="module")
def rt():
    nb.load()
    from paper_2006_03031_amd import runtime
    return runtime


def _gen(*seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(zlib.crc32(repr(seed).encode()))
    return g


def _codes(g, shape):
    return torch.randint(-128, 128, shape, dtype=torch.int16, device="cuda", generator=g).to(torch.int8)


def _scales(g, shape):
    return torch.empty(shape, device="cuda").uniform_(0.001, 0.02, generator=g)


def _normal(g, shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0, std, generator=g).to(torch.bfloat16)


def _guarded(shape, dtype):
    """An output and the whole buffer it is the front of."""
    n = math.prod(shape)
    buf = torch.full((n + 512,), KEPT, dtype=dtype, device="cuda")
    return buf[:n].view(shape), buf[n:]


def _reference(x, w, xs, ws, bias, epi):
    """The result and how far an output may be from it before it is rounded to the output's type."""
    s = x.double() @ w.double().t().contiguous()
    if xs is not None:
        s = s * (xs.double()[:, None] * ws.double()[None, :])
        err = 3 * U * s.abs()
    else:
        err = (x.shape[1] + 1) * U * (x.double().abs() @ w.double().abs().t().contiguous())
    v = s if bias is None else s + bias.double()
    err = 1.01 * (err + U * v.abs()) + 1e-37
    if epi == "gelu":
        err = 1.13 * err + FIT + 2.0 ** -21 * v.abs()
        v = 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    return v, err


def _check(y, v, err):
    if y.dtype == torch.bfloat16:
        err = err + 2.0 ** -8 * (v.abs() + err)
    else:
        err = err + U * v.abs()
    d = (y.double() - v).abs()
    assert bool(torch.isfinite(y).all())
    worst = (d / err).max().item() if d.numel() else 0.0
    assert worst <= 1.0, worst


# --------------------------------------------------------------------------------------------- quantize_rows
def _codes_of(x, cols):
    """float64 from the definition: 127 x is exact, the quotient correctly rounded, which keeps ties ties."""
    x64 = x.double()
    top = x64.abs().amax(1) if x.shape[1] else x64.new_zeros(x.shape[0])
    q = torch.where(top[:, None] > 0, torch.round(127 * x64 / top[:, None]), 0.0)
    bad = ~torch.isfinite(top)
    q[bad] = 0
    scale = (top / 127).float()
    scale[bad] = float("nan")
    wide = torch.zeros((x.shape[0], cols), dtype=torch.float64, device=x.device)
    wide[:, :x.shape[1]] = q
    return wide.to(torch.int8), scale


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K,cols", [(1, 1, 0), (3, 7, 7), (5, 8, 0), (2, 64, 65), (7, 129, 0), (4, 1000, 1000), (300, 512, 0), (9, 4096, 0),
                                      (3, 8191, 8191), (2, 20001, 0), (1025, 384, 0), (2500, 33, 40), (4000, 128, 0), (3, 0, 16), (70000, 8, 8)])
def test_codes_and_scales(rt, dtype, M, K, cols):
    g = _gen(M, K, cols)
    x = torch.empty((M, K), device="cuda").normal_(0, 1, generator=g) * torch.exp2(torch.randint(-30, 30, (M, 1), device="cuda", generator=g))
    x[::7] = 0
    x = x.to(dtype)
    q, scale = rt.quantize_rows(x, cols)
    rq, rs = _codes_of(x, q.shape[1])
    assert q.shape[1] == (cols or -(-K // 128) * 128)
    assert bool((q == rq).all()), (q != rq).nonzero()[:5]
    assert bool((scale == rs).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_codes_at_the_border_of_two(rt, dtype):
    """x = top (j + 1/2) / 127 exactly, and its neighbours; every mantissa of the largest value."""
    m = torch.arange(128, 256, device="cuda", dtype=torch.float64)                    # largest values, 8 bits
    j = torch.arange(-127, 127, device="cuda", dtype=torch.float64)
    x = (j[None, :] + 0.5) / 127 * m[:, None]
    x = x.to(dtype)
    x = torch.cat([x, torch.nextafter(x, x + 1), torch.nextafter(x, x - 1), m[:, None].to(dtype)], 1) if dtype is torch.float32 else \
        torch.cat([x, m[:, None].to(dtype), -m[:, None].to(dtype) / 2], 1)
    for scale in (1.0, 2.0 ** -120, 2.0 ** 119):
        y = (x.double() * scale).to(dtype)
        q, s = rt.quantize_rows(y, y.shape[1])
        rq, rs = _codes_of(y, y.shape[1])
        assert bool((q == rq).all()), (scale, (q != rq).nonzero()[:5])
        assert bool((s == rs).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_that_are_tiny_huge_or_no_numbers(rt, dtype):
    fi = torch.finfo(dtype)
    rows = [[fi.tiny, -fi.tiny / 2, fi.smallest_normal / 128], [fi.tiny / 128, 0, 0], [fi.max, -fi.max, fi.max / 3], [0, 0, 0], [-0.0, 0, 0],
            [float("inf"), 1, 2], [1, float("nan"), 2], [1, -float("inf"), float("nan")], [1, 2, -3], [2.0 ** -101, 2.0 ** -100, 0]]
    x = torch.tensor(rows, dtype=dtype, device="cuda")
    for wide in (3, 700, 9000):        # one thread, one wave, rows that are read twice
        y = torch.zeros((len(rows), wide), dtype=dtype, device="cuda")
        y[:, -3:] = x
        q, s = rt.quantize_rows(y, wide)
        rq, rs = _codes_of(y, wide)
        assert bool((q == rq).all())
        assert bool(((s == rs) | (s.isnan() & rs.isnan())).all()), (s, rs)


# --------------------------------------------------------------------------------------------- dense_i8
I8_SHAPES = [(1, 1, 1), (1, 16, 64), (1, 4096, 1024), (2, 5, 15), (3, 17, 17), (5, 130, 100), (15, 33, 128), (16, 64, 192), (17, 128, 256),
             (31, 100, 1040), (33, 256, 4096), (48, 48, 48), (63, 1001, 1003), (64, 512, 144), (65, 65, 65), (100, 2048, 512), (127, 136, 2064), (128, 128, 128),
             (129, 260, 640), (200, 1024, 4096), (255, 255, 255), (257, 264, 272), (515, 1001, 1040), (1000, 504, 1008), (2049, 256, 128), (1030, 1032, 400),
             (700, 2056, 1024), (3000, 768, 768), (9, 3, 131071), (300, 128, 20000)]


@pytest.mark.parametrize("M,N,K", I8_SHAPES)
@pytest.mark.parametrize("epi,out", [("none", nb.F32), ("bias", nb.BF16), ("gelu", nb.BF16), ("gelu", nb.F32)])
def test_dense_i8(rt, M, N, K, epi, out):
    g = _gen(M, N, K)
    x, w, xs, ws = _codes(g, (M, K)), _codes(g, (N, K)), _scales(g, (M,)), _scales(g, (N,)) / K ** 0.5
    bias = None if epi == "none" else _normal(g, (N,))
    y, behind = _guarded((M, N), DTYPES[out])
    assert rt.dense_i8(x, xs, w, ws, bias, EPIS[epi], out, out=y) is y
    _check(y, *_reference(x, w, xs, ws, bias, epi))
    assert bool((behind == KEPT).all())


def test_dense_i8_sums_are_exact(rt):
    """Every product 16384, the largest sum there is: 131071 times; and one off it."""
    K = 131071
    x = torch.full((3, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((5, K), -128, dtype=torch.int8, device="cuda")
    x[1, K - 1] = 127
    x[2] = 127
    one = torch.ones(5, device="cuda")
    y = rt.dense_i8(x, one[:3], w, one, None, nb.EPI_NONE, nb.F32)
    s = (x.double() @ w.double().t()).float()
    assert bool((y == s).all())


@pytest.mark.parametrize("M,N,K", [(1, 64, 128), (40, 100, 256), (300, 300, 384)])
def test_dense_i8_passes_scales_that_are_no_numbers_on(rt, M, N, K):
    g = _gen(M)
    x, w, xs, ws = _codes(g, (M, K)), _codes(g, (N, K)), _scales(g, (M,)), _scales(g, (N,))
    xs[M // 2], ws[3] = float("nan"), float("inf")
    y = rt.dense_i8(x, xs, w, ws, None, nb.EPI_NONE, nb.F32)
    s = (x.double() @ w.double().t()).float() * (xs[:, None] * ws)
    assert bool((torch.isnan(y) == torch.isnan(s)).all()) and bool((torch.isinf(y) == torch.isinf(s)).all())


# --------------------------------------------------------------------------------------------- grouped products
def _offsets(kind, R, E, g):
    if kind == "one":           # all rows in one group, the others empty
        cuts = [0] * (E // 2 + 1) + [R] * (E - E // 2)
    elif kind == "empty":
        cuts = [R // 2] * (E + 1)
    else:                       # ragged, some empty; rows ahead of the first and behind the last group
        lo, hi = (R // 9, R - R // 7) if kind == "inside" else (0, R)
        inner = torch.randint(lo, hi + 1, (E - 1,), generator=g, device="cuda").tolist()
        if E > 3:
            inner[1] = inner[0]
        cuts = [lo] + sorted(inner) + [hi]
    return torch.tensor(cuts, dtype=torch.int64, device="cuda")


GROUPED_SHAPES = [(1, 1, 16, 64), (1, 64, 128, 256), (5, 3, 33, 40), (8, 16, 512, 1024), (16, 64, 1024, 512), (40, 4, 100, 100), (64, 7, 72, 1000),
                  (100, 1, 256, 128), (130, 5, 1001, 56), (200, 33, 130, 264), (515, 7, 1001, 1000), (600, 2, 264, 64), (700, 1024, 40, 32),
                  (1000, 65, 128, 192), (1500, 3, 260, 1024), (2000, 8, 512, 512), (3001, 20, 136, 333), (5000, 129, 128, 128)]


@pytest.mark.parametrize("R,E,N,K", GROUPED_SHAPES)
@pytest.mark.parametrize("split", ["whole", "inside", "one", "empty"])
@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("epi,out", [("none", nb.F32), ("gelu", nb.BF16)])
def test_grouped(rt, R, E, N, K, split, int8, epi, out):
    g = _gen(R, E, N, K, split)
    offsets = _offsets(split, R, E, g)
    bias = None if epi == "none" else _normal(g, (E, N))
    y, behind = _guarded((R, N), DTYPES[out])
    if int8:
        x, w, xs, ws = _codes(g, (R, K)), _codes(g, (E, N, K)), _scales(g, (R,)), _scales(g, (E, N)) / K ** 0.5
        rt.grouped_dense_i8(x, xs, w, ws, bias, offsets, EPIS[epi], out, out=y)
    else:
        x, w, xs, ws = _normal(g, (R, K)), _normal(g, (E, N, K), K ** -0.5), None, None
        rt.grouped_dense(x, w, bias, offsets, EPIS[epi], out, out=y)
    cuts = offsets.tolist()
    for e in range(E):
        lo, hi = cuts[e], cuts[e + 1]
        if lo < hi:
            _check(y[lo:hi], *_reference(x[lo:hi], w[e], xs[lo:hi] if int8 else None, ws[e] if int8 else None,
                                         None if bias is None else bias[e], epi))
    assert bool((y[:cuts[0]] == KEPT).all()) and bool((y[cuts[E]:] == KEPT).all()) and bool((behind == KEPT).all())


@pytest.mark.parametrize("int8", [False, True])
def test_grouped_rows_do_not_depend_on_what_is_in_other_rows(rt, int8):
    """NaN in rows of no group, in other groups' rows and weights, and at the neighbours in memory stays there."""
    g = _gen(3)
    for R, N, K in ((90, 72, 200), (700, 300, 256), (20, 64, 1024)):
        offsets = torch.tensor([2, R // 3, R // 3, R - 5], device="cuda")
        w = _normal(g, (3, N, K), 0.05)
        x = _normal(g, (R, K))
        if int8:
            x, xs = rt.quantize_rows(x)
            w, ws = rt.quantize_rows(w.view(3 * N, K))
            w, ws = w.view(3, N, -1), ws.view(3, N)
            xs[:2], xs[R - 5:], ws[1] = float("nan"), float("nan"), float("nan")
            y = rt.grouped_dense_i8(x, xs, w, ws, None, offsets, nb.EPI_NONE)
        else:
            x[:2], x[R - 5:], w[1] = float("nan"), float("nan"), float("nan")
            y = rt.grouped_dense(x, w, None, offsets, nb.EPI_NONE)
        assert bool(torch.isfinite(y[2:R - 5]).all())


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_bf16_infinities_and_nan_reach_their_own_rows_only(rt, int8, value):
    g = _gen(4)
    for R, N, K in ((3, 64, 264), (300, 256, 264), (600, 256, 1000)):
        x, w = _normal(g, (R, K)), _normal(g, (2, N, K), 0.05)
        x[1, K - 1] = value
        offsets = torch.tensor([0, R // 2 + 1, R], device="cuda")
        if int8:
            xq, xs = rt.quantize_rows(x)
            wq, ws = rt.quantize_rows(w.view(2 * N, K))
            y = rt.grouped_dense_i8(xq, xs, wq.view(2, N, -1), ws.view(2, N), None, offsets, nb.EPI_NONE)
        else:
            y = rt.grouped_dense(x, w, None, offsets, nb.EPI_NONE)
        bad = ~torch.isfinite(y)
        assert bool(bad[1].all()) and int(bad.sum()) == N


# Offsets that fall or leave the tensor: rows of unspecified content, nothing outside the output.
@pytest.mark.parametrize("cuts", [[-5, 10, 400, 999], [0, 200, 100, 300], [300, 200, 100, 0], [2 ** 40, 2 ** 40, 7, 8], [-2 ** 62, 2 ** 62, -1, 2 ** 62]])
@pytest.mark.parametrize("int8", [False, True])
def test_offsets_that_do_not_keep_to_the_rows(rt, cuts, int8):
    R, N, K = 300, 128, 128
    g = _gen(5)
    y, behind = _guarded((R, N), torch.float32)
    offsets = torch.tensor(cuts, device="cuda")
    if int8:
        rt.grouped_dense_i8(_codes(g, (R, K)), _scales(g, (R,)), _codes(g, (3, N, K)), _scales(g, (3, N)), None, offsets, nb.EPI_NONE, nb.F32, out=y)
    else:
        rt.grouped_dense(_normal(g, (R, K)), _normal(g, (3, N, K)), None, offsets, nb.EPI_NONE, nb.F32, out=y)
    assert bool(torch.isfinite(y).all()) and bool((behind == KEPT).all())


# Each height of the large tiles, as the dispatch takes it: a last tile that is not full, N not of whole tiles, K not of whole stages,
# tiles that follow others; K of exactly the stages that are loaded ahead, and of fewer.
@pytest.mark.parametrize("bm,M,N,K", [(128, 4100, 520, 656), (160, 4100, 2040, 656), (192, 3000, 4088, 656), (224, 2048, 6136, 656),
                                      (256, 8177, 2040, 656), (256, 8177, 2040, 256), (128, 4100, 520, 384), (128, 4100, 520, 272),
                                      (128, 5000, 520, 48), (160, 4100, 4088, 80), (192, 4100, 2040, 128), (224, 2048, 6136, 144),
                                      (256, 5000, 6136, 48), (256, 5000, 6136, 16)])
@pytest.mark.parametrize("epi,out", [("none", nb.F32), ("gelu", nb.BF16), ("bias", nb.BF16)])
def test_dense_i8_in_large_tiles(rt, bm, M, N, K, epi, out):
    p = nb.product_plan(M, None, N, K)
    assert (p.kernel, p.bm) == (1, bm)
    g = _gen(M, N, K)
    x, w, xs, ws = _codes(g, (M, K)), _codes(g, (N, K)), _scales(g, (M,)), _scales(g, (N,)) / K ** 0.5
    bias = None if epi == "none" else _normal(g, (N,))
    y, behind = _guarded((M, N), DTYPES[out])
    rt.dense_i8(x, xs, w, ws, bias, EPIS[epi], out, out=y)
    _check(y, *_reference(x, w, xs, ws, bias, epi))
    assert bool((behind == KEPT).all())


@pytest.mark.parametrize("bm,R,E,N,K", [(128, 300, 3, 6136, 656), (160, 1500, 8, 4088, 656), (192, 2048, 8, 4088, 656), (224, 3000, 3, 4088, 656),
                                        (256, 2048, 3, 6136, 656), (128, 700, 3, 3064, 48), (160, 4100, 8, 4088, 128), (192, 1200, 3, 6136, 80),
                                        (224, 6000, 3, 2040, 144), (256, 1500, 8, 6136, 48)])
@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("epi,out", [("none", nb.F32), ("gelu", nb.BF16)])
def test_grouped_in_large_tiles(rt, bm, R, E, N, K, int8, epi, out):
    p = nb.product_plan(R, E, N, K, nb.I8 if int8 else nb.BF16)
    assert (p.kernel, p.bm) == (1, bm)
    g = _gen(R, E, N, K)
    cuts = [7] + sorted(torch.randint(7, R - 8, (E - 1,), generator=g, device="cuda").tolist()) + [R - 9]
    offsets = torch.tensor(cuts, device="cuda")
    bias = None if epi == "none" else _normal(g, (E, N))
    y, behind = _guarded((R, N), DTYPES[out])
    for turn in range(2):   # the second time the groups lie elsewhere, the rest of the output is as it was
        if int8:
            x, w, xs, ws = _codes(g, (R, K)), _codes(g, (E, N, K)), _scales(g, (R,)), _scales(g, (E, N)) / K ** 0.5
            rt.grouped_dense_i8(x, xs, w, ws, bias, offsets, EPIS[epi], out, out=y)
        else:
            x, w, xs, ws = _normal(g, (R, K)), _normal(g, (E, N, K), K ** -0.5), None, None
            rt.grouped_dense(x, w, bias, offsets, EPIS[epi], out, out=y)
        for e in range(E):
            lo, hi = cuts[e], cuts[e + 1]
            if lo < hi:
                _check(y[lo:hi], *_reference(x[lo:hi], w[e], xs[lo:hi] if int8 else None, ws[e] if int8 else None,
                                             None if bias is None else bias[e], epi))
        assert bool((y[:cuts[0]] == KEPT).all()) and bool((y[cuts[E]:] == KEPT).all()) and bool((behind == KEPT).all())
        cuts = [7] + [R - 9] * E   # all rows in the first group
        offsets.copy_(torch.tensor(cuts))


@pytest.mark.parametrize("epi", ["none", "gelu"])
def test_no_k_at_all(rt, epi):
    """Sums of nothing are 0: what comes out is the bias (or its GELU)."""
    M, N, E = 70, 40, 3
    bias = None if epi == "none" else _normal(_gen(9), (E, N))
    x, w, xs, ws = (torch.empty((M, 0), dtype=torch.int8, device="cuda"), torch.empty((E, N, 0), dtype=torch.int8, device="cuda"),
                    torch.ones(M, device="cuda"), torch.ones((E, N), device="cuda"))
    off = torch.tensor([0, 30, 30, M], device="cuda")
    group = torch.tensor([0] * 30 + [2] * 40, device="cuda")
    v = torch.zeros((M, N), dtype=torch.float64, device="cuda") if bias is None else bias.double()[group]
    if epi == "gelu":
        v = 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    b0 = None if bias is None else bias[0]
    err = FIT + 2.0 ** -21 * (v.abs() if bias is None else bias.double()[group].abs())
    for y in (rt.grouped_dense_i8(x, xs, w, ws, bias, off, EPIS[epi], nb.F32), rt.grouped_dense(x.bfloat16(), w.bfloat16(), bias, off, EPIS[epi], nb.F32)):
        _check(y, v, err)
    _check(rt.dense_i8(x[:30], xs[:30], w[0], ws[0], b0, EPIS[epi], nb.F32), v[:30], err[:30])


# Byte offsets past 2^32 in each operand: the streaming, the large-tile and the any-alignment kernel.
@pytest.mark.parametrize("M,N,K", [(300000, 24, 16384), (600000, 16, 8191), (140000, 16384, 192), (24, 300000, 16384), (530000, 4099, 64)])
def test_operands_past_4_gib(rt, M, N, K):
    g = _gen(M, N, K)
    x = torch.randint(-128, 128, (M, K), dtype=torch.int8, device="cuda", generator=g)
    w = torch.randint(-128, 128, (N, K), dtype=torch.int8, device="cuda", generator=g)
    xs, ws = _scales(g, (M,)), _scales(g, (N,))
    y = rt.dense_i8(x, xs, w, ws, None, nb.EPI_NONE)
    rows = torch.tensor(sorted({0, 1, M // 3, M // 2, M - 2, M - 1}), device="cuda")
    v, err = _reference(x[rows], w, xs[rows], ws, None, "none")
    _check(y[rows], v, err)
    columns = torch.tensor(sorted({0, 1, N // 3, N // 2, N - 2, N - 1}), device="cuda")
    v, err = _reference(x[-50:], w[columns], xs[-50:], ws[columns], None, "none")
    _check(y[-50:][:, columns], v, err)
    del y
    torch.cuda.empty_cache()


def test_grouped_weights_past_4_gib(rt):
    """The last of many experts lies past 2^32 bytes of weights; a row for it, one for the first."""
    E, N, K = 300, 2048, 4096
    w = torch.zeros((E, N, K), dtype=torch.bfloat16, device="cuda")
    g = _gen(1)
    w[0], w[E - 1] = _normal(g, (N, K), 0.02), _normal(g, (N, K), 0.02)
    for R in (2, 700):
        x = _normal(g, (R, K))
        off = torch.full((E + 1,), R // 2, dtype=torch.int64, device="cuda")
        off[0], off[E] = 0, R
        y = rt.grouped_dense(x, w, None, off, nb.EPI_NONE, nb.F32)
        _check(y[:R // 2], *_reference(x[:R // 2], w[0], None, None, None, "none"))
        _check(y[R // 2:], *_reference(x[R // 2:], w[E - 1], None, None, None, "none"))


# --------------------------------------------------------------------------------------------- together
def test_a_layer_of_experts_in_8_bits(rt):
    """Tokens to two experts each: grouped up with GELU, down, as a program runs them, in 8 bits and in bf16."""
    g = _gen(6)
    T, E, D, F = 150, 6, 256, 640
    x = _normal(g, (T, D))
    w1, w2 = _normal(g, (E, F, D), D ** -0.5), _normal(g, (E, D, F), F ** -0.5)
    b1, b2 = _normal(g, (E, F), 0.1), _normal(g, (E, D), 0.1)
    chosen = torch.stack([torch.randperm(E - 1, device="cuda", generator=g)[:2] for _ in range(T)])   # the last expert gets none
    order = torch.argsort(chosen.flatten(), stable=True)
    sizes = torch.bincount(chosen.flatten(), minlength=E)
    offsets = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)])
    rows = x[order // 2].contiguous()
    h = rt.grouped_dense(rows, w1, b1, offsets, nb.EPI_BIAS_GELU_ERF)
    y = rt.grouped_dense(h, w2, b2, offsets, nb.EPI_BIAS, nb.F32)
    w1q, w1s = rt.quantize_rows(w1.view(E * F, D))
    w2q, w2s = rt.quantize_rows(w2.view(E * D, F))
    hq = rt.grouped_dense_i8(*rt.quantize_rows(rows), w1q.view(E, F, -1), w1s.view(E, F), b1, offsets, nb.EPI_BIAS_GELU_ERF)
    yq = rt.grouped_dense_i8(*rt.quantize_rows(hq), w2q.view(E, D, -1), w2s.view(E, D), b2, offsets, nb.EPI_BIAS, nb.F32)
    # float64 from the same operands, layer by layer from the GPU's own hidden rows
    cuts = offsets.tolist()
    for e in range(E):
        lo, hi = cuts[e], cuts[e + 1]
        if lo == hi:
            continue
        _check(h[lo:hi], *_reference(rows[lo:hi], w1[e], None, None, b1[e], "gelu"))
        _check(y[lo:hi], *_reference(h[lo:hi], w2[e], None, None, b2[e], "bias"))
        a, sa = rt.quantize_rows(rows[lo:hi].contiguous())
        _check(hq[lo:hi], *_reference(a, w1q.view(E, F, -1)[e], sa, w1s.view(E, F)[e], b1[e], "gelu"))
        a, sa = rt.quantize_rows(hq[lo:hi].contiguous())
        _check(yq[lo:hi], *_reference(a, w2q.view(E, D, -1)[e], sa, w2s.view(E, D)[e], b2[e], "bias"))
    # an 8-bit code is off by at most half a step of its row: K steps of x and w side by side bound a result
    bound = 0.5 * (F * (hq.double().abs().amax(1) / 127)[:, None] * w2.double().abs().amax() + F * h.double().abs().amax() * w2.double().abs().amax() / 127)
    assert bool(((yq.double() - y.double()).abs() <= 2 * bound).all())


@pytest.mark.parametrize("M", [1, 70, 700])
def test_replays_of_a_captured_layer(rt, M):
    """quantize_rows, dense_i8 and a grouped product in a graph: replays on new inputs and offsets against eager calls."""
    g = _gen(M)
    D, F, E = 256, 512, 3
    w, ws = rt.quantize_rows(_normal(g, (F, D), 0.05))
    w2, b2 = _normal(g, (E, D, F), 0.05), _normal(g, (E, D))
    bias = _normal(g, (F,))
    x, offsets = _normal(g, (M, D)), torch.tensor([0, M // 2, M // 2, M], device="cuda")

    def layer():
        q, s = rt.quantize_rows(x)
        h = rt.dense_i8(q, s, w, ws, bias, nb.EPI_BIAS_GELU_ERF)
        return rt.grouped_dense(h, w2, b2, offsets, nb.EPI_BIAS, nb.F32)

    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer()
    for turn in range(4):
        x.copy_(_normal(g, (M, D)))
        offsets.copy_(torch.tensor([0, M * turn // 4, M, M], device="cuda"))
        graph.replay()
        first = y.clone()
        assert bool((first == layer()).all()), turn
        torch.cuda.synchronize()


def test_calls_on_two_streams_at_once(rt):
    g = _gen(8)
    x, w, xs, ws = _codes(g, (300, 512)), _codes(g, (640, 512)), _scales(g, (300,)), _scales(g, (640,))
    gx, gw, off = _normal(g, (300, 512)), _normal(g, (4, 128, 512)), torch.tensor([0, 10, 200, 200, 300], device="cuda")
    want = rt.dense_i8(x, xs, w, ws, None, nb.EPI_NONE), rt.grouped_dense(gx, gw, None, off, nb.EPI_NONE)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for i in range(20):
        with torch.cuda.stream(streams[i % 2]):
            got.append((rt.dense_i8(x, xs, w, ws, None, nb.EPI_NONE), rt.grouped_dense(gx, gw, None, off, nb.EPI_NONE)))
    torch.cuda.synchronize()
    for a, b in got:
        assert bool((a == want[0]).all()) and bool((b == want[1]).all())


def test_refused_tensors(rt):
    x, w = torch.zeros((4, 64), dtype=torch.int8, device="cuda"), torch.zeros((2, 8, 64), dtype=torch.int8, device="cuda")
    s, ws, off = torch.ones(4, device="cuda"), torch.ones((2, 8), device="cuda"), torch.tensor([0, 1, 4], device="cuda")
    none = nb.EPI_NONE
    for call, code in ((lambda: rt.dense_i8(x.t().contiguous().t(), s, w[0], ws[0], None, none), -8),
                       (lambda: rt.dense_i8(x, s, w[0], ws[0], None), -1),
                       (lambda: rt.dense_i8(x, s.double(), w[0], ws[0], None, none), -4),
                       (lambda: rt.dense_i8(x, s, w[0], ws[0].cpu(), None, none), -8),
                       (lambda: rt.dense_i8(x, s, w[0], ws[0], None, none, nb.I8), -4),
                       (lambda: rt.dense_i8(x, s, w[0], ws[0], None, none, out=torch.empty((4, 9), dtype=torch.bfloat16, device="cuda")), -3),
                       (lambda: rt.dense_i8(x, s, w[0], ws[0], None, none, nb.F32, out=torch.empty((4, 8), dtype=torch.bfloat16, device="cuda")), -4),
                       (lambda: rt.dense_i8(x.view(-1)[8:200].view(3, 64), s[:3], w[0], ws[0], None, none), -5),
                       (lambda: rt.dense_i8(x, s, w[0], ws[0], torch.zeros(9, dtype=torch.bfloat16, device="cuda")), -3),
                       (lambda: rt.grouped_dense_i8(x, s, w, ws, None, off.int(), none), -4),
                       (lambda: rt.grouped_dense_i8(x, s, w, ws, None, off[:2], none), -3),
                       (lambda: rt.grouped_dense(x.bfloat16(), w.bfloat16(), None, off.cpu(), none), -8),
                       (lambda: rt.grouped_dense(x, w, None, off, none), -4),
                       (lambda: rt.quantize_rows(x.half()), -4),
                       (lambda: rt.quantize_rows(x.float()[:, ::2]), -8)):
        with pytest.raises(nb.NimbleError) as e:
            call()
        assert e.value.code == code, (e.value, code)
