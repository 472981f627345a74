"""Calls of the 8-bit and the grouped products that the other tests do not reach: more tiles or rows than a launch has workgroups, so that
these go round, and what lies far behind an output whose last tile is nearly empty."""
import pytest

import paper_2006_03031_amd as nb

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

MOST = 1 << 21      # workgroups of a launch
U = 2.0 ** -24


def _codes(seed, shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-128, 128, shape, dtype=torch.int8, device="cuda", generator=g)


def _parts(n, size=1 << 23):
    return [slice(a, min(a + size, n)) for a in range(0, n, size)]


def _check(y, s, scale, bias, where):
    """y against the exact sums s (integers), in float64: u each for the sum to f32, the scales' product, its product with the sum, the sum with the bias."""
    v = s.double() * scale.double()
    err = 1.01 * (3 * U * v.abs() + U * (v + bias).abs()) + 1e-37
    assert bool(((y.double() - (v + bias)).abs() <= err).all()), where


# (kernel, K, N): the streaming and the any-alignment kernel
@pytest.mark.parametrize("kernel,N,K", [(2, 70000000 + 19, 16), (0, 35000000 + 7, 15)])
def test_dense_i8_goes_round(kernel, N, K):
    from paper_2006_03031_amd import runtime as rt
    p = nb.product_plan(1, None, N, K)
    assert p.kernel == kernel and p.grid == MOST < p.tiles
    x, w = _codes(1, (1, K)), _codes(2, (N, K))
    ws = torch.rand(N, device="cuda") + 0.5
    bias = torch.full((N,), 0.25, dtype=torch.bfloat16, device="cuda")
    y = rt.dense_i8(x, torch.full((1,), 0.5, device="cuda"), w, ws, bias, nb.EPI_BIAS, nb.F32)
    for part in _parts(N):
        _check(y[0, part], (w[part].int() * x.int()).sum(1), 0.5 * ws[part], 0.25, part)


@pytest.mark.parametrize("cuts", [[0, 2, 3], [0, 3, 3]])   # (the second leaves before the tiles that the host allowed for: a group less)
@pytest.mark.parametrize("kernel,N,K", [(2, 35000000 + 3, 16), (0, 17500000 + 5, 15)])
def test_grouped_dense_i8_goes_round(kernel, N, K, cuts):
    from paper_2006_03031_amd import runtime as rt
    p = nb.product_plan(3, 2, N, K)
    assert p.kernel == kernel and p.grid == MOST < p.tiles
    x, w = _codes(3, (3, K)), _codes(4, (2, N, K))
    xs, ws = torch.rand(3, device="cuda") + 0.5, torch.rand((2, N), device="cuda") + 0.5
    y = rt.grouped_dense_i8(x, xs, w, ws, None, torch.tensor(cuts, device="cuda"), nb.EPI_NONE, nb.F32)
    for r in range(3):
        e = 0 if r < cuts[1] else 1
        for part in _parts(N):
            _check(y[r, part], (w[e, part].int() * x[r].int()).sum(1), ws[e, part].double() * xs[r].double(), 0.0, (r, part))


# a wave per row (four rows a workgroup), and four waves per row
@pytest.mark.parametrize("M,K", [(4 * MOST + 21, 8), (MOST + 13, 1030)])
def test_quantize_rows_goes_round(M, K):
    from paper_2006_03031_amd import runtime as rt
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.empty((M, K), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    x *= torch.exp2((torch.arange(M, device="cuda") % 7).bfloat16())[:, None]
    q, scale = rt.quantize_rows(x, K)
    for part in _parts(M, (1 << 27) // K):
        v = x[part].double()
        top = v.abs().amax(1)
        assert bool((q[part] == torch.round(127 * v / top[:, None])).all()), part
        assert bool((scale[part] == (top / 127).float()).all()), part


# A last tile of 4 rows (one of 16: 1) and more than a tile's rows of memory behind it, for each kernel and each height of the large tiles.
@pytest.mark.parametrize("M,N,K", [(4100, 520, 656), (4164, 2040, 656), (2692, 4088, 656), (2020, 6136, 656), (7940, 2040, 656), (68, 72, 1024), (36, 1000, 256),
                                   (17, 4096, 1024), (68, 1001, 1003), (4100, 1001, 101)])
@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("out", [nb.BF16, nb.F32])
def test_nothing_behind_the_output_changes(M, N, K, grouped, out):
    from paper_2006_03031_amd import runtime as rt
    dtype = torch.bfloat16 if out == nb.BF16 else torch.float32
    buf = torch.full(((M + 300) * N + 4096,), 768.0, dtype=dtype, device="cuda")
    y = buf[:M * N].view(M, N)
    x, w = _codes(6, (M, K)), _codes(7, (2, N, K))
    xs, ws = torch.ones(M, device="cuda"), torch.full((2, N), 2.0 ** -20, device="cuda")
    rows = M
    if grouped:     # the last group ends 290 rows ahead of the output's end where there are so many
        rows = M - 290 if M > 600 else M
        rt.grouped_dense_i8(x, xs, w, ws, None, torch.tensor([0, 1, rows], device="cuda"), nb.EPI_NONE, out, out=y)
    else:
        rt.dense_i8(x, xs, w[0], ws[0], None, nb.EPI_NONE, out, out=y)
    assert bool((buf[rows * N:] == 768).all())
    assert bool((y[:rows].abs() < 768).all())
