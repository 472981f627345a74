"""Shape functions, refusals and dispatch of the 8-bit and the grouped products (no GPU needed)."""
import ctypes

import pytest

import paper_2006_03031_amd as nb

torch = pytest.importorskip("torch")


def test_shapes():
    assert nb.quantize_rows_shape((5, 300)) == ((5, 384), (5,))
    assert nb.quantize_rows_shape((5, 256)) == ((5, 256), (5,))
    assert nb.quantize_rows_shape((0, 300), 301) == ((0, 301), (0,))
    assert nb.quantize_rows_shape((3, 0)) == ((3, 0), (3,))
    assert nb.dense_i8_shape((7, 64), (7,), (9, 64), (9,)) == (7, 9)
    assert nb.grouped_dense_shape((7, 64), (3, 9, 64), (4,)) == (7, 9)
    assert nb.grouped_dense_shape((0, 64), (0, 9, 64), (1,)) == (0, 9)
    assert nb.storage_bytes((3, 5), nb.I8) == 15


@pytest.mark.parametrize("call,code", [
    (lambda: nb.quantize_rows_shape((3,)), -2),
    (lambda: nb.quantize_rows_shape((3, -1)), -8),
    (lambda: nb.quantize_rows_shape((3, 20), 19), -3),
    (lambda: nb.quantize_rows_shape((3, 20), -1), -8),
    (lambda: nb.dense_i8_shape((7, 64), (7, 1), (9, 64), (9,)), -2),
    (lambda: nb.dense_i8_shape((7, 64), (7,), (9, 65), (9,)), -3),
    (lambda: nb.dense_i8_shape((7, 64), (8,), (9, 64), (9,)), -3),
    (lambda: nb.dense_i8_shape((7, 64), (7,), (9, 64), (1,)), -3),
    (lambda: nb.grouped_dense_shape((7, 64), (9, 64), (4,)), -2),
    (lambda: nb.grouped_dense_shape((7, 64), (3, 9, 60), (4,)), -3),
    (lambda: nb.grouped_dense_shape((7, 64), (3, 9, 64), (3,)), -3),
    (lambda: nb.product_plan(7, 1025, 9, 64), -8),
    (lambda: nb.product_plan(7, -1, 9, 64), -8),
    (lambda: nb.product_plan(7, None, 9, 131072), -8),
    (lambda: nb.product_plan(7, None, 9, 64, nb.BF16), -8),
    (lambda: nb.product_plan(7, 3, 9, 64, nb.F32), -4),
    (lambda: nb.product_plan(7, 3, 9, 64, nb.BF16, nb.I8), -4),
])
def test_refused_shapes(call, code):
    with pytest.raises(nb.NimbleError) as e:
        call()
    assert e.value.code == code


# Refused on the host before anything is launched: no GPU is needed to see it.  Pointers are numbers that are never followed.
P = 4096
QUANTIZE = dict(x=P, t=0, q=P, s=P, rows=3, K=64, cols=64)
I8 = dict(x=P, xs=P, w=P, ws=P, b=P, y=P, M=3, N=64, K=64, epi=1, out=0)
GROUPED = dict(x=P, w=P, b=P, off=P, y=P, R=3, E=2, N=64, K=64, epi=1, out=0)
GROUPED_I8 = dict(x=P, xs=P, w=P, ws=P, b=P, off=P, y=P, R=3, E=2, N=64, K=64, epi=1, out=0)


@pytest.mark.parametrize("name,good,wrong,code", [
    ("nimble_quantize_rows_dyn", QUANTIZE, dict(t=3), -4),
    ("nimble_quantize_rows_dyn", QUANTIZE, dict(cols=63), -3),
    ("nimble_quantize_rows_dyn", QUANTIZE, dict(rows=-1), -8),
    ("nimble_quantize_rows_dyn", QUANTIZE, dict(rows=1 << 31), -8),
    ("nimble_quantize_rows_dyn", QUANTIZE, dict(x=0), -1),
    ("nimble_quantize_rows_dyn", QUANTIZE, dict(s=0), -1),
    ("nimble_quantize_rows_dyn", QUANTIZE, dict(q=P + 8), -5),
    ("nimble_dense_i8_dyn", I8, dict(epi=3), -8),
    ("nimble_dense_i8_dyn", I8, dict(out=3), -4),
    ("nimble_dense_i8_dyn", I8, dict(K=131072), -8),
    ("nimble_dense_i8_dyn", I8, dict(M=-1), -8),
    ("nimble_dense_i8_dyn", I8, dict(b=0), -1),
    ("nimble_dense_i8_dyn", I8, dict(xs=0), -1),
    ("nimble_dense_i8_dyn", I8, dict(x=P + 4), -5),
    ("nimble_dense_i8_dyn", I8, dict(M=(1 << 31) - 1, N=1 << 30, K=64), -8),
    ("nimble_grouped_dense_dyn", GROUPED, dict(off=0), -1),
    ("nimble_grouped_dense_dyn", GROUPED, dict(off=P + 4), -5),
    ("nimble_grouped_dense_dyn", GROUPED, dict(E=1025), -8),
    ("nimble_grouped_dense_dyn", GROUPED, dict(E=-1), -8),
    ("nimble_grouped_dense_dyn", GROUPED, dict(y=0), -1),
    ("nimble_grouped_dense_dyn", GROUPED, dict(epi=-1), -8),
    ("nimble_grouped_dense_i8_dyn", GROUPED_I8, dict(E=-1), -8),
    ("nimble_grouped_dense_i8_dyn", GROUPED_I8, dict(ws=0), -1),
    ("nimble_grouped_dense_i8_dyn", GROUPED_I8, dict(out=2), -4),
])
def test_refused_calls(name, good, wrong, code):
    assert getattr(nb.load(), name)(*{**good, **wrong}.values(), None) == code
    assert nb.last_error()


@pytest.mark.parametrize("name,good,nothing", [
    ("nimble_quantize_rows_dyn", QUANTIZE, dict(rows=0, x=0, q=0, s=0)),
    ("nimble_dense_i8_dyn", I8, dict(M=0, x=0, y=0)),
    ("nimble_dense_i8_dyn", I8, dict(N=0, w=0, y=0)),
    ("nimble_grouped_dense_dyn", GROUPED, dict(R=0, x=0, y=0)),
    ("nimble_grouped_dense_dyn", GROUPED, dict(E=0, w=0, off=0)),
    ("nimble_grouped_dense_i8_dyn", GROUPED_I8, dict(R=0, x=0, y=0)),
])
def test_nothing_to_do(name, good, nothing):
    assert getattr(nb.load(), name)(*{**good, **nothing}.values(), None) == 0


def test_host_tensors_are_refused():
    from paper_2006_03031_amd import runtime as rt
    x, w = torch.zeros((3, 64), dtype=torch.int8), torch.zeros((2, 5, 64), dtype=torch.int8)
    s, ws, off = torch.zeros(3), torch.zeros((2, 5)), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: rt.quantize_rows(x.float()), lambda: rt.dense_i8(x, s, w[0], ws[0], None, nb.EPI_NONE),
                 lambda: rt.grouped_dense(x.bfloat16(), w.bfloat16(), None, off, nb.EPI_NONE),
                 lambda: rt.grouped_dense_i8(x, s, w, ws, None, off, nb.EPI_NONE)):
        with pytest.raises(nb.NimbleError) as e:
            call()
        assert e.value.code == -8
    with pytest.raises(nb.NimbleError) as e:
        rt.quantize_rows(x)
    assert e.value.code == -4
    with pytest.raises(nb.NimbleError) as e:
        rt.grouped_dense_i8(x, s[:2], w, ws, None, off)
    assert e.value.code == -3


# The grid is for the most tiles there can be, whatever the offsets: every split of R rows over E groups fits.
@pytest.mark.parametrize("in_dtype", [nb.BF16, nb.I8])
def test_the_grid_holds_the_tiles_of_every_split(in_dtype):
    import random
    rng = random.Random(3)
    for _ in range(300):
        R, E = rng.randint(1, rng.choice((5, 100, 5000))), rng.choice((1, 2, 7, 64, 300))
        N, K = rng.choice((1, 8, 128, 1001, 4096)), rng.choice((8, 64, 130, 1024, 4096))
        p = nb.product_plan(R, E, N, K, in_dtype)
        cuts = sorted(rng.randint(0, R) for _ in range(E + 1)) if rng.random() < 0.7 else sorted(rng.sample(range(R + 1), min(E + 1, R + 1)))
        rows = sum(-(-(b - a) // p.bm) for a, b in zip(cuts, cuts[1:]))
        assert rows * -(-N // p.bn) <= p.tiles, (R, E, N, K, p)
        assert p.grid * p.block < 1 << 32
    one = nb.product_plan(1000, None, 500, 64)
    assert one.tiles == -(-1000 // one.bm) * -(-500 // one.bn)


def test_plan_struct_matches_the_header():
    from paper_2006_03031_amd import binding
    assert ctypes.sizeof(binding._CProductPlan) == 32


def test_the_gelus_fit():
    """The constants of the epilogue's GELU (v sigmoid of an odd quintic, csrc/device_common.h) in float64 against the erf form: the GPU
    tests allow 2.52e-5 for it.  Beyond 9.5 either is v or 0 to within 1e-18."""
    import math
    import os
    import re
    from paper_2006_03031_amd import build
    with open(os.path.join(build.CSRC, "device_common.h")) as f:
        body = re.search(r"float gelu_exponent\(float v\) \{(.*?)\n\}", f.read(), re.S).group(1)
    c2, c1, c0 = (torch.tensor(float(c)).double() for c in re.findall(r"(-?\d\.\d+)f", body)[-3:])
    v = torch.linspace(-9.5, 9.5, 2000001, dtype=torch.float64)
    t = (v * v).clamp(max=81.0)
    fit = v / (1 + torch.exp2(((c2 * t + c1) * t + c0) * v))
    worst = (fit - 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))).abs().max().item()
    assert 2.5e-5 < worst < 2.52e-5, worst


# Two workgroups of 16 x 32 share a compute unit in a grouped call (58 KB of LDS each, the map of the groups among it), three in one without
# groups.  These shapes were taken for one round of three: 7.2, 7.2 and 25.9 us, where the members named here take 4.9, 4.9 and 9.9.
@pytest.mark.parametrize("R,E,N,K,tile", [(506, 8, 536, 128, (32, 32)), (907, 13, 384, 128, (32, 32)), (181, 17, 5808, 128, (128, 256))])
def test_the_rounds_of_grouped_calls(R, E, N, K, tile):
    p = nb.product_plan(R, E, N, K)
    assert (p.bm, p.bn) == tile


# Large products take tiles of 256 rows (53, 53, 397 and, N = 30528, 290 us; of 128 rows 61, 61, 463 and 340), one turn of 128 rows stays (31.5; 42.0 of 256).
@pytest.mark.parametrize("M,N,K,bm", [(8177, 30528, 1024, 256), (16384, 1024, 4096, 256), (4096, 4096, 4096, 256), (8192, 8192, 8192, 256), (8192, 1024, 4096, 128)])
def test_the_tiles_of_large_products(M, N, K, bm):
    p = nb.product_plan(M, None, N, K)
    assert (p.kernel, p.bm) == (1, bm)
