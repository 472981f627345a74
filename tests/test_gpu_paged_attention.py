"""paged_attention against the formula in 64 bits: types, head layouts, pages, lengths, masks that leave nothing, values behind masks, graphs."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paged_util as pu
from paged_util import BF, Batch


def _q(batch, H, D, seed=3):
    return torch.randn(batch.rows, H, D, generator=torch.Generator().manual_seed(seed)).to(BF)


def _run(q, cache, batch, **kw):
    from paper_2006_03031_amd import runtime as rt
    kw = {k: v.cuda() if torch.is_tensor(v) else v for k, v in kw.items()}
    return rt.paged_attention(q.cuda(), pu.to_gpu(cache), batch.on_gpu(), **kw)


def _check(got, q, cache, batch, window=0, alpha=None, weight_step=None):
    want, bound = pu.attention(q, cache, batch, window, alpha, weight_step)
    got = got.double().cpu()
    rows = [r for _, r, _ in batch.each()]
    off = ((got - want).abs() - bound)[rows]
    assert bool((off <= 0).all()), f"beyond the bound by up to {float(off.max())} (NaN: {int(got[rows].isnan().sum())})"


SHAPES = [(1, 1), (4, 1), (6, 2), (16, 16), (24, 8), (20, 1), (32, 2)]
SIZES = {
    "one": [(0, 1)],
    "two_tokens": [(0, 2)],
    "short": [(4, 1), (0, 1), (16, 1), (14, 1), (31, 1), (32, 1), (63, 1)],
    "empty_ones": [(0, 0), (30, 1), (0, 0), (5, 3), (0, 0)],
    "ragged": [(0, 37), (100, 1), (63, 5), (0, 1), (257, 20), (15, 2)],
    "long": [(700, 1), (3, 1)],
}


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,G", SHAPES)
@pytest.mark.parametrize("sizes", SIZES)
def test_formula(sizes, H, G, D, int8):
    batch = Batch(SIZES[sizes], 16)
    cache, q = pu.random_cache(batch, G, D, int8), _q(batch, H, D)
    _check(_run(q, cache, batch), q, cache, batch)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sizes", ["short", "ragged", "long"])
def test_probabilities_of_few_rows_are_kept_in_two_parts(sizes, D, int8):
    batch = Batch(SIZES[sizes] if sizes != "long" else [(5000, 1), (12, 1), (2100, 1)], 32)
    cache, q = pu.random_cache(batch, 2, D, int8, seed=7), _q(batch, 4, D, seed=8)
    _check(_run(q, cache, batch), q, cache, batch, weight_step=pu.half_step(BF) ** 2)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
def test_pages(page, D, int8):
    batch = Batch([(0, 19), (100, 7), (page - 1, 1), (page, 1), (2 * page - 3, 9)], page)
    cache, q = pu.random_cache(batch, 2, D, int8), _q(batch, 6, D)
    _check(_run(q, cache, batch), q, cache, batch)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 33, 100, 5000])
def test_window(window, D, int8):
    batch = Batch([(0, 40), (300, 1), (77, 50), (0, 1), (1000, 3)], 16)
    cache, q = pu.random_cache(batch, 2, D, int8), _q(batch, 4, D)
    _check(_run(q, cache, batch, window=window), q, cache, batch, window)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("sizes", [[(4999, 1)], [(3000, 1), (0, 1), (1000, 1), (9000, 1)], [(2000, 40), (6000, 3)], [(2047, 1), (2048, 1), (2049, 2)]])
@pytest.mark.parametrize("H,G,D", [(8, 2, 64), (5, 1, 128)])
def test_sequences_that_are_cut(H, G, D, sizes, int8):
    batch = Batch(sizes, 32)
    cache, q = pu.random_cache(batch, G, D, int8), _q(batch, H, D)
    _check(_run(q, cache, batch), q, cache, batch)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("D,window", [(64, 0), (128, 0), (64, 20000)])
def test_many_rows_over_many_keys(D, window, int8):
    """Parts of more than 16 blocks, of which heads of 64 have more: a sequence's 256 rows of each of 16 heads over 30056 keys."""
    G, n, L = 16, 256, 30056
    batch = Batch([(L - n, n)], 64)
    cache, q = pu.random_cache(batch, G, D, int8), _q(batch, G, D)
    got = _run(q, cache, batch, window=window).double()
    page, slot = batch.slots(0, torch.arange(L))
    positions, keys = torch.arange(L - n, L).cuda()[:, None], torch.arange(L).cuda()[None]
    unseen = (keys > positions) | ((keys <= positions - window) if window else False)
    for h in range(G):
        k, v = (pu.values(cache, which)[page, h, slot].cuda() for which in range(2))
        x = q[:, h].double().cuda()
        w = torch.softmax((x @ k.t().contiguous() * D ** -0.5).masked_fill(unseen, -math.inf), 1)
        want = w @ v
        scores_off = (D + 4) * 2.0 ** -24 * D ** -0.5 * float((x.abs() @ k.abs().t().contiguous()).max())
        step = pu.half_step(BF)
        bound = step * want.abs() + (step + 2 * scores_off + 2.0 ** -18) * (w @ v.abs()) + 2.0 ** -124 * v.abs().sum(0)
        assert bool(((got[:, h] - want).abs() <= bound).all()), h


@pytest.mark.parametrize("count", [65, 300])
def test_many_sequences(count):
    batch = Batch([(i * 7 % 90, i % 3) for i in range(count)], 16)
    cache, q = pu.random_cache(batch, 2, 64, False), _q(batch, 4, 64)
    _check(_run(q, cache, batch), q, cache, batch)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("alpha", [1e-3, 1.0, 30.0])
def test_scale(alpha, int8):
    batch = Batch([(50, 3), (700, 1)], 16)
    cache, q = pu.random_cache(batch, 1, 64, int8), _q(batch, 2, 64)
    _check(_run(q, cache, batch, alpha=alpha), q, cache, batch, alpha=alpha)


def test_rows_of_no_sequence_are_left():
    batch = Batch([(20, 3), (0, 5)], 16, ahead=3, behind=4)
    cache, q = pu.random_cache(batch, 2, 64, False), _q(batch, 4, 64)
    out = torch.full((batch.rows, 4, 64), 7.0, dtype=BF)
    got = _run(q, cache, batch, out=out)
    _check(got, q, cache, batch)
    assert bool((got[:3] == 7).all()) and bool((got[-4:] == 7).all())


@pytest.mark.parametrize("int8", [False, True])
def test_rows_that_see_nothing_are_zero(int8):
    """More new rows than the sequence has tokens: the first are at positions below 0."""
    batch = Batch([(-4, 9), (30, 2), (-3, 3)], 16)
    cache, q = pu.random_cache(batch, 2, 64, int8), _q(batch, 4, 64)
    got = _run(q, cache, batch)
    _check(got, q, cache, batch)
    assert bool((got[:4] == 0).all()) and bool((got[-3:] == 0).all())


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("old", [20, 900])
def test_what_a_row_does_not_see_has_no_part(old, bad):
    """Values and keys of later rows, of keys ahead of the window and of slots behind the sequence that are infinite or NaN."""
    batch = Batch([(old, 6), (40, 1)], 16)
    cache, q = pu.random_cache(batch, 2, 64, False), _q(batch, 4, 64)
    want, bound = pu.attention(q, cache, batch, 11)
    k, v = cache[0].clone(), cache[1].clone()
    page, slot = batch.slots(0, torch.tensor([old + 5]))    # the last row's own
    v[page, 0, slot, 3] = bad
    k[page, 1, slot, 3] = bad
    page, slot = batch.slots(0, torch.tensor([old - 11]))   # just ahead of every window
    v[page, :, slot] = bad
    k[page, :, slot] = bad
    tail = torch.arange(41, 48)                              # behind the second sequence, on its last page
    page, slot = batch.slots(1, tail)
    v[page, :, slot] = bad
    k[page, :, slot] = bad
    got = _run(q, (k, v, None, None), batch, window=11).double().cpu()
    rows = [0, 1, 2, 3, 4, 6]
    assert bool((got[rows] - want[rows]).abs().le(bound[rows]).all())
    assert not bool(got[5, :2, 3].isfinite().any())         # the row that sees it, the heads that share it
    keep = [d for d in range(64) if d != 3]
    assert bool((got[5, :2][:, keep] - want[5, :2][:, keep]).abs().le(bound[5, :2][:, keep]).all())


def _plan(batch, H, G, D, int8=False, window=0):
    import paper_2006_03031_amd as nb
    return nb.paged_attention_plan(batch.rows, len(batch.sizes), batch.pages.shape[1], H, G, batch.page, D, nb.I8 if int8 else nb.BF16, window)


CHUNKS = [[(0, 300), (0, 1), (1200, 129), (0, 0), (64, 64)], [(0, 128), (0, 127)], [(2000, 200)], [(0, 700), (30, 90), (-50, 150), (-40, 40)]]


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("window", [0, 1, 70, 128, 1500])
@pytest.mark.parametrize("H,G,D", [(2, 1, 64), (3, 1, 128), (4, 4, 64)])
@pytest.mark.parametrize("sizes", range(len(CHUNKS)))
def test_many_rows(sizes, H, G, D, window, int8):
    """128 rows a workgroup: tiles and waves that are partly or not at all filled, rows at positions below 0, a sequence without tokens."""
    batch = Batch(CHUNKS[sizes], 32, ahead=1, behind=2, extra_columns=40)
    assert _plan(batch, H, G, D, int8, window).kernel == (1 if not 0 < window <= 1000 else 0)
    cache, q = pu.random_cache(batch, G, D, int8), _q(batch, H, D)
    out = torch.full((batch.rows, H, D), 7.0, dtype=BF)
    got = _run(q, cache, batch, window=window, out=out)
    _check(got, q, cache, batch, window)
    assert bool((got[:1] == 7).all()) and bool((got[-2:] == 7).all())
    low = torch.tensor([r for _, r, p in batch.each() if p < 0], dtype=torch.int64)
    assert bool((got.cpu()[low] == 0).all())


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("old", [0, 1500])
def test_many_rows_and_what_they_do_not_see(old, bad):
    """An infinite or NaN key and value among the new ones: rows ahead of it are as without it, rows behind it are not finite where it counts."""
    batch = Batch([(old, 180), (old, 150)], 16, extra_columns=80)
    assert _plan(batch, 4, 2, 64).kernel == 1
    cache, q = pu.random_cache(batch, 2, 64, False), _q(batch, 4, 64)
    want, bound = pu.attention(q, cache, batch)
    page, slot = batch.slots(0, torch.tensor([old + 100]))
    cache[1][page, 0, slot, 5] = bad
    cache[0][page, 1, slot, 5] = bad
    got = _run(q, cache, batch).double().cpu()
    clean = list(range(100)) + list(range(180, 330))
    assert bool((got[clean] - want[clean]).abs().le(bound[clean]).all())
    seen = got[100:180]
    assert not bool(seen[:, :2, 5].isfinite().any()) and bool(seen[:, :2, :5].isfinite().all())
    # the other head's scores: NaN, or plus or minus infinity by the query's sign, which leaves its weights NaN or 0
    if math.isnan(bad):
        assert bool(seen[:, 2:].isnan().all())


def test_many_rows_and_nan_scales_of_hidden_keys():
    batch = Batch([(1100, 200)], 16)
    assert _plan(batch, 2, 1, 64, True).kernel == 1
    cache, q = pu.random_cache(batch, 1, 64, True), _q(batch, 2, 64)
    want, bound = pu.attention(q, cache, batch)
    page, slot = batch.slots(0, torch.tensor([1100 + 150]))
    cache[2][page, 0, slot] = math.nan
    cache[3][page, 0, slot] = math.nan
    got = _run(q, cache, batch).double().cpu()
    assert bool((got[:150] - want[:150]).abs().le(bound[:150]).all()) and bool(got[150:].isnan().all())


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("count,waves", [(1, 8), (300, 4)])
def test_the_tokens_workgroups(count, waves, D, int8):
    """Eight waves for few short tiles, four for many (and for bf16 heads of 128)."""
    batch = Batch([(700 - i, 1) for i in range(count)], 32)
    p = _plan(batch, 8, 4, D, int8)
    assert p.kernel == 0 and p.block == 64 * (4 if D == 128 and not int8 else waves)
    cache, q = pu.random_cache(batch, 4, D, int8), _q(batch, 8, D)
    got = _run(q, cache, batch)
    few = Batch(batch.sizes, 32)
    few.sizes = batch.sizes[:5]
    _check(got, q, cache, few)


@pytest.mark.parametrize("int8,D", [(False, 128), (True, 64)])
def test_walks_of_more_than_64_blocks_a_wave(int8, D):
    """Sequences so long that a wave looks its pages up more than once; the reference in 64 bits on the GPU."""
    from paper_2006_03031_amd import runtime as rt
    G, page, lengths = 16, 64, (150001, 149000) if int8 else (90001, 80000)
    W = -(-max(lengths) // page)
    shape = (2 * W, G, page, D)
    g = torch.Generator(device="cuda").manual_seed(2)
    if int8:
        cache = rt.PagedCache(*(torch.randint(-127, 128, shape, dtype=torch.int8, device="cuda", generator=g) for _ in "kv"),
                              *(torch.rand(shape[:3], device="cuda", generator=g) * 0.02 for _ in "kv"))
    else:
        cache = rt.PagedCache(*(torch.randn(shape, device="cuda", generator=g, dtype=BF) for _ in "kv"))
    pages = torch.randperm(2 * W, device="cuda", generator=g).to(torch.int32).view(2, W)
    q = torch.randn(2, G, D, device="cuda", generator=g, dtype=BF)
    seqs = rt.Sequences(torch.arange(3, device="cuda"), torch.tensor(lengths, device="cuda"), pages)
    got = rt.paged_attention(q, cache, seqs).double()
    half = pu.half_step(BF)
    for s, L in enumerate(lengths):
        j = torch.arange(L, device="cuda")
        for h in (0, 7, 15):
            at = pages[s].long()[j // page], h, j % page
            k, v = cache.k[at].double(), cache.v[at].double()
            if int8:
                k, v = k * cache.k_scale[at].double()[:, None], v * cache.v_scale[at].double()[:, None]
            terms = k * q[s, h].double()
            w = torch.softmax(terms.sum(1) * D ** -0.5, 0)
            want = (w[:, None] * v).sum(0)
            off = (D + 4) * 2.0 ** -24 * D ** -0.5 * float(terms.abs().sum(1).max())
            bound = half * want.abs() + (half + 2 * off + 2.0 ** -18) * (w[:, None] * v.abs()).sum(0)
            assert bool(((got[s, h] - want).abs() <= bound).all()), (s, h)


def test_pages_ahead_of_the_window_may_be_gone():
    batch = Batch([(500, 3)], 16)
    cache, q = pu.random_cache(batch, 2, 64, False), _q(batch, 4, 64)
    want, bound = pu.attention(q, cache, batch, 40)
    batch.pages[0, :(500 - 40) // 16] = -1
    got = _run(q, cache, batch, window=40).double().cpu()
    assert bool((got - want).abs().le(bound).all())


def test_nan_scales_of_hidden_keys():
    batch = Batch([(20, 4)], 16)
    cache, q = pu.random_cache(batch, 1, 64, True), _q(batch, 4, 64)
    want, bound = pu.attention(q, cache, batch)
    page, slot = batch.slots(0, torch.tensor([23]))
    cache[2][page, 0, slot] = math.nan
    cache[3][page, 0, slot] = math.nan
    got = _run(q, cache, batch).double().cpu()
    assert bool((got[:3] - want[:3]).abs().le(bound[:3]).all()) and bool(got[3].isnan().all())


def test_pages_out_of_range_stay_inside_the_cache():
    """Every access is held to the cache: rows of sequences whose pages are in range are as ever, the others' content is unspecified."""
    batch = Batch([(60, 2), (60, 2)], 16)
    cache, q = pu.random_cache(batch, 2, 64, False), _q(batch, 4, 64)
    want, bound = pu.attention(q, cache, batch)
    batch.pages[1, 1] = batch.count
    batch.pages[1, 2] = 2 ** 31 - 1
    batch.pages[1, 0] = -7
    got = _run(q, cache, batch).double().cpu()
    assert bool((got[:2] - want[:2]).abs().le(bound[:2]).all())


def test_lengths_beyond_the_page_table_are_held_to_it():
    batch = Batch([(60, 2)], 16, extra_columns=0)
    cache, q = pu.random_cache(batch, 2, 64, False), _q(batch, 4, 64)
    batch.lengths[0] = 1 << 40
    assert bool(_run(q, cache, batch).isfinite().all())
    batch.lengths[0] = -5
    assert bool((_run(q, cache, batch) == 0).all())


def test_queries_out_of_wider_rows():
    batch = Batch([(60, 5), (9, 1)], 16)
    cache = pu.random_cache(batch, 2, 64, False)
    rows = torch.randn(batch.rows, 9, 64, generator=torch.Generator().manual_seed(5)).to(BF)
    from paper_2006_03031_amd import runtime as rt
    q = rows[:, 1:7]
    got = rt.paged_attention(rows.cuda()[:, 1:7], pu.to_gpu(cache), batch.on_gpu())
    _check(got, q, cache, batch)


def test_same_bits_every_time_and_on_another_stream():
    from paper_2006_03031_amd import runtime as rt
    batch = Batch([(3000, 1), (0, 70), (900, 2)], 32)
    cache, q = pu.to_gpu(pu.random_cache(batch, 2, 128, False)), _q(batch, 8, 128).cuda()
    seqs = batch.on_gpu()
    first = rt.paged_attention(q, cache, seqs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = [rt.paged_attention(q, cache, seqs) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(first, x) for x in again)


def test_a_captured_call_follows_the_lengths():
    from paper_2006_03031_amd import runtime as rt
    batch = Batch([(4000, 1), (200, 1)], 32, extra_columns=0)
    cpu = pu.random_cache(batch, 2, 64, False)
    q = _q(batch, 4, 64)
    cache, seqs, qg = pu.to_gpu(cpu), batch.on_gpu(), q.cuda()
    rt.paged_attention(qg, cache, seqs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = rt.paged_attention(qg, cache, seqs)
    for lengths in ((4001, 201), (1, 201), (300, 7), (0, 150), (4001, 1)):
        batch.lengths = torch.tensor(lengths)
        seqs.lengths.copy_(batch.lengths)
        o.fill_(3.0)
        eager = rt.paged_attention(qg, cache, seqs)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager, o), lengths
        _check(o, q, cpu, batch)


def test_a_cache_past_4_gib():
    """Rows whose byte offsets pass 32 bits, in codes and in scales' neighbours."""
    from paper_2006_03031_amd import runtime as rt
    pages, G, page, D = 5 * 2 ** 30 // (8 * 64 * 128 * 2) + 3, 8, 64, 128
    k, v = (torch.empty(pages, G, page, D, dtype=BF, device="cuda") for _ in range(2))
    batch = Batch([(150, 2), (3, 1)], page, extra_columns=0)
    small = pu.random_cache(batch, G, D, False)
    high = pages - batch.count
    k[high:], v[high:] = small[0].cuda(), small[1].cuda()
    q = _q(batch, 8, D)
    seqs = batch.on_gpu()
    seqs.pages[seqs.pages >= 0] += high
    _check(rt.paged_attention(q.cuda(), rt.PagedCache(k, v), seqs), q, small, batch)


def test_nothing_to_do():
    from paper_2006_03031_amd import runtime as rt
    batch = Batch([(0, 0), (0, 0)], 16)
    cache = pu.to_gpu(pu.random_cache(batch, 2, 64, False))
    assert rt.paged_attention(torch.empty(0, 4, 64, dtype=BF, device="cuda"), cache, batch.on_gpu()).shape == (0, 4, 64)
    none = rt.Sequences(torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"),
                        torch.zeros(0, 0, dtype=torch.int32, device="cuda"))
    out = torch.full((2, 4, 64), 5.0, dtype=BF, device="cuda")
    assert bool((rt.paged_attention(torch.zeros(2, 4, 64, dtype=BF, device="cuda"), cache, none, out=out) == 5).all())
