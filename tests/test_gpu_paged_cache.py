"""rotary, rotary_table, cache_write and cache_read against their formulas in 64 bits, and a layer of them together."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paged_util as pu
from paged_util import BF, Batch

F32_STEP = 2.0 ** -24


def _randn(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def _check_turned(got, x, rows, interleaved):
    """Half a step of bf16 of the result; three roundings of f32 of the products and their sum."""
    want, size = pu.turned(x, rows, interleaved)
    off = (got.double().cpu() - want).abs() - pu.half_step(BF) * want.abs() - 4 * F32_STEP * size
    assert bool((off <= 0).all()), float(off.max())
    R = rows.shape[1]
    assert torch.equal(got[..., 2 * R:].cpu(), x[..., 2 * R:])


@pytest.mark.parametrize("kw", [dict(), dict(factor=8.0), dict(factor=4.0, trained=2048.0, magnitude=1.14), dict(base=500000.0, factor=8.0,
                                trained=8192.0, low=1.0, high=4.0), dict(factor=2.0, trained=100.0, low=-1.0, high=0.5)])
@pytest.mark.parametrize("positions,rot", [(1, 2), (5, 64), (130001, 4), (1000, 128), (7, 0), (0, 64)])
def test_table(positions, rot, kw):
    """Half a step of f32 of the value, and of the angle's own error: position * f in 64 bits, whose f is off by a few 2^-52."""
    from paper_2006_03031_amd import runtime as rt
    got = rt.rotary_table(positions, rot, **kw).double().cpu()
    want = pu.angles(positions, rot, **kw)
    assert got.shape == want.shape
    bound = F32_STEP * want.abs() + positions * 2.0 ** -48 + 2.0 ** -50
    assert bool(((got - want).abs() <= bound).all())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 64, 64), (3, 5, 64, 32), (17, 12, 128, 128), (4, 3, 128, 16), (5, 2, 80, 48), (2, 3, 64, 0), (5, 2, 24, 16),
                                       (9, 3, 7, 6), (6, 2, 33, 20), (4, 1, 2, 2), (3, 2, 72, 24), (300, 16, 64, 64)])
def test_rotary(T, H, D, rot, interleaved):
    from paper_2006_03031_amd import runtime as rt
    x = _randn(T, H, D).to(BF)
    table = pu.angles(50, rot, magnitude=1.2).float()
    positions = torch.arange(T) * 13 % 50
    got = rt.rotary(x.cuda(), positions.cuda(), table.cuda(), interleaved=interleaved)
    _check_turned(got, x, table[positions], interleaved)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("H,D,first,wide", [(4, 64, 2, 9), (3, 40, 1, 5), (3, 7, 1, 6)])
def test_rotary_parts_of_rows_and_in_place(H, D, first, wide, interleaved):
    from paper_2006_03031_amd import runtime as rt
    rows = _randn(11, wide, D).to(BF)
    table, positions = pu.angles(90, D // 2 // 2 * 2).float(), torch.arange(11) * 8
    dev = rows.cuda()
    part = dev[:, first:first + H]
    got = rt.rotary(part, positions.cuda(), table.cuda(), interleaved=interleaved, out=part)
    assert got is part
    _check_turned(part, rows[:, first:first + H], table[positions], interleaved)
    rows[:, first:first + H] = part.cpu()
    assert torch.equal(dev.cpu(), rows)


def test_rotary_of_addresses_of_two_bytes():
    from paper_2006_03031_amd import runtime as rt
    flat = _randn(5 * 2 * 64 + 1).to(BF)
    table, positions = pu.angles(90, 64).float(), torch.arange(5) * 8
    out = torch.zeros(5 * 2 * 64 + 3, dtype=BF, device="cuda")
    got = rt.rotary(flat.cuda()[1:].view(5, 2, 64), positions.cuda(), table.cuda(), out=out[3:].view(5, 2, 64))
    _check_turned(got, flat[1:].view(5, 2, 64), table[positions], False)


def test_rotary_holds_positions_to_the_table():
    from paper_2006_03031_amd import runtime as rt
    x, table = _randn(3, 2, 64).to(BF), pu.angles(10, 64).float()
    got = rt.rotary(x.cuda(), torch.tensor([-3, 1 << 40, 9]).cuda(), table.cuda())
    _check_turned(got, x, table[[0, 9, 9]], False)


def test_rotary_past_4_gib():
    from paper_2006_03031_amd import runtime as rt
    T, H, D = 2 ** 31 // (64 * 64) + 5, 64, 64
    x = torch.zeros(T, H, D, dtype=BF, device="cuda")
    some = _randn(3, H, D).to(BF)
    x[-3:] = some.cuda()
    table = pu.angles(7, 64).float()
    positions = torch.arange(T, device="cuda") % 7
    got = rt.rotary(x, positions, table.cuda(), out=x)
    _check_turned(got[-3:], some, table[positions[-3:].cpu()], False)


SIZES = [[(0, 1)], [(5, 3), (0, 0), (31, 1), (15, 2)], [(100, 1), (0, 50), (16, 16)]]


def _write(batch, cache, k, v, q, table, interleaved, **kw):
    from paper_2006_03031_amd import runtime as rt
    gpu = pu.to_gpu(cache)
    dev = [None if t is None else t.cuda() for t in (k, v, q, table)]
    out = rt.cache_write(gpu, dev[0], dev[1], batch.on_gpu(), q=dev[2], table=dev[3], interleaved=interleaved, **kw)
    return out, tuple(None if t is None else t.cpu() for t in gpu)


def _expect(batch, cache, k, v, rows, interleaved, got):
    """Where nothing was written the bits of before; keys and values as rounded or quantised from 64 bits."""
    int8 = cache[2] is not None
    want = tuple(None if t is None else t.clone() for t in cache)
    written = torch.zeros(cache[0].shape[:3], dtype=torch.bool)
    for s, row, p in batch.each():
        if p < 0 or p >= batch.pages.shape[1] * batch.page or not 0 <= int(batch.pages[s, p // batch.page]) < batch.count:
            continue
        page, slot = int(batch.pages[s, p // batch.page]), p % batch.page
        written[page, :, slot] = True
        for which, x in ((0, k[row:row + 1]), (1, v[row:row + 1])):
            y = x.double()
            if which == 0 and rows is not None:
                y, size = pu.turned(x, rows[row:row + 1], interleaved)
            if int8:
                codes, scales = pu.quantized(y)
                assert torch.equal(got[which][page, :, slot], codes[0]), (s, row, which)
                # a / 127 in f32 from a rounded to f32: two roundings
                close = (got[2 + which][page, :, slot].double() - scales[0].double()).abs() <= 2 * F32_STEP * scales[0].double()
                assert bool((close | (scales[0].isnan() & got[2 + which][page, :, slot].isnan())).all())
            elif which == 0 and rows is not None:
                _check_turned(got[0][page, :, slot][None], x, rows[row:row + 1], interleaved)
            else:
                assert torch.equal(got[which][page, :, slot], x[0])
    for which in range(4):
        if want[which] is not None:
            assert torch.equal(got[which][~written], want[which][~written])


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 16), (128, 128), (128, 64), (128, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("sizes", range(len(SIZES)))
@pytest.mark.parametrize("H,G", [(4, 4), (25, 3)])
def test_write(H, G, sizes, interleaved, D, rot, int8):
    batch = Batch(SIZES[sizes], 16, ahead=1, behind=2)
    cache = pu.random_cache(batch, G, D, int8)
    k, v, q = (_randn(batch.rows, n, D, seed=i).to(BF) for i, n in enumerate((G, G, H)))
    k[0] = 0
    table = pu.angles(120, rot, magnitude=1.1).float() if rot else None
    out = torch.full_like(q, 9.0)
    got_q, got = _write(batch, cache, k, v, q, table, interleaved, out=out.cuda())
    positions = torch.zeros(batch.rows, dtype=torch.int64)
    for _, row, p in batch.each():
        positions[row] = p
    rows = table[positions] if rot else None
    _expect(batch, cache, k, v, rows, interleaved, got)
    mine = [r for _, r, _ in batch.each()]
    if rot:
        _check_turned(got_q[mine], q[mine], rows[mine], interleaved)
    else:
        assert torch.equal(got_q[mine].cpu(), q[mine])
    assert bool((got_q[:1] == 9).all()) and bool((got_q[-2:] == 9).all())


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("H,G,D", [(33, 16, 128), (64, 64, 64), (300, 5, 128)])
def test_few_rows_of_many_heads_are_written_by_several_workgroups(H, G, D, int8):
    test_write(H, G, 0, False, D, D, int8)
    test_write(H, G, len(SIZES) - 1, True, D, 16, int8)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("D,G", [(128, 41), (64, 100)])
def test_few_rows_of_many_heads_are_read_by_several_workgroups(D, G, int8):
    test_read(D, G, 16, False, int8)


@pytest.mark.parametrize("int8", [False, True])
def test_write_without_queries_and_rows_without_a_place(int8):
    batch = Batch([(40, 3), (-2, 5), (20, 2), (30, 4)], 16, extra_columns=0)
    batch.pages[0, 2] = -1                   # dropped
    batch.pages[2, 1] = batch.count          # not one of the cache's
    batch.lengths[3] = 10 ** 12              # held to the page table
    cache = pu.random_cache(batch, 2, 64, int8)
    k, v = (_randn(batch.rows, 2, 64, seed=i).to(BF) for i in range(2))
    got_q, got = _write(batch, cache, k, v, None, None, False)
    assert got_q is None
    batch.lengths[3] = batch.pages.shape[1] * 16
    _expect(batch, cache, k, v, None, False, got)


def test_codes_are_those_of_quantize_rows():
    """Ties, zeros, tiny and huge heads, infinities and NaN."""
    from paper_2006_03031_amd import runtime as rt
    batch = Batch([(0, 40)], 16)
    k = _randn(40, 3, 64).to(BF)
    k[1] = 0
    k[2] = (torch.arange(64) - 31.5).to(BF)          # 127 x / a: many of them halves
    k[3] *= 1e-38
    k[4] *= 1e38
    k[5, 1, 7] = math.inf
    k[6, 0, 3] = math.nan
    k[7] = torch.randint(-127, 128, (3, 64)).to(BF) / 2
    k[8] = k[8].sign() * 2.0 ** -133                 # subnormal
    cache = pu.random_cache(batch, 3, 64, True)
    _, got = _write(batch, cache, k, k, None, None, False)
    codes, scales = rt.quantize_rows(k.view(120, 64).cuda(), 64)
    page, slot = batch.slots(0, torch.arange(40))
    for which in (0, 1):
        assert torch.equal(got[which][page, :, slot], codes.view(40, 3, 64).cpu())
        mine, theirs = got[2 + which][page, :, slot], scales.view(40, 3).cpu()
        assert torch.equal(mine.view(torch.int32)[~mine.isnan()], theirs.view(torch.int32)[~theirs.isnan()])
        assert torch.equal(mine.isnan(), theirs.isnan())


def test_write_of_parts_of_rows_with_queries_in_place():
    from paper_2006_03031_amd import runtime as rt
    batch = Batch([(5, 6), (0, 1)], 16)
    rows = _randn(batch.rows, 8 + 2 + 2, 64).to(BF)
    dev = rows.cuda()
    table = pu.angles(20, 64).float()
    cache = pu.random_cache(batch, 2, 64, False)
    q = rt.cache_write(gpu := pu.to_gpu(cache), dev[:, 8:10], dev[:, 10:], batch.on_gpu(), q=dev[:, :8], table=table.cuda())
    positions = torch.tensor([p for _, _, p in batch.each()])
    _check_turned(q, rows[:, :8], table[positions], False)
    _expect(batch, cache, rows[:, 8:10], rows[:, 10:], table[positions], False, tuple(None if t is None else t.cpu() for t in gpu))
    assert torch.equal(dev.cpu(), rows)
    own = rows[:, :8].contiguous().cuda()
    back = rt.cache_write(gpu, dev[:, 8:10], dev[:, 10:], batch.on_gpu(), q=own, table=table.cuda(), out=own)
    assert back is own and torch.equal(own, q)


def test_bf16_keys_are_those_of_rotary():
    from paper_2006_03031_amd import runtime as rt
    batch = Batch([(7, 30)], 32)
    k = _randn(30, 2, 128).to(BF).cuda()
    table = rt.rotary_table(40, 128)
    cache = rt.PagedCache.empty(batch.count, 2, 32, 128)
    seqs = batch.on_gpu()
    q = rt.cache_write(cache, k, k, seqs, q=k, table=table)
    want = rt.rotary(k, torch.arange(7, 37, device="cuda"), table)
    got, v = rt.cache_read(cache, seqs, 30)
    assert torch.equal(got, want) and torch.equal(q, want) and torch.equal(v, k)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("D,G,page", [(64, 12, 16), (128, 3, 64), (64, 1, 1024), (128, 17, 32)])
def test_read(D, G, page, f32, int8):
    import paper_2006_03031_amd as nb
    from paper_2006_03031_amd import runtime as rt
    batch = Batch([(0, 37), (0, 0), (9, 3), (-2, 4), (0, page + 1)], page, ahead=2, behind=1)
    cache = pu.random_cache(batch, G, D, int8)
    dtype = torch.float32 if f32 else BF
    out = tuple(torch.full((batch.rows, G, D), 9.0, dtype=dtype, device="cuda") for _ in "kv")
    got = rt.cache_read(pu.to_gpu(cache), batch.on_gpu(), batch.rows, nb.F32 if f32 else nb.BF16, out=out)
    left = torch.ones(batch.rows, dtype=torch.bool)
    for which in range(2):
        assert got[which] is out[which]
        x = cache[which].float() * (cache[2 + which][..., None] if int8 else 1)
        for s, row, p in batch.each():
            if p >= 0:
                pg, slot = batch.slots(s, p)
                left[row] = False
                assert torch.equal(got[which][row].cpu(), x[pg, :, slot].to(dtype))
        assert bool((got[which][left.cuda()] == 9).all())


@pytest.mark.parametrize("count", [64, 65, 4096, 4097, 5000])
def test_rows_find_their_sequence_among_many(count):
    """Sequences are looked for 64 at a time, over one, two or three steps."""
    from paper_2006_03031_amd import runtime as rt
    batch = Batch([(0, i % 3) for i in range(count)], 16, ahead=3)
    cache = rt.PagedCache.empty(batch.count, 1, 16, 64)
    k = torch.arange(batch.rows * 64, device="cuda").view(batch.rows, 1, 64).to(BF)
    seqs = batch.on_gpu()
    rt.cache_write(cache, k, -k, seqs)
    got, v = rt.cache_read(cache, seqs, batch.rows)
    assert torch.equal(got[3:], k[3:]) and torch.equal(v[3:], -k[3:])
    want = torch.full((batch.count, 1, 16), False)
    for s, _, p in batch.each():
        want[int(batch.pages[s, 0]), 0, p] = True
    first = torch.tensor([(int(batch.pages[s, 0]), row) for s, row, p in batch.each() if p == 0])
    assert torch.equal(cache.k[first[:, 0].cuda(), 0, 0], k[first[:, 1].cuda(), 0])


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("count,most", [(40, 500), (70, 300), (64, 2300)])
def test_workgroups_of_several_rows(count, most, int8):
    """Batches of so many rows that a workgroup takes 2 to 16 of them: rows of several sequences, of none, and without a place beside each other."""
    import paper_2006_03031_amd as nb
    from paper_2006_03031_amd import runtime as rt
    g = torch.Generator().manual_seed(count)
    new = torch.randint(0, most, (count,), generator=g).tolist()
    batch = Batch([(0, n) for n in new], 64, ahead=5, behind=11)
    assert batch.rows > 8192
    batch.pages[3, 1] = -1                                    # rows 64 .. 127 of one sequence are dropped
    assert new[3] > 70
    cache = pu.to_gpu(pu.random_cache(batch, 1, 64, int8))
    before = [None if t is None else t.clone() for t in cache]
    k, v, q = (torch.randn(batch.rows, n, 64, generator=g).to(BF).cuda() for n in (1, 1, 3))
    seqs = batch.on_gpu()
    out = torch.full_like(q, 9.0)
    table = pu.angles(most, 32).float().cuda()
    rt.cache_write(cache, k, v, seqs, q=q, table=table, out=out)
    positions = torch.zeros(batch.rows, dtype=torch.int64)
    mine = torch.zeros(batch.rows, dtype=torch.bool)
    placed = mine.clone()
    for s, row, p in batch.each():
        positions[row], mine[row], placed[row] = p, True, int(batch.pages[s, p // 64]) >= 0
    want_q, want_k = (rt.rotary(t, positions.cuda(), table) for t in (q, k))
    mine, placed = mine.cuda(), placed.cuda()
    assert torch.equal(out[mine], want_q[mine]) and bool((out[~mine] == 9).all())
    filled = tuple(torch.full((batch.rows, 1, 64), 9.0, dtype=BF, device="cuda") for _ in "kv")
    got_k, got_v = rt.cache_read(cache, seqs, batch.rows, out=filled)
    assert bool((got_k[~placed] == 9).all()) and bool((got_v[~placed] == 9).all())
    if int8:
        # half a step of the code, and the roundings of the scale, the product and the bf16 result
        for got, want in ((got_k, want_k), (got_v, v)):
            top = want[placed].float().abs().amax(-1, keepdim=True)
            assert bool(((got - want)[placed].float().abs() <= top * (0.5 / 127 + 3 * pu.half_step(BF))).all())
    else:
        assert torch.equal(got_k[placed], want_k[placed]) and torch.equal(got_v[placed], v[placed])
    used = torch.zeros(batch.count, 64, dtype=torch.bool)
    for s, _, p in batch.each():
        if int(batch.pages[s, p // 64]) >= 0:
            used[int(batch.pages[s, p // 64]), p % 64] = True
    for a, b in zip(cache, before):
        if a is not None:
            assert torch.equal(a[:, 0].cpu()[~used], b[:, 0].cpu()[~used])


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("window", [0, 20])
def test_a_decoder_layer_in_chunks_is_the_layer_at_once(int8, window):
    """A prompt through dense, cache_write and paged_attention as one batch, and the same tokens a few at a time, at the end one by one as
    replays of one captured step: either way the rows are those of the formula in 64 bits on what the cache holds."""
    import paper_2006_03031_amd as nb
    from paper_2006_03031_amd import runtime as rt
    H, G, D, page, L = 6, 2, 64, 16, 75
    g = torch.Generator().manual_seed(0)
    w = (torch.randn((H + 2 * G) * D, 128, generator=g) * 0.1).to(BF).cuda()
    x = torch.randn(L, 128, generator=g).to(BF).cuda()
    table = rt.rotary_table(128, D)

    def fresh():
        return rt.PagedCache.empty(9, G, page, D, nb.I8 if int8 else nb.BF16)

    def step(rows, cache, seqs):
        qkv = rt.dense(rows, w, None, nb.EPI_NONE).view(-1, H + 2 * G, D)
        q = rt.cache_write(cache, qkv[:, H:H + G], qkv[:, H + G:], seqs, q=qkv[:, :H], table=table)
        return q, rt.paged_attention(q, cache, seqs, window=window)

    whole = Batch([(0, L)], page, seed=4)
    cache = fresh()
    q, o = step(x, cache, whole.on_gpu())
    cpu = tuple(None if t is None else t.cpu() for t in cache)
    want, bound = pu.attention(q.cpu(), cpu, whole, window)
    assert bool(((o.double().cpu() - want).abs() <= bound).all())

    parts = fresh()
    got, at = [], 0
    for n in (40, 1, 17, 7):
        chunk = Batch([(at, n)], page, seed=4)
        chunk.pages = whole.pages
        got.append(step(x[at:at + n], parts, chunk.on_gpu()))
        at += n
    one = rt.Sequences(torch.tensor([0, 1]).cuda(), torch.tensor([at + 1]).cuda(), whole.pages.cuda())
    row = x[at:at + 1].clone()
    step(row, parts, one)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(row, parts, one)
    while at < L:
        row.copy_(x[at:at + 1])
        one.lengths.fill_(at + 1)
        graph.replay()
        got.append(tuple(t.clone() for t in out))
        at += 1
    torch.cuda.synchronize()
    # (a row sees what was written up to its own step, and nothing of that is written again)
    cpu = tuple(None if t is None else t.cpu() for t in parts)
    want, bound = pu.attention(torch.cat([q for q, _ in got]).cpu(), cpu, whole, window)
    assert bool(((torch.cat([o for _, o in got]).double().cpu() - want).abs() <= bound).all())
    # the same keys and values as at once, up to dense's order of sums, which another number of rows may change by a step of bf16 (2^-7 of the
    # value), of what a turn adds up twice that of the head's largest; a code in 8 bits by one, 2^-6 of the largest covers it and its scale
    used = whole.slots(0, torch.arange(L))
    for which in (0, 1):
        a, b = (pu.values(tuple(None if t is None else t.cpu() for t in c), which)[used[0], :, used[1]] for c in (cache, parts))
        assert bool(((a - b).abs() <= 2.0 ** -6 * a.abs().amax(-1, keepdim=True)).all())
