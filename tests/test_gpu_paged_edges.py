"""Calls of the paged cache's operators at the ends of their ranges, on the GPU."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paged_util as pu
from paged_util import BF, Batch


@pytest.mark.parametrize("rows", [2, 300])
def test_an_idle_step_with_a_table_of_full_width(rows):
    """No sequence, padded queries, pages [0, W] for many keys: nothing is written, eagerly, with a workspace or in a graph."""
    from paper_2006_03031_amd import runtime as rt
    cache = pu.to_gpu(pu.random_cache(Batch([(20, 1)], 16), 2, 64, False))
    none = rt.Sequences(torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"),
                        torch.zeros(0, 1000, dtype=torch.int32, device="cuda"))
    q = torch.zeros(rows, 4, 64, dtype=BF, device="cuda")
    out = torch.full_like(q, 5.0)
    for workspace in (None, torch.empty(64, dtype=torch.uint8, device="cuda")):
        for _ in range(2):  # (through the steps, then natively)
            assert rt.paged_attention(q, cache, none, out=out, workspace=workspace) is out
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out.add_(1.0)
        rt.paged_attention(q, cache, none, out=out)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert bool((out == 8).all())


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("sizes", [[(300, 1), (20, 3)], [(5000, 1), (100, 2)], [(1500, 200)]])
def test_a_window_beyond_all_positions_is_none(sizes, int8):
    from paper_2006_03031_amd import runtime as rt
    batch = Batch(sizes, 32)
    cache = pu.to_gpu(pu.random_cache(batch, 2, 64, int8))
    q = torch.randn(batch.rows, 4, 64, generator=torch.Generator().manual_seed(3)).to(BF).cuda()
    seqs = batch.on_gpu()
    want = rt.paged_attention(q, cache, seqs)
    for window in (1 << 30, 1 << 62, 2 ** 63 - 1):
        assert torch.equal(rt.paged_attention(q, cache, seqs, window=window), want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_scales_of_turned_keys_beyond_the_largest_number(interleaved, D):
    """Pairs of the largest bf16 turned by an eighth of a circle are 1.41 times it, more than f32 holds; their scale, a 127th of that, is not."""
    from paper_2006_03031_amd import runtime as rt
    batch = Batch([(0, 3)], 16)
    cache = pu.to_gpu(pu.random_cache(batch, 1, D, True))
    g = torch.Generator().manual_seed(1)
    most = torch.finfo(BF).max
    k = (torch.randint(-4, 5, (3, 1, D), generator=g) / 4 * most).to(BF)
    k[:, :, 0], k[:, :, 1], k[:, :, D // 2] = most, -most, -most
    table = torch.full((3, D // 2, 2), 0.5 ** 0.5)
    rt.cache_write(cache, k.cuda(), k.cuda(), batch.on_gpu(), table=table.cuda(), interleaved=interleaved)
    page, slot = batch.slots(0, torch.arange(3))
    for which, rows in ((0, pu.turned(k, table, interleaved)[0]), (1, k.double())):
        codes, scales = cache[which].cpu()[page, :, slot], cache[2 + which].cpu()[page, :, slot]
        top = rows.abs().amax(-1)
        assert bool(((scales.double() - top / 127).abs() <= 2 * 2.0 ** -24 * top / 127).all())   # (two roundings to f32 at most)
        assert bool(((codes.double() - 127 * rows / top[..., None]).abs() <= 0.5 + 1e-9).all())
    assert bool((pu.turned(k, table, interleaved)[0].abs().amax(-1) > torch.finfo(torch.float32).max).all())
    back = rt.cache_read(cache, batch.on_gpu(), 3, 1)[1]
    assert bool(back.isfinite().all())


def test_scales_that_no_number_holds():
    """A table whose magnitude takes a 127th of the keys beyond f32: as keys that are infinite, codes 0 and a scale that is NaN."""
    from paper_2006_03031_amd import runtime as rt
    batch = Batch([(0, 2)], 16)
    cache = pu.to_gpu(pu.random_cache(batch, 1, 64, True))
    k = torch.full((2, 1, 64), 1e30, dtype=BF)
    table = torch.tensor([1e12, 0.0]).expand(2, 32, 2).contiguous()
    rt.cache_write(cache, k.cuda(), k.cuda(), batch.on_gpu(), table=table.cuda())
    page, slot = batch.slots(0, torch.arange(2))
    assert bool((cache.k.cpu()[page, :, slot] == 0).all()) and bool(cache.k_scale.cpu()[page, :, slot].isnan().all())
    assert bool((cache.v.cpu()[page, :, slot] == 127).all()) and bool(cache.v_scale.cpu()[page, :, slot].isfinite().all())


def test_parts_of_one_buffer_that_do_not_overlap():
    """Outputs beside operands: heads of the same wider rows, in place, behind each other in one allocation."""
    import paper_2006_03031_amd as nb
    from paper_2006_03031_amd import runtime as rt
    batch = Batch([(40, 3), (0, 9)], 16)
    T, H, G, D = batch.rows, 4, 2, 64
    rows = torch.randn(T, 2 * H + 2 * G, D, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    q, k, v, y = rows.split([H, G, G, H], 1)
    table, positions = pu.angles(60, D).float().cuda(), torch.arange(T, device="cuda")
    for _ in range(2):  # (through the steps, then natively)
        want = rt.rotary(q.contiguous(), positions, table)
        assert rt.rotary(q, positions, table, out=y) is y and torch.equal(y, want)
        x = q.contiguous()
        assert rt.rotary(x, positions, table, out=x) is x and torch.equal(x, want)
        cache, seqs = pu.to_gpu(pu.random_cache(batch, G, D, False)), batch.on_gpu()
        turned = rt.cache_write(cache, k, v, seqs, q=q, table=table)
        one = torch.empty(2, T, H, D, dtype=BF, device="cuda")
        one[0] = q
        assert torch.equal(rt.cache_write(cache, k, v, seqs, q=one[0], table=table, out=one[0]), turned)
        one[0] = q
        assert torch.equal(rt.cache_write(cache, k, v, seqs, q=one[0], table=table, out=one[1]), turned)
        assert torch.equal(rt.paged_attention(one[1], cache, seqs, out=one[0]), rt.paged_attention(turned, cache, seqs))
        shared = rt.PagedCache(cache.k, cache.k)  # keys that are the values
        assert torch.equal(rt.paged_attention(turned, shared, seqs), rt.paged_attention(turned, rt.PagedCache(cache.k, cache.k.clone()), seqs))
        for call in (lambda: rt.paged_attention(turned, cache, seqs, out=turned), lambda: rt.cache_write(shared, k, v, seqs),
                     lambda: rt.cache_write(cache, k, v, seqs, q=one[0], out=one.view(-1, H, D)[1:T + 1]),
                     lambda: rt.cache_read(cache, seqs, T, out=(one[0, :, :G].contiguous(),) * 2)):
            with pytest.raises(nb.NimbleError) as e:
                call()
            assert e.value.code == -8 and "overlap" in str(e.value)
