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
