"""Calls of the paged cache's operators at the ends of their ranges: what the host makes of them (no GPU needed)."""
import pytest

import paper_2006_03031_amd as nb

P = 4096  # an address that is never followed


def _cache(**kw):
    return nb.cache(**{**dict(k=P, v=P, k_scale=P, v_scale=P, pages=9, kv_heads=2, page=16, D=64, dtype=nb.BF16), **kw})


@pytest.mark.parametrize("kv_heads,D,dtype", [(2, 64, nb.BF16), (8, 128, nb.I8)])
@pytest.mark.parametrize("width", [0, 1, 80, 1000, 1 << 20])
@pytest.mark.parametrize("rows,count", [(7, 0), (1, 0), (500, 0), (1 << 20, 0), (0, 0), (0, 1), (0, 300)])
def test_batches_without_rows_or_sequences(rows, count, width, kv_heads, D, dtype):
    """An idle step of a server: padded rows, a page table of full width, no sequence.  Nothing is launched, no workspace is needed."""
    p = nb.paged_attention_plan(rows, count, width, 2 * kv_heads, kv_heads, 16, D, dtype)
    assert (p.parts, p.grid, p.join_grid, p.slots, p.workspace_bytes) == (0, 0, (0, 0), 0, 0)
    seqs = nb.sequences(P, P, P, count, width, rows)
    nb.nimble_paged_attention_dyn(P, 2 * kv_heads * D, _cache(kv_heads=kv_heads, D=D, dtype=dtype), seqs, 1 << 20, 2 * kv_heads, 0.125)


def test_batches_without_sequences_are_checked_all_the_same():
    for call, code in ((lambda: nb.paged_attention_plan(7, 0, 1000, 5, 2, 16, 64), -3), (lambda: nb.paged_attention_plan(7, 0, 1000, 4, 2, 16, 96), -8),
                       (lambda: nb.paged_attention_plan(7, 0, 1 << 27, 4, 2, 16, 64), -8),
                       (lambda: nb.paged_attention_plan(0, 0, 10, 4, 2, 16, 64, nb.BF16, -1), -8)):
        with pytest.raises(nb.NimbleError) as e:
            call()
        assert e.value.code == code


@pytest.mark.parametrize("rows,count,width", [(7, 2, 5), (7, 2, 1000), (4000, 3, 1 << 26), (64, 64, 20000)])
@pytest.mark.parametrize("window", [1 << 30, (1 << 30) + 1, 1 << 62, 2 ** 63 - 16, 2 ** 63 - 1])
def test_a_window_beyond_all_positions_is_none(window, rows, count, width):
    for D, dtype in ((64, nb.BF16), (128, nb.I8)):
        args = (rows, count, width, 4, 2, 16, D, dtype)
        assert nb.paged_attention_plan(*args, window) == nb.paged_attention_plan(*args, 0)
