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


# Every tensor 16 MB behind the one before; one of them moved onto another is refused.
AT = {name: (i + 1) << 24 for i, name in enumerate("ck cv cks cvs off len pages q k v out table pos ws y".split())}


def _rotary(at, xs=256, ys=256, T=7):
    return nb.nimble_rotary_dyn(at["q"], xs, at["pos"], at["table"], 100, at["y"], ys, T, 4, 64, 32, False)


def _write(at, qs=256):
    return nb.nimble_cache_write_dyn(_described(at), _batch(at), at["k"], 128, at["v"], 128, at["q"], qs, at["out"], 4, at["table"], 100, 32, False)


def _read(at):
    return nb.nimble_cache_read_dyn(_described(at), _batch(at), at["k"], at["v"], nb.F32)


def _attend(at):
    return nb.nimble_paged_attention_dyn(at["q"], 256, _described(at), _batch(at), at["out"], 4, 0.125, 0, at["ws"], 15 << 20)


def _described(at):
    return nb.cache(at["ck"], at["cv"], at["cks"], at["cvs"], 9, 2, 16, 64, nb.I8)


def _batch(at):
    return nb.sequences(at["off"], at["len"], at["pages"], 2, 1000, 7)


SHARED = [(_rotary, "y", ("pos", "table")), (_write, "out", ("k", "v", "table", "off", "len", "pages", "ck", "cv", "cks", "cvs")),
          (_write, "ck", ("q", "k", "v", "table", "off", "len", "pages", "cv", "cks", "cvs")), (_write, "cv", ("q", "k", "v", "table", "cvs")),
          (_write, "cks", ("q", "k", "v", "cvs")), (_write, "cvs", ("q", "k", "v")),
          (_read, "k", ("v", "ck", "cv", "cks", "cvs", "off", "len", "pages")), (_read, "v", ("ck", "cv", "cks", "cvs", "off", "len", "pages")),
          (_attend, "out", ("q", "ck", "cv", "cks", "cvs", "off", "len", "pages", "ws")),
          (_attend, "ws", ("q", "ck", "cv", "cks", "cvs", "off", "len", "pages"))]


@pytest.mark.parametrize("call,output,other", [(c, o, x) for c, o, others in SHARED for x in others])
def test_outputs_that_share_memory_are_refused(call, output, other):
    """Whatever begins in the output, and the other way round (the lengths are 16 bytes, behind which nothing is shared)."""
    for at in ({**AT, other: AT[output] + 16}, {**AT, output: AT[other]}):
        with pytest.raises(nb.NimbleError) as e:
            call(at)
        assert e.value.code == -8 and "overlap" in str(e.value)


@pytest.mark.parametrize("call,change,kw", [
    (_rotary, dict(y=AT["q"] + 2), {}), (_rotary, dict(y=AT["q"] + 6 * 512), {}), (_rotary, dict(y=AT["q"] + 512), dict(xs=512, ys=256)),
    (_rotary, dict(y=AT["q"] + 128), dict(xs=512, ys=512)), (_write, dict(out=AT["q"] + 16), {}), (_write, dict(out=AT["q"] - 512), {}),
    (_write, dict(out=AT["q"] + 512), dict(qs=1024)), (_write, dict(out=AT["q"], k=AT["q"] + 512), {}), (_write, dict(out=AT["q"], ck=AT["q"] - 512), {}),
    (_attend, dict(out=AT["q"]), {}), (_attend, dict(out=AT["q"] + 512), {})])
def test_rows_that_lie_over_each_other_are_refused(call, change, kw):
    with pytest.raises(nb.NimbleError) as e:
        call({**AT, **change}, **kw)
    assert e.value.code == -8 and "overlap" in str(e.value)


@pytest.mark.parametrize("rows,count,keys,heads,kv_heads,D,dtype,step", [
    (1, 1, 2000, 32, 8, 128, nb.BF16, 128), (1, 1, 4000, 32, 8, 128, nb.I8, 128), (1, 1, 2000, 16, 16, 64, nb.I8, 128), (4, 4, 2000, 8, 2, 64, nb.I8, 128),
    (1, 1, 8000, 32, 8, 128, nb.BF16, 256), (2, 2, 4000, 32, 8, 128, nb.I8, 256), (2, 1, 2000, 32, 8, 128, nb.I8, 256), (8, 1, 4000, 16, 16, 64, nb.I8, 256),
    (64, 64, 2000, 32, 8, 128, nb.I8, 256), (16, 1, 4000, 16, 16, 64, nb.BF16, 256)])
def test_steps_of_few_rows(rows, count, keys, heads, kv_heads, D, dtype, step):
    """Short ones where tiles have up to 4 rows, and spans are few."""
    p = nb.paged_attention_plan(rows, count, -(-keys // 16), heads, kv_heads, 16, D, dtype)
    assert (p.kernel, p.parts, p.step) == (0, 1, step)
