"""Shape functions, refusals and the dispatch of rotary, cache_write, cache_read and paged_attention (no GPU needed)."""
import ctypes
import math
import os
import random
import re
import shutil
import subprocess

import pytest

import paper_2006_03031_amd as nb
from paper_2006_03031_amd import binding

torch = pytest.importorskip("torch")

CACHE = (9, 2, 16, 64)


def test_shapes():
    assert nb.rotary_shape((7, 4, 80), (7,), (100, 40, 2)) == (7, 4, 80)
    assert nb.rotary_shape((0, 4, 80), (0,), (0, 0, 2)) == (0, 4, 80)
    nb.cache_check(CACHE, CACHE, None, None, nb.BF16, (4,), (3,), (3, 5))
    nb.cache_check(CACHE, CACHE, CACHE[:3], CACHE[:3], nb.I8, (1,), (0,), (0, 0))
    assert nb.cache_write_shape(CACHE, (7, 2, 64), (7, 2, 64)) is None
    assert nb.cache_write_shape(CACHE, (7, 2, 64), (7, 2, 64), (7, 6, 64)) == (7, 6, 64)
    assert nb.cache_read_shape(CACHE, 11) == (11, 2, 64)
    assert nb.paged_attention_shape((7, 6, 64), CACHE) == (7, 6, 64)


@pytest.mark.parametrize("call,code", [
    (lambda: nb.rotary_shape((7, 80), (7,), (100, 40, 2)), -2),
    (lambda: nb.rotary_shape((7, 4, 80), (7, 1), (100, 40, 2)), -2),
    (lambda: nb.rotary_shape((7, 4, 80), (6,), (100, 40, 2)), -3),
    (lambda: nb.rotary_shape((7, 4, 80), (7,), (100, 41, 2)), -3),
    (lambda: nb.rotary_shape((7, 4, 80), (7,), (100, 40, 1)), -3),
    (lambda: nb.rotary_shape((-7, 4, 80), (7,), (100, 40, 2)), -8),
    (lambda: nb.cache_check(CACHE, CACHE, None, None, nb.F32, (4,), (3,), (3, 5)), -4),
    (lambda: nb.cache_check(CACHE, CACHE, None, None, nb.I8, (4,), (3,), (3, 5)), -1),
    (lambda: nb.cache_check(CACHE[1:], CACHE, None, None, nb.BF16, (4,), (3,), (3, 5)), -2),
    (lambda: nb.cache_check(CACHE, (9, 2, 32, 64), None, None, nb.BF16, (4,), (3,), (3, 5)), -3),
    (lambda: nb.cache_check(CACHE, CACHE, CACHE[:3], (9, 2, 15), nb.I8, (4,), (3,), (3, 5)), -3),
    (lambda: nb.cache_check(CACHE, CACHE, CACHE, CACHE, nb.I8, (4,), (3,), (3, 5)), -2),
    (lambda: nb.cache_check(CACHE, CACHE, None, None, nb.BF16, (3,), (3,), (3, 5)), -3),
    (lambda: nb.cache_check(CACHE, CACHE, None, None, nb.BF16, (4,), (3,), (4, 5)), -3),
    (lambda: nb.cache_check(CACHE, CACHE, None, None, nb.BF16, (4,), (3,), (15,)), -2),
    (lambda: nb.cache_check(CACHE, CACHE, None, None, nb.BF16, (4,), (3,), (3, 1 << 27)), -8),
    (lambda: nb.cache_check((9, 2, 24, 64), (9, 2, 24, 64), None, None, nb.BF16, (4,), (3,), (3, 5)), -8),
    (lambda: nb.cache_check((9, 2, 8, 64), (9, 2, 8, 64), None, None, nb.BF16, (4,), (3,), (3, 5)), -8),
    (lambda: nb.cache_check((9, 2, 16, 80), (9, 2, 16, 80), None, None, nb.BF16, (4,), (3,), (3, 5)), -8),
    (lambda: nb.cache_check((9, 0, 16, 64), (9, 0, 16, 64), None, None, nb.BF16, (4,), (3,), (3, 5)), -8),
    (lambda: nb.cache_write_shape(CACHE, (7, 3, 64), (7, 3, 64)), -3),
    (lambda: nb.cache_write_shape(CACHE, (7, 2, 64), (8, 2, 64)), -3),
    (lambda: nb.cache_write_shape(CACHE, (7, 128), (7, 128)), -2),
    (lambda: nb.cache_write_shape(CACHE, (7, 2, 64), (7, 2, 64), (6, 4, 64)), -3),
    (lambda: nb.cache_write_shape(CACHE, (7, 2, 64), (7, 2, 64), (7, 4, 128)), -3),
    (lambda: nb.cache_write_shape(CACHE, (7, 2, 64), (7, 2, 64), ()), -2),
    (lambda: nb.cache_read_shape(CACHE, -1), -8),
    (lambda: nb.paged_attention_shape((7, 6, 128), CACHE), -3),
    (lambda: nb.paged_attention_shape((7, 5, 64), CACHE), -3),
    (lambda: nb.paged_attention_shape((7, 0, 64), CACHE), -3),
    (lambda: nb.paged_attention_shape((7, 384), CACHE), -2),
    (lambda: nb.paged_attention_plan(7, 2, 5, 5, 2, 16, 64), -3),
    (lambda: nb.paged_attention_plan(7, 2, 5, 0, 2, 16, 64), -8),
    (lambda: nb.paged_attention_plan(7, 2, 5, 4, 2, 16, 96), -8),
    (lambda: nb.paged_attention_plan(7, 2, 5, 4, 2, 2048, 64), -8),
    (lambda: nb.paged_attention_plan(7, 2, 5, 4, 2, 16, 64, nb.F32), -4),
    (lambda: nb.paged_attention_plan(7, 2, 5, 4, 2, 16, 64, nb.BF16, -1), -8),
    (lambda: nb.paged_attention_plan(-1, 2, 5, 4, 2, 16, 64), -8),
    (lambda: nb.paged_attention_plan(1 << 25, 2, 5, 4, 2, 16, 64), -8),
    (lambda: nb.paged_attention_plan(7, 1 << 17, 5, 4, 2, 16, 64), -8),
    (lambda: nb.paged_attention_plan(1 << 24, 2, 5, 128, 2, 16, 64), -8),
])
def test_refused_shapes(call, code):
    with pytest.raises(nb.NimbleError) as e:
        call()
    assert e.value.code == code


# Refused on the host before anything is launched: no GPU is needed to see it.  Pointers are numbers that are never followed.
P = 4096


def _cache(**kw):
    return nb.cache(**{**dict(k=P, v=P, k_scale=P, v_scale=P, pages=9, kv_heads=2, page=16, D=64, dtype=nb.BF16), **kw})


def _seqs(**kw):
    return nb.sequences(**{**dict(offsets=P, lengths=P, pages=P, count=2, width=5, rows=7), **kw})


TABLE = dict(t=P, n=5, rot=64, base=1e4, factor=1.0, trained=0.0, low=1.0, high=32.0, m=1.0)
ROTARY = dict(x=P, xs=256, p=P, t=P, rows=9, y=P, ys=256, T=7, H=4, D=64, R=32, i=0)
WRITE = dict(c=_cache(), s=_seqs(), k=P, ks=128, v=P, vs=128, q=P, qs=256, o=2 * P, heads=4, t=P, rows=9, R=32, i=0)
READ = dict(c=_cache(), s=_seqs(), k=P, v=P, t=0)
ATTENTION = dict(q=P, qs=256, c=_cache(), s=_seqs(), o=P, heads=4, alpha=0.125, window=0, ws=P, n=1 << 30)
LONG = dict(s=_seqs(width=1000))
CACHES = [(dict(c=_cache(k=0)), -1), (dict(c=_cache(v=P + 8)), -5), (dict(c=_cache(dtype=nb.I8, k_scale=0)), -1), (dict(c=_cache(dtype=nb.F32)), -4),
          (dict(c=_cache(D=32)), -8), (dict(c=_cache(page=48)), -8), (dict(c=_cache(pages=-1)), -8), (dict(c=_cache(dtype=nb.I8, v_scale=P + 4)), -5),
          (dict(s=_seqs(offsets=0)), -1), (dict(s=_seqs(lengths=P + 4)), -5), (dict(s=_seqs(pages=0)), -1), (dict(s=_seqs(pages=P + 2)), -5),
          (dict(s=_seqs(rows=-1)), -8), (dict(s=_seqs(rows=1 << 25)), -8), (dict(s=_seqs(width=1 << 27)), -8), (dict(c=None), -1), (dict(s=None), -1)]


@pytest.mark.parametrize("name,good,wrong,code", [
    ("nimble_rotary_table_dyn", TABLE, dict(t=0), -1),
    ("nimble_rotary_table_dyn", TABLE, dict(t=P + 8), -5),
    ("nimble_rotary_table_dyn", TABLE, dict(rot=3), -8),
    ("nimble_rotary_table_dyn", TABLE, dict(n=-1), -8),
    ("nimble_rotary_table_dyn", TABLE, dict(base=0.0), -8),
    ("nimble_rotary_table_dyn", TABLE, dict(factor=-1.0), -8),
    ("nimble_rotary_table_dyn", TABLE, dict(high=1.0), -8),
    ("nimble_rotary_table_dyn", TABLE, dict(trained=math.nan), -8),
    ("nimble_rotary_table_dyn", TABLE, dict(m=math.inf), -8),
    ("nimble_rotary_dyn", ROTARY, dict(R=33), -3),
    ("nimble_rotary_dyn", ROTARY, dict(T=-1), -8),
    ("nimble_rotary_dyn", ROTARY, dict(x=0), -1),
    ("nimble_rotary_dyn", ROTARY, dict(p=0), -1),
    ("nimble_rotary_dyn", ROTARY, dict(t=0), -1),
    ("nimble_rotary_dyn", ROTARY, dict(rows=0), -3),
    ("nimble_rotary_dyn", ROTARY, dict(x=P + 1), -5),
    ("nimble_rotary_dyn", ROTARY, dict(t=P + 4), -5),
    ("nimble_rotary_dyn", ROTARY, dict(xs=255), -8),
    ("nimble_rotary_dyn", ROTARY, dict(ys=-256), -8),
    ("nimble_rotary_dyn", ROTARY, dict(xs=512), -8),       # in place with two strides
    ("nimble_rotary_dyn", ROTARY, dict(H=1 << 20, D=1 << 20), -8),
    *[("nimble_cache_write_dyn", WRITE, *x) for x in CACHES],
    ("nimble_cache_write_dyn", WRITE, dict(k=0), -1),
    ("nimble_cache_write_dyn", WRITE, dict(o=0), -1),
    ("nimble_cache_write_dyn", WRITE, dict(v=P + 8), -5),
    ("nimble_cache_write_dyn", WRITE, dict(ks=120), -8),
    ("nimble_cache_write_dyn", WRITE, dict(vs=132), -8),
    ("nimble_cache_write_dyn", WRITE, dict(qs=128), -8),
    ("nimble_cache_write_dyn", WRITE, dict(R=33), -3),
    ("nimble_cache_write_dyn", WRITE, dict(R=20), -8),
    ("nimble_cache_write_dyn", WRITE, dict(rows=0), -3),
    ("nimble_cache_write_dyn", WRITE, dict(t=P + 8), -5),
    ("nimble_cache_write_dyn", WRITE, dict(o=P, qs=512), -8),
    *[("nimble_cache_read_dyn", READ, *x) for x in CACHES],
    ("nimble_cache_read_dyn", READ, dict(t=3), -4),
    ("nimble_cache_read_dyn", READ, dict(k=0), -1),
    ("nimble_cache_read_dyn", READ, dict(v=P + 2), -5),
    *[("nimble_paged_attention_dyn", ATTENTION, *x) for x in CACHES],
    ("nimble_paged_attention_dyn", ATTENTION, dict(q=0), -1),
    ("nimble_paged_attention_dyn", ATTENTION, dict(o=0), -1),
    ("nimble_paged_attention_dyn", ATTENTION, dict(o=P + 8), -5),
    ("nimble_paged_attention_dyn", ATTENTION, dict(qs=250), -8),
    ("nimble_paged_attention_dyn", ATTENTION, dict(heads=5), -3),
    ("nimble_paged_attention_dyn", ATTENTION, dict(alpha=0.0), -8),
    ("nimble_paged_attention_dyn", ATTENTION, dict(alpha=math.nan), -8),
    ("nimble_paged_attention_dyn", ATTENTION, dict(alpha=math.inf), -8),
    ("nimble_paged_attention_dyn", ATTENTION, dict(alpha=3e38), -8),
    ("nimble_paged_attention_dyn", ATTENTION, dict(window=-1), -8),
    ("nimble_paged_attention_dyn", ATTENTION, dict(**LONG, n=1000), -6),
    ("nimble_paged_attention_dyn", ATTENTION, dict(**LONG, ws=0), -6),
    ("nimble_paged_attention_dyn", ATTENTION, dict(**LONG, ws=P + 8), -5),
])
def test_refused_calls(name, good, wrong, code):
    assert getattr(nb.load(), name)(*{**good, **wrong}.values(), None) == code
    assert nb.last_error()


@pytest.mark.parametrize("name,good,nothing", [
    ("nimble_rotary_table_dyn", TABLE, dict(n=0, t=0)),
    ("nimble_rotary_dyn", ROTARY, dict(T=0, x=0, y=0)),
    ("nimble_rotary_dyn", ROTARY, dict(H=0, x=0, y=0)),
    ("nimble_cache_write_dyn", WRITE, dict(s=_seqs(rows=0, offsets=0), k=0)),
    ("nimble_cache_write_dyn", WRITE, dict(s=_seqs(count=0, offsets=0, lengths=0, pages=0))),
    ("nimble_cache_read_dyn", READ, dict(s=_seqs(rows=0), k=0)),
    ("nimble_paged_attention_dyn", ATTENTION, dict(s=_seqs(rows=0), q=0, o=0)),
    ("nimble_paged_attention_dyn", ATTENTION, dict(s=_seqs(count=0))),
])
def test_nothing_to_do(name, good, nothing):
    assert getattr(nb.load(), name)(*{**good, **nothing}.values(), None) == 0


def test_host_tensors_and_wrong_types_are_refused():
    from paper_2006_03031_amd import runtime as rt
    cache = rt.PagedCache.empty(3, 2, 16, 64, device="cpu")
    codes = rt.PagedCache.empty(3, 2, 16, 64, nb.I8, device="cpu")
    assert codes.k.dtype is torch.int8 and codes.v_scale.shape == (3, 2, 16)
    seqs = rt.Sequences(torch.tensor([0, 3]), torch.tensor([3]), torch.zeros(1, 1, dtype=torch.int32))
    x, table = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(9, 32, 2)
    for call in (lambda: rt.rotary(x, torch.arange(3), table), lambda: rt.cache_write(cache, x, x, seqs), lambda: rt.cache_read(codes, seqs, 3),
                 lambda: rt.paged_attention(x, cache, seqs)):
        with pytest.raises(nb.NimbleError) as e:
            call()
        assert e.value.code == -8
    for call, code in ((lambda: rt.cache_write(cache, x, x, seqs, table=table[..., 0]), -3), (lambda: rt.cache_write(cache, x, x, seqs, out=x), -8),
                       (lambda: rt.PagedCache.empty(3, 2, 16, 65), -8), (lambda: rt.PagedCache.empty(3, 2, 16, 64, nb.F32), -4)):
        with pytest.raises(nb.NimbleError) as e:
            call()
        assert e.value.code == code


def test_structs_match_the_header():
    assert ctypes.sizeof(binding._CSequences) == 48
    assert ctypes.sizeof(binding._CCache) == 72
    assert ctypes.sizeof(binding._CPagedPlan) == 48


def _f32(x):
    return ctypes.c_float(x).value


def _tiles(p, sizes, group, window, width_keys, block_keys):
    for old, n in sizes:
        tiles = -(-n * group // p.rows)
        keys = min(old + n, width_keys)
        if window and window + p.rows < keys:
            keys = window + p.rows
        yield tiles, -(-keys // block_keys) if tiles else 0


def _check_parts(p, sizes, group, kv_heads, window, width_keys, target):
    """The units that the chunks' kernel makes of a batch, as it works them out: totals in f32."""
    work = list(_tiles(p, sizes, group, window, width_keys, 64))
    total = 0.0
    for tiles, blocks in work:
        total = _f32(total + _f32(tiles * blocks))
    per = [_f32(_f32(total * kv_heads) / units) for units in (target, min(target, 512))] if p.parts else None
    most = min(max(4, math.ceil(per[per[0] < 16]) + 1), 1 << 30) if p.parts else 1 << 30
    units = slots = cut = 0
    for tiles, blocks in work:
        parts = max(1, (blocks + most // 2) // most)
        units += tiles * parts
        if parts > 1:
            slots, cut = slots + tiles * parts, cut + tiles
    assert units * kv_heads <= p.grid and slots * kv_heads <= p.slots and cut * kv_heads <= target
    return slots > 0


def _check_spans(p, sizes, group, kv_heads, window, width_keys, target):
    """The spans of the tokens' kernel: every step has a workgroup, every part a slot, and every cut tile is found by its first."""
    ends, at = [], 0
    for tiles, blocks in _tiles(p, sizes, group, window, width_keys, 32):
        steps = (max(1, -(-blocks // (p.step // 32))) if p.parts else 1) if tiles else 0
        for _ in range(tiles * kv_heads):
            ends.append((at, at + steps))
            at += steps
    assert at < 1 << 31
    per = max(1, -(-at // target)) if p.parts else 1
    assert -(-at // per) <= p.grid
    begun = set()
    for first, end in ends:
        a, b = first // per, (end - 1) // per
        if a != b:
            assert p.parts and a not in begun and 2 * b + 1 < p.slots
            begun.add(a)
    return bool(begun)


def test_grid_and_workspace_hold_every_batch():
    """Whatever the lengths, the device's units fit the grid, their parts the workspace, and the tiles that were cut the second launch."""
    rng = random.Random(7)
    seen = set()
    for _ in range(3000):
        S = rng.choice((1, 1, 2, 7, 64, 300))
        kv_heads = rng.choice((1, 2, 8, 12, 16))
        group = rng.choice((1, 2, 3, 4, 8, 16, 20))
        page = rng.choice((16, 32, 128, 1024))
        most_new, most_old = rng.choice((1, 1, 5, 300, 4000)), rng.choice((0, 100, 5000, 200000))
        sizes = [(rng.randint(0, most_old), rng.randint(0, most_new)) for _ in range(S)]
        rows = sum(n for _, n in sizes)
        width = -(-max(o + n for o, n in sizes) // page) + rng.randint(0, 3)
        window = rng.choice((0, 0, 1, 100, 5000))
        D = rng.choice((64, 128))
        if not 0 < rows * group * kv_heads < 1 << 20:
            continue
        p = nb.paged_attention_plan(rows, S, width, group * kv_heads, kv_heads, page, D, rng.choice((nb.BF16, nb.I8)), window)
        target = (p.slots - 8) // 2 if p.parts else 0
        cut = (_check_spans, _check_parts)[p.kernel](p, sizes, group, kv_heads, window, width * page, target)
        if p.parts:
            assert p.join_grid[0] and 1 <= p.join_grid[1] <= p.rows
            assert p.workspace_bytes >= p.slots * p.rows * (D * 4 + 8) + (1 + target) * 48
        else:
            assert not cut and p.workspace_bytes == 0
        seen.add((p.kernel, p.parts, cut))
    assert seen >= {(0, 1, True), (0, 1, False), (0, 0, False), (1, 1, True), (1, 1, False), (1, 0, False)}


def test_queries_without_elements_are_refused_by_their_shape():
    from paper_2006_03031_amd import runtime as rt
    k = torch.zeros(CACHE, dtype=torch.bfloat16)
    batch = rt.Sequences(torch.zeros(2, dtype=torch.int64), torch.zeros(1, dtype=torch.int64), torch.zeros((1, 3), dtype=torch.int32))
    for shape in ((7, 4, 0), (7, 4, 32), (7, 3, 64), (7, 256)):
        with pytest.raises(nb.NimbleError):
            rt.paged_attention(torch.zeros(shape, dtype=torch.bfloat16), rt.PagedCache(k, k), batch)


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")
def test_kernels_that_count_their_loads_have_no_others_under_way(tmp_path):
    """They wait for loads to LDS by how many there are behind: registers that spill to memory would be counted too."""
    from paper_2006_03031_amd import build
    out = tmp_path / "paged.s"
    subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "paged_attention.hip"), "-o", str(out)], check=True,
                   stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    kernels = re.findall(r"\.amdhsa_kernel (\S+).*?\.amdhsa_private_segment_fixed_size (\d+)", out.read_text(), re.S)
    counted = [(name, int(size)) for name, size in kernels if "paged_tokens_kernel" in name or "paged_chunks_kernel" in name]
    assert len(counted) == 15
    assert not [k for k in counted if k[1]]
