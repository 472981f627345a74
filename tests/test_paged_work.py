"""How paged_attention divides its work: the device's own code (csrc/paged_work.h), built for the CPU (no GPU needed)."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

import paper_2006_03031_amd as nb
from paper_2006_03031_amd import build

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not on PATH")

UNWRITTEN = 0x7b7b7b7b
FIELDS = "workgroup s first n length tile head slot parts part low high block0 block1".split()


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("work") / "paged_work.so")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run(["g++", "-O1", "-U_FORTIFY_SOURCE", "-std=c++17", "-fPIC", "-shared", "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC,
                    os.path.join(here, "paged_work_cpu.cpp"), os.path.join(build.CSRC, "cache_host.cpp"), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.apart.argtypes = [ctypes.c_int64] * 8
    i64, p = ctypes.c_int64, ctypes.c_void_p
    lib.paged_work.argtypes = [i64] * 7 + [ctypes.c_int, i64, p, p, i64, p, i64, p]
    lib.paged_work.restype = i64
    return lib


@pytest.fixture(scope="module")
def work(lib):
    def run(offsets, lengths, rows, width, heads, kv_heads, page, D, dtype, window=0, stride=1):
        """(plan, records of all workgroups, table of the second launch)"""
        S = len(lengths)
        plan = nb.paged_attention_plan(rows, S, width, heads, kv_heads, page, D, dtype, window)
        off, lens = (ctypes.c_int64 * len(offsets))(*offsets), (ctypes.c_int64 * max(S, 1))(*lengths)
        room = 4 * plan.grid + 400000
        out = (ctypes.c_int64 * (len(FIELDS) * room))()
        items = (ctypes.c_int * (12 * (2 + plan.join_grid[0] + plan.grid)))(*[UNWRITTEN] * (12 * (2 + plan.join_grid[0] + plan.grid)))
        n = lib.paged_work(rows, S, width, heads, kv_heads, page, D, dtype, window, off, lens, stride, out, room, items)
        assert 0 <= n <= room
        flat = out[:n * len(FIELDS)]
        records = [dict(zip(FIELDS, flat[i * len(FIELDS):(i + 1) * len(FIELDS)])) for i in range(n)]
        return plan, records, [items[i * 12:(i + 1) * 12] for i in range(len(items) // 12)]
    return run


def check_bounds(plan, records, items, rows, group, kv_heads):
    """Whatever the offsets: nothing outside of the tensors and the workspace, by either launch."""
    for r in records:
        assert 0 <= r["first"] <= r["first"] + r["n"] <= rows
        assert 0 <= r["tile"] * plan.rows < r["n"] * group and 0 <= r["head"] < kv_heads
        assert -1 <= r["slot"] < plan.slots or (r["slot"] == -1 and not plan.parts)
        assert r["block0"] >= 0 and r["block1"] * (32, 64)[plan.kernel] <= max(r["length"], 0) + (32, 64)[plan.kernel]
    if not plan.parts:
        return 0
    joined = 0
    for i in range(min(items[0][0], plan.join_grid[0])):   # what a workgroup of the second launch goes by
        parts, slot, second, apart, tile, head, first, n, length = items[1 + i][:9]
        assert parts != UNWRITTEN, "an entry that nobody has written"
        if parts < 2:
            continue
        joined += 1
        assert 0 <= slot < plan.slots and 0 <= second and second + (parts - 2) * apart < plan.slots
        assert 0 <= tile * plan.rows < n * group and 0 <= head < kv_heads and 0 <= first <= first + n <= rows
    return joined


def check_whole(plan, records, items, offsets, lengths, group, kv_heads, window):
    """Offsets that keep to their description: every tile's blocks once, its parts where the second launch looks for them."""
    keys = (32, 64)[plan.kernel]
    seen = {}
    for r in records:
        seen.setdefault((r["s"], r["tile"], r["head"]), []).append(r)
    expect = {(s, t, h) for s in range(len(lengths)) for t in range(-(-(offsets[s + 1] - offsets[s]) * group // plan.rows)) for h in range(kv_heads)}
    assert set(seen) == expect
    entries = {}
    if plan.parts:
        for e in items[1:1 + min(items[0][0], plan.join_grid[0])]:
            if e[0] >= 2:
                entries[(e[6], e[7], e[4], e[5])] = e
    cut = 0
    for (s, t, h), shares in seen.items():
        n, length = offsets[s + 1] - offsets[s], lengths[s]
        before = length - n
        last = before + (min((t + 1) * plan.rows, n * group) - 1) // group
        low = max(0, before + t * plan.rows // group - window + 1) if window else 0
        blocks = [b for r in sorted(shares, key=lambda r: r["block0"]) for b in range(r["block0"], r["block1"])]
        assert blocks == (list(range(low // keys, last // keys + 1)) if last >= 0 else [])
        slots = sorted(r["slot"] for r in shares)
        if slots == [-1]:
            continue
        cut += 1
        e = entries[(offsets[s], n, t, h)]
        assert e[0] == len(slots) and e[8] == length
        assert slots == sorted([e[1]] + [e[2] + x * e[3] for x in range(e[0] - 1)])
    assert cut == len(entries)
    slots = [r["slot"] for r in records if r["slot"] >= 0]
    assert len(slots) == len(set(slots))
    return cut


def test_every_block_of_every_tile_has_one_workgroup(work):
    rng = random.Random(11)
    seen = set()
    for _ in range(150):
        S = rng.choice((1, 1, 2, 7, 64, 65, 200))
        kv_heads, group, page = rng.choice((1, 2, 3, 8)), rng.choice((1, 2, 4, 5)), rng.choice((16, 64, 256))
        most_new, most_old = rng.choice((1, 1, 5, 300, 3000)), rng.choice((0, 100, 3000, 60000))
        sizes = [(rng.randint(0, most_old), rng.randint(0, most_new)) for _ in range(S)]
        offsets, lengths = [0], []
        for old, n in sizes:
            offsets.append(offsets[-1] + n)
            lengths.append(old + n)
        if not 0 < offsets[-1] * group * kv_heads < 60000:
            continue
        width = -(-max(lengths) // page) + rng.choice((0, 1, 3, 500))
        window = rng.choice((0, 0, 1, 100, 1500, 5000))
        dtype, D = rng.choice((nb.BF16, nb.I8)), rng.choice((64, 128))
        got = work(offsets, lengths, offsets[-1], width, group * kv_heads, kv_heads, page, D, dtype, window)
        check_bounds(*got, offsets[-1], group, kv_heads)
        cut = check_whole(*got, offsets, lengths, group, kv_heads, window)
        seen.add((got[0].kernel, got[0].parts, cut > 0, window > 0))
    assert {s[:3] for s in seen} >= {(0, 1, True), (0, 1, False), (0, 0, False), (1, 1, True), (1, 1, False), (1, 0, False)}
    assert (0, 1, True, True) in seen and (1, 1, True, True) in seen


def falling(rng, rows, S):
    """Offsets that do not keep to their description."""
    kind = rng.randrange(4)
    if kind == 0:
        return [(s & 1) * rows for s in range(S + 1)]
    if kind == 1:
        return [rng.randint(0, rows) for _ in range(S + 1)]
    if kind == 2:
        return [rng.choice((0, rows, -5, rows + 7, -2 ** 63, 2 ** 63 - 1, rng.randint(0, rows))) for _ in range(S + 1)]
    return sorted((rng.randint(0, rows) for _ in range(S + 1)), reverse=True)


def test_cut_tiles_beyond_the_grid_are_not_joined(work):
    """Sequences that share rows: more tiles than the grid was made for, so that parts of some are computed by nobody."""
    rows, S = 2048, 129
    offsets = [(s & 1) * rows for s in range(S)] + [16]
    plan, records, items = work(offsets, [1] * (S - 1) + [16384], rows, 1024, 32, 8, 16, 64, nb.BF16)
    assert plan.kernel == 1 and plan.parts
    check_bounds(plan, records, items, rows, 4, 8)


def test_falling_offsets_stay_inside(work):
    rng = random.Random(5)
    seen = set()
    for _ in range(60):
        S, rows = rng.choice((1, 2, 7, 64, 65, 300)), rng.choice((1, 16, 70, 500, 2048))
        kv_heads, group, page = rng.choice((1, 2, 8)), rng.choice((1, 4, 7)), rng.choice((16, 256))
        width = rng.choice((1, 100, 1000))
        offsets = falling(rng, rows, S)
        few = rng.random() < 0.5  # (a long sequence behind many short ones)
        lengths = [1 if few and s < S - 2 else rng.choice((0, 1, width * page, rng.randint(0, width * page), -3, 2 ** 62)) for s in range(S)]
        window = rng.choice((0, 0, 100, 3000))
        got = work(offsets, lengths, rows, width, group * kv_heads, kv_heads, page, rng.choice((64, 128)), rng.choice((nb.BF16, nb.I8)), window)
        seen.add((got[0].kernel, got[0].parts, check_bounds(*got, rows, group, kv_heads) > 0))
    assert seen >= {(0, 1, True), (1, 1, True), (0, 0, False), (1, 0, False)}


@pytest.mark.parametrize("window", [0, 3000])
@pytest.mark.parametrize("S,rows,keys", [(17, 256, 1 << 30), (65, 1024, 1 << 28), (129, 2048, 1 << 26)])
def test_steps_past_32_bits_are_not_joined(work, S, rows, keys, window):
    """Sequences that share rows, each over so many keys that the steps of all together pass 32 bits, by so little or so much."""
    for last in (51200, 256, keys):
        lengths = [keys] * (S - 1) + [last]
        got = work([(s & 1) * rows for s in range(S + 1)], lengths, rows, keys // 1024, 8, 8, 1024, 128, nb.BF16, window)
        assert got[0].kernel == 0 and got[0].parts
        check_bounds(*got, rows, 1, 8)


def test_tensors_that_share_memory(lib):
    """Whether rows of bytes share one, against the sets of their addresses."""
    rng = random.Random(3)
    seen = set()
    for _ in range(20000):
        a_rows, b_rows = rng.choice((1, 1, 2, 3, 7)), rng.choice((1, 2, 5))
        a_bytes, b_bytes = rng.randint(1, 9), rng.randint(1, 9)
        stride = rng.randint(max(a_bytes, b_bytes), 40)
        a, b = 1000, 1000 + rng.randint(-150, 150)
        sets = [{at + i * stride + x for i in range(rows) for x in range(n)} for at, rows, n in ((a, a_rows, a_bytes), (b, b_rows, b_bytes))]
        refused = lib.apart(a, a_rows, a_bytes, stride, b, b_rows, b_bytes, stride) != 0
        assert refused == bool(sets[0] & sets[1])
        inside = max(sets[0]) >= min(sets[1]) and max(sets[1]) >= min(sets[0])
        seen.add((refused, inside))
        # of two strides: refused where one does not lie behind the other
        other = stride + rng.randint(1, 5)
        sets[1] = {b + j * other + x for j in range(b_rows) for x in range(b_bytes)}
        inside = max(sets[0]) >= min(sets[1]) and max(sets[1]) >= min(sets[0])
        refused = lib.apart(a, a_rows, a_bytes, stride, b, b_rows, b_bytes, other) != 0
        assert refused == (inside if a_rows > 1 and b_rows > 1 else bool(sets[0] & sets[1]))
    assert seen == {(True, True), (False, True), (False, False)}
    assert lib.apart(0, 1, 10, 10, 0, 1, 10, 10) == 0 and lib.apart(4096, 0, 10, 10, 4096, 1, 10, 10) == 0
    far = 2 ** 62
    assert lib.apart(4096, 2 ** 31, 2, 2 ** 41, 8192, 2 ** 31, 2, 2 ** 41) == 0 and lib.apart(far, 2 ** 31, 2 ** 40, 2 ** 41, 4096, 2 ** 31, 2 ** 40, 2 ** 41) != 0
