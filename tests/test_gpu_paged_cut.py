"""paged_attention over sequences that are cut into parts: few rows under a window, what they do not see, and single tokens beside long prompts."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paged_util as pu
from paged_util import BF, Batch
from test_gpu_paged_attention import _check, _plan, _q, _run

TOKENS = [(8999, 1), (5000, 1), (30, 1), (9100, 1)]
ROWS = [(8000, 3), (20, 1), (5001, 2), (1400, 3)]


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("window", [1500, 4000])
@pytest.mark.parametrize("H,G,D", [(4, 2, 64), (5, 1, 128), (4, 4, 128)])
@pytest.mark.parametrize("sizes", [TOKENS, ROWS])
def test_few_rows_under_a_window(sizes, H, G, D, window, int8):
    batch = Batch(sizes, 32, ahead=1, behind=1)
    p = _plan(batch, H, G, D, int8, window)
    assert (p.kernel, p.parts) == (0, 1)
    cache, q = pu.random_cache(batch, G, D, int8), _q(batch, H, D)
    _check(_run(q, cache, batch, window=window), q, cache, batch, window, weight_step=pu.half_step(BF) ** 2)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [0, 1500])
def test_few_rows_and_what_they_do_not_see(window, D, bad):
    """The first key of the first row's window, which the next do not see, and the last row's own, which the ones before do not see."""
    old, n = 8000, 3
    batch = Batch([(old, n), (3000, 2)], 32)
    p = _plan(batch, 4, 2, D, False, window)
    assert (p.kernel, p.parts) == (0, 1)
    cache, q = pu.random_cache(batch, 2, D, False), _q(batch, 4, D)
    want, bound = pu.attention(q, cache, batch, window)
    k, v = cache[0].clone(), cache[1].clone()
    positions = [old + n - 1] + ([old - window + 1, old - window] if window else [])
    page, slot = batch.slots(0, torch.tensor(positions))
    v[page, 0, slot, 3] = bad
    k[page, 1, slot, 5] = bad
    got = _run(q, (k, v, None, None), batch, window=window).double().cpu()
    clean = [1, 3, 4] if window else [0, 1, 3, 4]
    assert bool((got[clean] - want[clean]).abs().le(bound[clean]).all())
    keep = [d for d in range(D) if d != 3]
    for row in {0, 1, 2} - set(clean):
        assert not bool(got[row, :2, 3].isfinite().any())      # a value that the row sees, in the heads that share it
        assert bool((got[row, :2][:, keep] - want[row, :2][:, keep]).abs().le(bound[row, :2][:, keep]).all())
        if math.isnan(bad):
            assert bool(got[row, 2:].isnan().all())            # a key
    assert bool((got[[1], :2, 3] - want[[1], :2, 3]).abs().le(bound[[1], :2, 3]).all())


@pytest.mark.parametrize("D", [64, 128])
def test_few_rows_and_nan_scales_that_they_do_not_see(D):
    window, old, n = 1500, 8000, 3
    batch = Batch([(old, n), (3000, 2)], 32)
    assert _plan(batch, 4, 2, D, True, window).parts
    cache, q = pu.random_cache(batch, 2, D, True), _q(batch, 4, D)
    want, bound = pu.attention(q, cache, batch, window)
    page, slot = batch.slots(0, torch.tensor([old + n - 1, old - window + 1, old - window]))
    cache[2][page, 0, slot] = math.nan
    cache[3][page, 1, slot] = math.nan
    got = _run(q, cache, batch, window=window).double().cpu()
    clean = [1, 3, 4]
    assert bool((got[clean] - want[clean]).abs().le(bound[clean]).all())
    assert bool(got[[0, 2]].isnan().all())


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("H,G,D", [(2, 1, 64), (1, 1, 128), (2, 2, 128)])
@pytest.mark.parametrize("window", [0, 3000])
def test_a_long_token_beside_a_prompt_without_cached_keys(window, H, G, D, int8):
    """The kernel of many rows cuts the one row's keys and leaves the prompt's early tiles few blocks."""
    batch = Batch([(9000, 1), (0, 2100), (40, 1)], 64)
    p = _plan(batch, H, G, D, int8, window)
    assert (p.kernel, p.parts) == (1, 1)
    cache, q = pu.random_cache(batch, G, D, int8), _q(batch, H, D)
    _check(_run(q, cache, batch, window=window), q, cache, batch, window)
