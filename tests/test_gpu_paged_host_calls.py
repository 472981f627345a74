"""The native calls of the paged cache's operators against the steps in Python: the same bits, and what they leave to the steps."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paged_util as pu  # noqa: E402
import paper_2006_03031_amd as nb  # noqa: E402
from paged_util import BF, Batch  # noqa: E402


@pytest.fixture(scope="module")
def rt():
    nb.load()
    from paper_2006_03031_amd import runtime
    runtime.default_workspace(torch.device("cuda", 0))   # from here on the native calls serve the device
    return runtime


class Steps:
    """In place of the native calls: every call goes through the steps."""
    rotary = cache_write = cache_read = paged_attention = staticmethod(lambda *a: None)


def _operands(int8=False, H=6, G=2, D=64):
    batch = Batch([(40, 3), (0, 9), (700, 1)], 16)
    rows = torch.randn(batch.rows, H + 2 * G, D, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    return batch, pu.random_cache(batch, G, D, int8), rows[:, :H], rows[:, H:H + G], rows[:, H + G:], pu.angles(800, D).float().cuda()


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_the_bits_of_the_steps(rt, monkeypatch, interleaved, D, int8):
    batch, cpu, q, k, v, table = _operands(int8, D=D)
    seqs = batch.on_gpu()
    positions = torch.arange(batch.rows, device="cuda") * 7

    def calls(native):
        cache = pu.to_gpu(cpu)
        if native:
            assert rt._host_calls.rotary(q, positions, table, interleaved, None) is not None
            assert rt._host_calls.cache_write(cache, k, v, seqs, None, None, interleaved, None) is True
            assert rt._host_calls.cache_read(cache, seqs, batch.rows, nb.F32) is not None
            assert rt._host_calls.paged_attention(q, cache, seqs, 0.125, 0, None) is not None
        out = [rt.rotary(q, positions, table, interleaved), rt.cache_write(cache, k, v, seqs, q=q, table=table, interleaved=interleaved)]
        assert rt.cache_write(cache, k, v, seqs, table=table, interleaved=interleaved) is None
        out += [t for t in cache if t is not None]
        out += rt.cache_read(cache, seqs, batch.rows) + rt.cache_read(cache, seqs, batch.rows, nb.F32)
        return out + [rt.paged_attention(q, cache, seqs), rt.paged_attention(q, cache, seqs, alpha=0.3, window=20)]
    got = calls(True)
    monkeypatch.setattr(rt, "_host_calls", Steps)
    want = calls(False)
    assert len(got) == len(want)
    for a, b in zip(got, want):
        assert a.dtype == b.dtype and a.shape == b.shape and a.device == b.device and torch.equal(a, b)


def test_outputs_of_the_callers(rt):
    batch, cpu, q, k, v, table = _operands()
    cache, seqs = pu.to_gpu(cpu), batch.on_gpu()
    y = torch.zeros(batch.rows, 6, 64, dtype=BF, device="cuda")
    positions = torch.arange(batch.rows, device="cuda")
    assert rt.rotary(q, positions, table, out=y) is y and torch.equal(y, rt.rotary(q, positions, table))
    assert rt.cache_write(cache, k, v, seqs, q=q, table=table, out=y) is y and torch.equal(y, rt.cache_write(cache, k, v, seqs, q=q, table=table))
    assert rt.paged_attention(q, cache, seqs, out=y) is y and torch.equal(y, rt.paged_attention(q, cache, seqs))
    seqs = seqs._replace(pages=torch.nn.functional.pad(seqs.pages, (0, 60)))
    need = nb.paged_attention_plan(batch.rows, 3, seqs.pages.shape[1], 6, 2, 16, 64).workspace_bytes
    assert need > 0
    ws = torch.empty(need + 64, dtype=torch.uint8, device="cuda")
    assert torch.equal(rt.paged_attention(q, cache, seqs), rt.paged_attention(q, cache, seqs, workspace=ws))


def test_what_is_left_to_the_steps(rt):
    batch, cpu, q, k, v, table = _operands()
    cache, seqs = pu.to_gpu(cpu), batch.on_gpu()
    T = batch.rows
    positions = torch.arange(T, device="cuda")
    native = rt._host_calls
    for args in ((q.float(), positions, table, False, None), (q, positions.int(), table, False, None), (q, positions[:3], table, False, None),
                 (q, positions, table[..., :1], False, None), (q[..., ::2], positions, table, False, None), (q, positions, table, 0, None),
                 (q, positions, table, False, q[:2]), (q.cpu(), positions, table, False, None), (q[0], positions, table, False, None)):
        assert native.rotary(*args) is None
    for args in ((cache[:3], k, v, seqs, None, None, False, None), (cache, k[:5], v, seqs, None, None, False, None), (cache, k, v, seqs, q[:4], None, False, None),
                 (cache, k, v, seqs, None, table[0], False, None), (cache, k, v, seqs, None, None, False, q), (cache, k, v, seqs, q, table, None, None),
                 (cache, k.float(), v, seqs, None, None, False, None), (cache, k, v, seqs[:2], None, None, False, None),
                 (cache._replace(v=cache.v[:-1]), k, v, seqs, None, None, False, None), (cache, k, v, seqs._replace(pages=seqs.pages.long()), None, None, False, None)):
        assert native.cache_write(*args) is None
    for args in ((cache, seqs, -1, nb.BF16), (cache, seqs, T, nb.I8), (cache, seqs, 1 << 25, nb.BF16), (cache, seqs, True, nb.BF16),
                 (cache._replace(k=cache.k.char()), seqs, T, nb.BF16)):
        assert native.cache_read(*args) is None
    for args in ((q, cache, seqs, 1, 0, None), (q, cache, seqs, 0.0, 0, None), (q, cache, seqs, 0.125, -1, None), (q[:, :5], cache, seqs, 0.125, 0, None),
                 (q, cache, seqs, 0.125, 0, q.float()), (q, cache, seqs._replace(lengths=seqs.lengths[:2]), 0.125, 0, None), (q[..., :32], cache, seqs, 0.125, 0, None)):
        assert native.paged_attention(*args) is None
    # a mode sees the steps
    from torch.overrides import TorchFunctionMode
    seen = []

    class Mode(TorchFunctionMode):
        def __torch_function__(self, func, types, args=(), kwargs=None):
            seen.append(func)
            return func(*args, **(kwargs or {}))
    with Mode():
        y = rt.paged_attention(q, cache, seqs)
    assert torch.empty in seen and torch.equal(y, rt.paged_attention(q, cache, seqs))


@pytest.mark.parametrize("call,code", [
    (lambda rt, c, s, q, k, v: rt.paged_attention(q, c, s, alpha=-1.0), -8),
    (lambda rt, c, s, q, k, v: rt.paged_attention(q, c, s, window=-2), -8),
    (lambda rt, c, s, q, k, v: rt.paged_attention(q[:, :5], c, s), -3),
    (lambda rt, c, s, q, k, v: rt.paged_attention(q.float(), c, s), -4),
    # (a table for more than 1024 keys: up to that no workspace is needed)
    (lambda rt, c, s, q, k, v: rt.paged_attention(q, c, s._replace(pages=s.pages.repeat(1, 3)), workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), -6),
    (lambda rt, c, s, q, k, v: rt.paged_attention(q, c, s._replace(lengths=s.lengths.cpu())), -8),
    (lambda rt, c, s, q, k, v: rt.paged_attention(q, c._replace(k=c.k.transpose(1, 2).contiguous().transpose(1, 2)), s), -8),
    (lambda rt, c, s, q, k, v: rt.cache_write(c, k[..., ::2], v[..., ::2], s), -3),
    (lambda rt, c, s, q, k, v: rt.cache_write(c, k.transpose(0, 1), v.transpose(0, 1), s), -3),
    (lambda rt, c, s, q, k, v: rt.cache_write(c, k, v, s, table=torch.zeros(9, 33, 2, device="cuda")), -3),
    (lambda rt, c, s, q, k, v: rt.cache_write(c, k, v, s, table=torch.zeros(9, 20, 2, device="cuda")), -8),
    (lambda rt, c, s, q, k, v: rt.cache_read(c, s, 13, nb.I8), -4),
    (lambda rt, c, s, q, k, v: rt.cache_read(c, s, 13, out=(q, q)), -3),
    (lambda rt, c, s, q, k, v: rt.rotary(q[..., ::2], torch.arange(13, device="cuda"), torch.zeros(9, 8, 2, device="cuda")), -8),
    (lambda rt, c, s, q, k, v: rt.rotary(q, torch.arange(13, device="cuda"), torch.zeros(9, 33, 2, device="cuda")), -3),
])
def test_errors_are_raised(rt, call, code):
    batch, cpu, q, k, v, _ = _operands()
    assert batch.rows == 13
    with pytest.raises(nb.NimbleError) as e:
        call(rt, pu.to_gpu(cpu), batch.on_gpu(), q, k, v)
    assert e.value.code == code
