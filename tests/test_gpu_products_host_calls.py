"""The native calls of the 8-bit and the grouped products against the steps in Python: the same bits, and what they leave to the steps."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2006_03031_amd as nb  # noqa: E402


@pytest.fixture(scope="module")
def rt():
    nb.load()
    from paper_2006_03031_amd import runtime
    runtime.default_workspace(torch.device("cuda", 0))   # from here on the native calls serve the device
    return runtime


class Steps:
    """In place of the native calls: every call goes through the steps."""
    quantize_rows = product = staticmethod(lambda *a: None)


def _operands(R=40, E=3, N=72, K=128):
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w = torch.randn((R, K), device="cuda", generator=g).bfloat16(), torch.randn((E, N, K), device="cuda", generator=g).bfloat16()
    bias = torch.randn((E, N), device="cuda", generator=g).bfloat16()
    return x, w, bias, torch.tensor([0, R // 3, R // 3, R], device="cuda")


@pytest.mark.parametrize("R,N,K", [(40, 72, 128), (0, 72, 128), (1, 7, 33), (700, 512, 512)])
@pytest.mark.parametrize("out", [nb.BF16, nb.F32])
def test_the_bits_of_the_steps(rt, monkeypatch, R, N, K, out):
    x, w, bias, off = _operands(R, 3, N, K)
    def calls(native):
        q, s = rt.quantize_rows(x)
        wq, ws = rt.quantize_rows(w.view(3 * N, K))
        wq, ws = wq.view(3, N, -1), ws.view(3, N)
        f = rt.quantize_rows(x.float(), K + 3)
        if native:
            assert rt._host_calls.quantize_rows(x, 0) is not None
            assert rt._host_calls.product(x, None, w, None, bias, off, nb.EPI_BIAS, out, None) is not None
        return [q, s, *f, rt.dense_i8(q, s, wq[0], ws[0], bias[0], nb.EPI_BIAS_GELU_ERF, out),
                rt.dense_i8(q, s, wq[0], ws[0], None, nb.EPI_NONE, out), rt.grouped_dense(x, w, bias, off, nb.EPI_BIAS, out),
                rt.grouped_dense_i8(q, s, wq, ws, bias, off, nb.EPI_BIAS, out)]
    got = calls(True)
    monkeypatch.setattr(rt, "_host_calls", Steps)
    want = calls(False)
    for a, b in zip(got, want):
        assert a.dtype == b.dtype and a.shape == b.shape and a.device == b.device and torch.equal(a, b)


def test_an_output_of_the_callers(rt):
    x, w, bias, off = _operands()
    y = torch.full((40, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    assert rt.grouped_dense(x, w, bias, off, out=y) is y
    assert torch.equal(y, rt.grouped_dense(x, w, bias, off))


def test_what_is_left_to_the_steps(rt):
    x, w, bias, off = _operands()
    q, s = rt.quantize_rows(x)
    wq, ws = rt.quantize_rows(w[0].contiguous())
    B, F = nb.EPI_BIAS, nb.BF16
    native = rt._host_calls.product
    wide = torch.cat((q, q), 1)
    for args in ((q, s, wq, None, bias[0], None, B, F, None), (q.cpu(), s, wq, ws, bias[0], None, B, F, None), (q, s[:3], wq, ws, bias[0], None, B, F, None),
                 (wide[:, :128], s, wq, ws, bias[0], None, B, F, None), (q, s, wq, ws, None, None, B, F, None), (q, s, wq, ws, bias, None, B, F, None),
                 (q, s, wq, ws, bias[0], None, 5, F, None), (q, s, wq, ws, bias[0], None, B, nb.I8, None), (x, None, w, None, bias, off.int(), B, F, None),
                 (x, None, w, None, bias, off[:3], B, F, None), (x, None, w, None, bias, None, B, F, None), (x, None, w[:, :, :64], None, bias, off, B, F, None),
                 (x, None, w, None, bias, off, B, F, torch.empty((40, 72), device="cuda")), (x, None, w, None, bias, off, B, nb.F32, torch.empty((41, 72), device="cuda"))):
        assert native(*args) is None
    for args in ((x.half(), 0), (x, 127), (x, -1), (x, 1 << 31), (x.t(), 0), (x[0], 0), (x.cpu(), 0), (x, True), (x, None)):
        assert rt._host_calls.quantize_rows(*args) is None
    # a mode sees the steps
    from torch.overrides import TorchFunctionMode
    seen = []

    class Mode(TorchFunctionMode):
        def __torch_function__(self, func, types, args=(), kwargs=None):
            seen.append(func)
            return func(*args, **(kwargs or {}))
    with Mode():
        y = rt.grouped_dense(x, w, bias, off)
    assert torch.empty in seen and torch.equal(y, rt.grouped_dense(x, w, bias, off))
