"""Caller-side sequence for one dynamic operator, on torch tensors.

For every operator this is the order the paper gives for a tensor whose
leading dimension is unknown until run time (Section 3.2, Section 3.3,
Appendix A): read the run-time shapes (host metadata, no device sync), run the
shape function, allocate the output from the shape it returns, then invoke the
kernel with inputs and outputs passed explicitly.  torch supplies device memory
and the stream; all arithmetic runs in the HIP library.
"""
from __future__ import annotations

import ctypes
import warnings
from typing import NamedTuple, Optional, Tuple

import torch

from . import binding as nb


class _StepsOnly:
    """In place of the native one-call sequences where they cannot be loaded (not built, or built for another torch):
    leaves every call to the steps, which give the same results, and says so on the first call on a GPU."""
    dense = attention = fused_attention = lstm_sequence = vm_run = set_workspace = staticmethod(lambda *a: None)
    quantize_rows = product = bind_products = staticmethod(lambda *a: None)
    rotary = cache_write = cache_read = paged_attention = bind_paged = staticmethod(lambda *a: None)

    def __init__(self, why: ImportError):
        self.why = why

    def bind(self, *a) -> None:
        warnings.warn(f"the native host calls do not load ({self.why}): calls go through Python step by step, which takes "
                      "some microseconds more each; to build them run "
                      "`python -c 'import __graft_entry__ as g; g.build()'`", RuntimeWarning, stacklevel=2)


try:
    from . import _host_calls
except ImportError as e:
    _host_calls = _StepsOnly(e)

_TORCH_DTYPE = {nb.BF16: torch.bfloat16, nb.F32: torch.float32, nb.I8: torch.int8}


try:  # raw handle of torch's current stream without building a Stream object (several us cheaper)
    _raw_stream = torch._C._cuda_getCurrentRawStream
except AttributeError:  # pragma: no cover - older torch
    _raw_stream = None


_bound = False


def _bind_host_calls(device) -> None:
    """Gives the native calls the entry points of the library that binding.py loads, on the first call that went
    through on a GPU; until then they leave every call to the steps below."""
    global _bound
    if _bound or _raw_stream is None or device.type != "cuda" or torch.overrides._get_current_function_mode() is not None:
        return
    lib = nb.load()
    addresses = [ctypes.cast(getattr(lib, f), ctypes.c_void_p).value
                 for f in ("nimble_dense_dyn", "nimble_attention_dyn", "nimble_attention_chain_dyn", "nimble_vm_run",
                           "nimble_lstm_seq_preferred", "nimble_lstm_seq_workspace_bytes", "nimble_lstm_seq_pre_dyn",
                           "nimble_lstm_seq_status")]
    _host_calls.bind(*addresses, torch._C._cuda_getDevice, _raw_stream, device.index or 0)
    _host_calls.bind_products(*[ctypes.cast(getattr(lib, f), ctypes.c_void_p).value
                                for f in ("nimble_quantize_rows_dyn", "nimble_dense_i8_dyn", "nimble_grouped_dense_dyn",
                                          "nimble_grouped_dense_i8_dyn")])
    _host_calls.bind_paged(*[ctypes.cast(getattr(lib, f), ctypes.c_void_p).value
                             for f in ("nimble_rotary_dyn", "nimble_cache_write_dyn", "nimble_cache_read_dyn", "nimble_paged_attention_plan_of",
                                       "nimble_paged_attention_dyn")])
    _bound = True


def _stream() -> int:
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


class StorageArena:
    """One backing storage allocated up front, tensors carved out of it at offsets computed
    from the shape function's result: alloc_storage once, then alloc_tensor(storage, offset,
    shape, dtype) per operator (Section 3.3, storage coalescing).  `reset()` rewinds the
    offset; the caller does that once per inference when the previous outputs are dead."""

    def __init__(self, capacity_bytes: int, device="cuda"):
        self.alignment = max(256, nb.storage_alignment())
        self.storage = torch.empty(int(capacity_bytes) + self.alignment, dtype=torch.uint8, device=device)
        base = self.storage.data_ptr()
        self._base_off = (-base) % self.alignment
        self.capacity = int(capacity_bytes)
        self.offset = 0
        # tensors already carved at (offset, shape, dtype): a request that repeats (the same run-time
        # shape at the same place of the same request sequence) gets the same view back instead of
        # three new Python tensor objects, which is what an allocation from the arena would otherwise cost
        self._views = {}

    def reset(self) -> None:
        self.offset = 0

    def alloc(self, shape, dtype: int) -> torch.Tensor:
        key = (self.offset, tuple(shape), dtype)
        hit = self._views.get(key)
        if hit is not None:
            self.offset = hit[1]
            return hit[0]
        nbytes = nb.storage_bytes(shape, dtype)
        start = (self.offset + self.alignment - 1) // self.alignment * self.alignment
        if start + nbytes > self.capacity:
            raise MemoryError(f"arena of {self.capacity} bytes cannot hold {nbytes} more at offset {start}")
        flat = self.storage[self._base_off + start:self._base_off + start + nbytes]
        t = flat.view(_TORCH_DTYPE[dtype]).view(tuple(shape))
        if len(self._views) >= 4096:
            self._views.clear()
        self._views[key] = (t, start + nbytes)
        self.offset = start + nbytes
        return t


_WORKSPACE = {}
WORKSPACE_BYTES = 64 << 20


def default_workspace(device) -> torch.Tensor:
    """Caller-owned scratch handed to every dense call (the library never allocates): holds the
    f32 partial sums when the dispatch function cuts K.  One per device, shared by the calls on
    one stream; calls that overlap on different streams must bring their own."""
    key = str(device)
    ws = _WORKSPACE.get(key)
    if ws is None:
        ws = torch.empty(WORKSPACE_BYTES, dtype=torch.uint8, device=device)
        _WORKSPACE[key] = ws
        if type(ws) is torch.Tensor and ws.is_cuda:  # from here on the native calls serve this device
            _bind_host_calls(ws.device)
            _host_calls.set_workspace(ws.device.index, ws)
    return ws


def _ptr(t: torch.Tensor, dtype, what: str) -> int:
    """Device address of a tensor the C ABI can take as a plain pointer: contiguous, on the GPU and
    of the element type the entry point reads; anything else is refused here (the library sees only
    an address and would read a strided view or another dtype as packed data)."""
    if t.dtype is not dtype or not t.is_cuda or not t.is_contiguous():
        raise nb.NimbleError(-4 if t.dtype is not dtype else -8,
                             f"{what}: need a contiguous {dtype} tensor on the GPU, got {t.dtype}, "
                             f"device {t.device}, strides {tuple(t.stride())}")
    return t.data_ptr()


_BF, _F32 = torch.bfloat16, torch.float32


def _alloc(shape, dtype: int, device) -> torch.Tensor:
    # alloc_storage(size, alignment, device) + alloc_tensor(storage, 0, shape, dtype):
    # torch's caching allocator returns storage aligned to at least 512 bytes.
    nb.storage_bytes(shape, dtype)  # validates the size computation
    return torch.empty(tuple(shape), dtype=_TORCH_DTYPE[dtype], device=device)


def dense(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor], epilogue: int = nb.EPI_BIAS,
          out_dtype: int = nb.BF16, force_variant: int = nb.VAR_AUTO,
          out: Optional[torch.Tensor] = None, arena: Optional[StorageArena] = None,
          workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    if out is None and arena is None and workspace is None and force_variant == nb.VAR_AUTO:
        y = _host_calls.dense(x, w, bias, epilogue, out_dtype)
        if y is not None:
            return y
    M, N = nb.nimble_dense_shape(tuple(x.shape), tuple(w.shape))
    K = x.shape[1]
    if out is not None:
        y = out
        if tuple(y.shape) != (M, N):
            raise nb.NimbleError(-3, f"dense: out is {tuple(y.shape)}, the shape function gives {(M, N)}")
    elif arena is not None:
        y = arena.alloc((M, N), out_dtype)
    else:
        y = _alloc((M, N), out_dtype, x.device)
    ws = workspace if workspace is not None else default_workspace(x.device)
    px, pw = _ptr(x, _BF, "x"), _ptr(w, _BF, "w")
    pb = _ptr(bias, _BF, "bias") if bias is not None else 0
    if bias is not None and bias.numel() != N:
        raise nb.NimbleError(-3, f"dense: bias has {bias.numel()} elements, N is {N}")
    py = _ptr(y, _TORCH_DTYPE[out_dtype], "y")
    if force_variant == nb.VAR_AUTO:
        nb.nimble_dense_dyn(px, pw, pb, py, M, N, K, epilogue, out_dtype, ws.data_ptr(),
                            ws.numel() * ws.element_size(), _stream())
    else:   # ablation, tuning and the per-variant tests pin one member of the kernel family
        nb.nimble_dense_variant_dyn(px, pw, pb, py, M, N, K, epilogue, out_dtype, force_variant, ws.data_ptr(),
                                    ws.numel() * ws.element_size(), _stream())
    return y


def batch_matmul(a: torch.Tensor, b: torch.Tensor, trans_b: bool, alpha: float = 1.0,
                 out_dtype: int = nb.BF16, out: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    T, M, N = nb.batch_matmul_shape(tuple(a.shape), tuple(b.shape), trans_b)
    K = a.shape[2]
    c = out if out is not None else _alloc((T, M, N), out_dtype, a.device)
    ws = workspace if workspace is not None else default_workspace(a.device)   # b transposed, for the NN product
    nb.nimble_batch_matmul_dyn(_ptr(a, _BF, "a"), _ptr(b, _BF, "b"), _ptr(c, _TORCH_DTYPE[out_dtype], "c"), T, M, N, K,
                               trans_b, alpha, out_dtype, ws.data_ptr(), ws.numel() * ws.element_size(), _stream())
    return c


def softmax_rows(s: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    cols = s.shape[-1]
    rows = s.numel() // cols if cols else 0
    p = out if out is not None else _alloc(tuple(s.shape), nb.BF16, s.device)
    nb.nimble_softmax_rows_dyn(_ptr(s, _F32, "s"), _ptr(p, _BF, "p"), rows, cols, _stream())
    return p


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
              alpha: float = 0.125) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """S = alpha Q.K^T (f32), P = softmax rows (bf16), O = P.V (bf16), through one entry point: one launch
    for head dimension 64 and up to 512 tokens, the three calls otherwise."""
    r = _host_calls.attention(q, k, v, alpha)
    if r is not None:
        return r
    T, M, N = nb.batch_matmul_shape(tuple(q.shape), tuple(k.shape), True)
    _, _, Dv = nb.batch_matmul_shape((T, M, N), tuple(v.shape), False)
    s, p = _alloc((T, M, N), nb.F32, q.device), _alloc((T, M, N), nb.BF16, q.device)
    o = _alloc((T, M, Dv), nb.BF16, q.device)
    ws = default_workspace(q.device)
    nb.nimble_attention_chain_dyn(_ptr(q, _BF, "q"), _ptr(k, _BF, "k"), _ptr(v, _BF, "v"), _ptr(s, _F32, "s"),
                                  _ptr(p, _BF, "p"), _ptr(o, _BF, "o"), T, M, N, q.shape[2], Dv, alpha, ws.data_ptr(),
                                  ws.numel() * ws.element_size(), _stream())
    return s, p, o


def fused_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, alpha: float = 0.125,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """O = softmax(alpha Q.K^T).V in one launch.  The composite's shape function is the two
    batch_matmul shape functions connected: (T,L,D)x(T,L,D)^T -> (T,L,L), then x(T,L,D) -> (T,L,D)."""
    if out is None:
        o = _host_calls.fused_attention(q, k, v, alpha)
        if o is not None:
            return o
    s_shape = nb.batch_matmul_shape(tuple(q.shape), tuple(k.shape), True)
    T, L, D = nb.batch_matmul_shape(s_shape, tuple(v.shape), False)
    o = out if out is not None else _alloc((T, L, D), nb.BF16, q.device)
    nb.nimble_attention_dyn(_ptr(q, _BF, "q"), _ptr(k, _BF, "k"), _ptr(v, _BF, "v"), _ptr(o, _BF, "o"), T, L, D, alpha,
                            _stream())
    if not _bound:
        _bind_host_calls(q.device)
    return o


def _together(**tensors):
    """The device that all of these tensors are on, made the current one for the call: the library launches on the stream of
    the current device."""
    device = None
    for what, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda or (device is not None and t.device != device):
            raise nb.NimbleError(-8, f"{what} is on {t.device}" + (f", the operands before it on {device}" if device is not None else
                                                                   ", not on a GPU"))
        device = t.device
    return torch.cuda.device(device)


def _output(out: Optional[torch.Tensor], shape, dtype: int, device, what: str) -> torch.Tensor:
    if dtype not in (nb.BF16, nb.F32):
        raise nb.NimbleError(-4, f"{what}: unknown output dtype {dtype}")
    if out is None:
        return _alloc(shape, dtype, device)
    if tuple(out.shape) != tuple(shape):
        raise nb.NimbleError(-3, f"{what}: out is {tuple(out.shape)}, the shape function gives {tuple(shape)}")
    return out


def _bias(bias: Optional[torch.Tensor], shape, epilogue: int, what: str) -> int:
    if epilogue == nb.EPI_NONE:
        return 0
    if bias is None:
        raise nb.NimbleError(-1, f"{what}: this epilogue needs a bias")
    if tuple(bias.shape) != tuple(shape):
        raise nb.NimbleError(-3, f"{what}: bias is {tuple(bias.shape)}, {tuple(shape)} needed")
    return _ptr(bias, _BF, "bias")


def quantize_rows(x: torch.Tensor, cols: int = 0) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows of x [M, K] (bf16 or f32) as 8-bit codes q [M, cols] and a scale each (f32 [M]): x is about q * scale.  Codes past K are
    0; cols = 0 rounds K up to whole 128 bytes.  Serves tokens and, row by row of w [N, K], output channels alike; a stack of
    experts' weights w [E, N, K] is quantised as w.view(E * N, K) and its results viewed back."""
    r = _host_calls.quantize_rows(x, cols)
    if r is not None:
        return r
    q_shape, s_shape = nb.quantize_rows_shape(tuple(x.shape), cols)
    if x.dtype not in (_BF, _F32):
        raise nb.NimbleError(-4, f"quantize_rows: x is {x.dtype}")
    with _together(x=x):
        px = _ptr(x, x.dtype, "x")
        q, scale = _alloc(q_shape, nb.I8, x.device), _alloc(s_shape, nb.F32, x.device)
        nb.nimble_quantize_rows_dyn(px, nb.BF16 if x.dtype is _BF else nb.F32, q.data_ptr(), scale.data_ptr(), x.shape[0], x.shape[1],
                                    q_shape[1], _stream())
    if not _bound:
        _bind_host_calls(x.device)
    return q, scale


def dense_i8(x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
             epilogue: int = nb.EPI_BIAS, out_dtype: int = nb.BF16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dense in 8-bit integers: y = epi(x_scale[m] w_scale[n] x.w^T + bias), x [M, K] and w [N, K] int8 with their scales (the results of
    quantize_rows), sums exact in 32 bits."""
    r = _host_calls.product(x, x_scale, w, w_scale, bias, None, epilogue, out_dtype, out)
    if r is not None:
        return r
    M, N = nb.dense_i8_shape(tuple(x.shape), tuple(x_scale.shape), tuple(w.shape), tuple(w_scale.shape))
    with _together(x=x, x_scale=x_scale, w=w, w_scale=w_scale, bias=bias, out=out):
        y = _output(out, (M, N), out_dtype, x.device, "dense_i8")
        nb.nimble_dense_i8_dyn(_ptr(x, torch.int8, "x"), _ptr(x_scale, _F32, "x_scale"), _ptr(w, torch.int8, "w"),
                               _ptr(w_scale, _F32, "w_scale"), _bias(bias, (N,), epilogue, "dense_i8"),
                               _ptr(y, _TORCH_DTYPE[out_dtype], "y"), M, N, x.shape[1], epilogue, out_dtype, _stream())
    if not _bound:
        _bind_host_calls(x.device)
    return y


def grouped_dense(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor], offsets: torch.Tensor, epilogue: int = nb.EPI_BIAS,
                  out_dtype: int = nb.BF16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dense for rows that belong to E groups (experts) with a weight each: rows offsets[e] .. offsets[e+1]-1 of x [R, K] times
    w[e] of [E, N, K], bias [E, N].  offsets [E+1] is int64 on the GPU and is not waited for.  Rows of no group are left as they
    were in `out` (unspecified in a new output)."""
    r = _host_calls.product(x, None, w, None, bias, offsets, epilogue, out_dtype, out)
    if r is not None:
        return r
    R, N = nb.grouped_dense_shape(tuple(x.shape), tuple(w.shape), tuple(offsets.shape))
    with _together(x=x, w=w, bias=bias, offsets=offsets, out=out):
        y = _output(out, (R, N), out_dtype, x.device, "grouped_dense")
        nb.nimble_grouped_dense_dyn(_ptr(x, _BF, "x"), _ptr(w, _BF, "w"), _bias(bias, w.shape[:2], epilogue, "grouped_dense"),
                                    _ptr(offsets, torch.int64, "offsets"), _ptr(y, _TORCH_DTYPE[out_dtype], "y"), R, w.shape[0], N,
                                    x.shape[1], epilogue, out_dtype, _stream())
    if not _bound:
        _bind_host_calls(x.device)
    return y


def grouped_dense_i8(x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor],
                     offsets: torch.Tensor, epilogue: int = nb.EPI_BIAS, out_dtype: int = nb.BF16,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """grouped_dense in 8-bit integers: x [R, K] int8 with x_scale [R], w [E, N, K] int8 with w_scale [E, N]."""
    r = _host_calls.product(x, x_scale, w, w_scale, bias, offsets, epilogue, out_dtype, out)
    if r is not None:
        return r
    R, N = nb.grouped_dense_shape(tuple(x.shape), tuple(w.shape), tuple(offsets.shape))
    if tuple(x_scale.shape) != (R,) or tuple(w_scale.shape) != tuple(w.shape[:2]):
        raise nb.NimbleError(-3, f"grouped_dense_i8: scales of {tuple(x_scale.shape)} and {tuple(w_scale.shape)} for x {tuple(x.shape)} "
                                 f"and w {tuple(w.shape)}")
    with _together(x=x, x_scale=x_scale, w=w, w_scale=w_scale, bias=bias, offsets=offsets, out=out):
        y = _output(out, (R, N), out_dtype, x.device, "grouped_dense_i8")
        nb.nimble_grouped_dense_i8_dyn(_ptr(x, torch.int8, "x"), _ptr(x_scale, _F32, "x_scale"), _ptr(w, torch.int8, "w"),
                                       _ptr(w_scale, _F32, "w_scale"), _bias(bias, w.shape[:2], epilogue, "grouped_dense_i8"),
                                       _ptr(offsets, torch.int64, "offsets"), _ptr(y, _TORCH_DTYPE[out_dtype], "y"), R, w.shape[0], N,
                                       x.shape[1], epilogue, out_dtype, _stream())
    if not _bound:
        _bind_host_calls(x.device)
    return y


class Sequences(NamedTuple):
    """The rows of one call, on the GPU: rows offsets[s] .. offsets[s+1]-1 are the new tokens of sequence s, the last of its lengths[s];
    position p of it is in slot p % page of page pages[s, p // page].  offsets [S+1] and lengths [S] int64, pages [S, W] int32."""
    offsets: torch.Tensor
    lengths: torch.Tensor
    pages: torch.Tensor


class PagedCache(NamedTuple):
    """Keys and values of sequences in pages: k, v [pages, kv_heads, page, D] bf16, or int8 with scales [pages, kv_heads, page] f32.  page is a
    power of two from 16 to 1024, D 64 or 128."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None

    @staticmethod
    def empty(pages: int, kv_heads: int, page: int, D: int, dtype: int = nb.BF16, device="cuda") -> "PagedCache":
        shape = (pages, kv_heads, page, D)
        scales = shape[:3] if dtype == nb.I8 else None
        nb.cache_check(shape, shape, scales, scales, dtype, (1,), (0,), (0, 0))
        k, v = (_alloc(shape, dtype, device) for _ in range(2))
        return PagedCache(k, v, *((_alloc(scales, nb.F32, device) for _ in range(2)) if scales else (None, None)))


def _paged(cache: PagedCache, sequences: Sequences, rows: int):
    """The checked descriptions of a cache and a batch as the C ABI takes them."""
    k, v, ks, vs = cache
    if k.dtype not in (_BF, torch.int8):
        raise nb.NimbleError(-4, f"cache: keys are {k.dtype}, bf16 or int8 needed")
    int8 = k.dtype is torch.int8
    if int8 and (ks is None or vs is None):
        raise nb.NimbleError(-1, "cache: 8-bit codes need scales")
    off, lengths, pages = sequences
    dtype = nb.I8 if int8 else nb.BF16
    nb.cache_check(tuple(k.shape), tuple(v.shape), tuple(ks.shape) if int8 else None, tuple(vs.shape) if int8 else None, dtype,
                   tuple(off.shape), tuple(lengths.shape), tuple(pages.shape))
    c = nb.cache(_ptr(k, k.dtype, "k"), _ptr(v, k.dtype, "v"), _ptr(ks, _F32, "k_scale") if int8 else 0,
                 _ptr(vs, _F32, "v_scale") if int8 else 0, *k.shape, dtype)
    s = nb.sequences(_ptr(off, torch.int64, "offsets"), _ptr(lengths, torch.int64, "lengths"), _ptr(pages, torch.int32, "pages"),
                     lengths.shape[0], pages.shape[1], rows)
    return c, s


def _rows_ptr(t: torch.Tensor, what: str) -> Tuple[int, int]:
    """Address and row stride of heads [T, H, D] that lie one after the other within a row, the rows any stride apart."""
    if t.dtype is not _BF or not t.is_cuda or (t.numel() and (t.stride(2) != 1 and t.shape[2] > 1 or t.stride(1) != t.shape[2] and t.shape[1] > 1)):
        raise nb.NimbleError(-4 if t.dtype is not _BF else -8, f"{what}: need a {_BF} tensor on the GPU whose heads are contiguous, got {t.dtype}, "
                                                               f"device {t.device}, strides {tuple(t.stride())}")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]


def rotary_table(positions: int, rot: int, base: float = 10000.0, factor: float = 1.0, trained: float = 0.0, low: float = 1.0,
                 high: float = 32.0, magnitude: float = 1.0, device="cuda") -> torch.Tensor:
    """cos and sin, times `magnitude`, of the angles position * f_i of `rot` turned elements: f32 [positions, rot/2, 2], computed in f64.
    f_i = base^(-2i/rot).  For contexts `factor` times as long as the trained ones f_i is divided by factor where pair i makes fewer than `low`
    turns within `trained` positions, kept where it makes more than `high`, blended between; trained = 0: all are divided."""
    shape = (int(positions), int(rot) // 2, 2)
    table = _alloc(shape, nb.F32, device)
    with _together(table=table):
        nb.nimble_rotary_table_dyn(table.data_ptr(), positions, rot, base, factor, trained, low, high, magnitude, _stream())
    return table


def rotary(x: torch.Tensor, positions: torch.Tensor, table: torch.Tensor, interleaved: bool = False,
           out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotary positions: the first 2R elements of each head of x [T, H, D] (bf16, rows any stride apart) turned in pairs (i, i + R), or (2i, 2i + 1)
    where interleaved, by table[positions[t]] of [P, R, 2] (rotary_table); the rest copied.  positions [T] int64; out may be x."""
    r = _host_calls.rotary(x, positions, table, interleaved, out)
    if r is not None:
        return r
    shape = nb.rotary_shape(tuple(x.shape), tuple(positions.shape), tuple(table.shape))
    with _together(x=x, positions=positions, table=table, out=out):
        y = out if out is not None else _alloc(shape, nb.BF16, x.device)
        if tuple(y.shape) != shape:
            raise nb.NimbleError(-3, f"rotary: out is {tuple(y.shape)}, the shape function gives {shape}")
        px, xs = _rows_ptr(x, "x")
        py, ys = _rows_ptr(y, "out")
        nb.nimble_rotary_dyn(px, xs, _ptr(positions, torch.int64, "positions"), _ptr(table, _F32, "table"), table.shape[0], py, ys, *shape,
                             table.shape[1], interleaved, _stream())
    if not _bound:
        _bind_host_calls(x.device)
    return y


def cache_write(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, sequences: Sequences, q: Optional[torch.Tensor] = None,
                table: Optional[torch.Tensor] = None, interleaved: bool = False, out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Keys and values k, v [T, kv_heads, D] of a batch's rows into their places of the cache; with a table (rotary_table) the keys are
    turned by their positions first, and the queries q [T, heads, D] with them: returns these, contiguous (`out` may be q where that is), or None without q.
    An 8-bit cache holds each token and head as quantize_rows does.  k, v and q may be parts of wider rows."""
    r = _host_calls.cache_write(cache, k, v, sequences, q, table, interleaved, out)
    if r is not None:
        return None if r is True else r
    shape = nb.cache_write_shape(tuple(cache.k.shape), tuple(k.shape), tuple(v.shape), None if q is None else tuple(q.shape))
    if table is not None and (table.dim() != 3 or table.shape[2] != 2):
        raise nb.NimbleError(-3, f"cache_write: a table of {tuple(table.shape)}, (positions, pairs, 2) needed")
    if q is None and out is not None:
        raise nb.NimbleError(-8, "cache_write: out without q")
    with _together(k=k, v=v, q=q, table=table, out=out, cache_k=cache.k, cache_v=cache.v, k_scale=cache.k_scale, v_scale=cache.v_scale,
                   **sequences._asdict()):
        c, s = _paged(cache, sequences, k.shape[0])
        y = out
        if q is not None and out is None:
            y = _alloc(shape, nb.BF16, k.device)
        elif q is not None and tuple(out.shape) != shape:
            raise nb.NimbleError(-3, f"cache_write: out is {tuple(out.shape)}, the shape function gives {shape}")
        nb.nimble_cache_write_dyn(c, s, *_rows_ptr(k, "k"), *_rows_ptr(v, "v"), *(_rows_ptr(q, "q") if q is not None else (0, 0)),
                                  _ptr(y, _BF, "out") if q is not None else 0, q.shape[1] if q is not None else 0,
                                  *((_ptr(table, _F32, "table"), table.shape[0], table.shape[1]) if table is not None else (0, 0, 0)),
                                  interleaved, _stream())
    if not _bound:
        _bind_host_calls(k.device)
    return y


def cache_read(cache: PagedCache, sequences: Sequences, rows: int, out_dtype: int = nb.BF16,
               out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The keys and values of a batch's rows back out of the cache, each [rows, kv_heads, D] of out_dtype: the inverse of cache_write.  offsets that
    count each sequence's whole length read all of it.  Rows of no sequence are left as they were in `out`."""
    if out is None:
        r = _host_calls.cache_read(cache, sequences, rows, out_dtype)
        if r is not None:
            return r
    shape = nb.cache_read_shape(tuple(cache.k.shape), rows)
    ko, vo = out if out is not None else (None, None)
    with _together(cache_k=cache.k, cache_v=cache.v, k_scale=cache.k_scale, v_scale=cache.v_scale, k_out=ko, v_out=vo, **sequences._asdict()):
        c, s = _paged(cache, sequences, rows)
        ko, vo = (_output(t, shape, out_dtype, cache.k.device, "cache_read") for t in (ko, vo))
        nb.nimble_cache_read_dyn(c, s, _ptr(ko, _TORCH_DTYPE[out_dtype], "k_out"), _ptr(vo, _TORCH_DTYPE[out_dtype], "v_out"), out_dtype, _stream())
    if not _bound:
        _bind_host_calls(ko.device)
    return ko, vo


def paged_attention(q: torch.Tensor, cache: PagedCache, sequences: Sequences, alpha: Optional[float] = None, window: int = 0,
                    out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of a batch's rows q [T, heads, D] over their sequences in the cache, what cache_write has just put there included: row i of a
    sequence, at position p, sees the keys max(0, p - window + 1) .. p (window = 0: all up to p); heads is a multiple of the cache's, whose
    heads / kv_heads query heads share keys.  alpha: 1 / sqrt(D) unless given.  A token of each sequence and chunks of many are served alike.
    out shares no memory with q or the cache.  workspace: of nb.paged_attention_plan's size, for one call at a time; by default a new one, so that calls
    may overlap."""
    if workspace is None:
        o = _host_calls.paged_attention(q, cache, sequences, alpha if alpha is not None else q.shape[2] ** -0.5 if q.dim() == 3 and q.shape[2] else None, window, out)
        if o is not None:
            return o
    shape = nb.paged_attention_shape(tuple(q.shape), tuple(cache.k.shape))
    with _together(q=q, out=out, workspace=workspace, cache_k=cache.k, cache_v=cache.v, k_scale=cache.k_scale, v_scale=cache.v_scale,
                   **sequences._asdict()):
        c, s = _paged(cache, sequences, q.shape[0])
        y = _output(out, shape, nb.BF16, q.device, "paged_attention")
        if workspace is None:
            need = nb.paged_attention_plan(shape[0], s.count, s.width, shape[1], c.kv_heads, c.page, c.D, c.dtype, window).workspace_bytes
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        nb.nimble_paged_attention_dyn(*_rows_ptr(q, "q"), c, s, _ptr(y, _BF, "out"), shape[1], alpha if alpha is not None else shape[2] ** -0.5,
                                      window, workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream())
    if not _bound:
        _bind_host_calls(q.device)
    return y


def lstm_step(x: torch.Tensor, h: torch.Tensor, w: torch.Tensor, bias: torch.Tensor, c: torch.Tensor,
              h_out: Optional[torch.Tensor] = None,
              c_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    (B, H), _ = nb.lstm_shape(tuple(x.shape), tuple(h.shape), tuple(c.shape), tuple(w.shape))
    Ix = x.shape[1]
    if h_out is None:
        h_out = _alloc((B, H), nb.BF16, x.device)
    if c_out is None:
        c_out = _alloc((B, H), nb.F32, x.device)
    nb.nimble_lstm_gates_dyn(_ptr(x, _BF, "x"), _ptr(h, _BF, "h"), _ptr(w, _BF, "w"), _ptr(bias, _BF, "bias"),
                             _ptr(c, _F32, "c"), _ptr(c_out, _F32, "c_out"), _ptr(h_out, _BF, "h_out"), B, Ix, H, 0, 0,
                             _stream())
    return h_out, c_out


def lstm_step_pre(pre: torch.Tensor, h: torch.Tensor, w_h: torch.Tensor, c: torch.Tensor,
                  h_out: Optional[torch.Tensor] = None,
                  c_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """One cell step from the precomputed input share of the gates pre [B, 4H] (f32)."""
    (B, H), _ = nb.lstm_pre_shape(tuple(pre.shape), tuple(h.shape), tuple(c.shape), tuple(w_h.shape))
    if h_out is None:
        h_out = _alloc((B, H), nb.BF16, h.device)
    if c_out is None:
        c_out = _alloc((B, H), nb.F32, h.device)
    nb.nimble_lstm_gates_pre_dyn(_ptr(pre, _F32, "pre"), _ptr(h, _BF, "h"), _ptr(w_h, _BF, "w_h"), _ptr(c, _F32, "c"),
                                 _ptr(c_out, _F32, "c_out"), _ptr(h_out, _BF, "h_out"), B, H, _stream())
    return h_out, c_out


# polls per wait of the one-launch token loop before it gives up (a poll is a round trip to memory, 0.5-1 us:
# a quarter of a second at the very most)
LSTM_SEQ_MAX_POLLS = 1 << 18
# polls per wait of the loop with a recovery launch behind it before that takes over (some 8 ms, about what it takes itself)
LSTM_LOOP_MAX_POLLS = 1 << 14


def lstm_sequence_pre(pre: torch.Tensor, w_h: torch.Tensor, h0: torch.Tensor, c0: torch.Tensor,
                      max_polls: int = LSTM_SEQ_MAX_POLLS, one_launch: Optional[bool] = None,
                      workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, bool]:
    """The token loop of one sequence from the inputs' share of the gates pre [T, B, 4H] (f32):
    returns (h_seq [T,B,H] bf16, c_T [B,H] f32, ran_in_one_launch).

    one_launch=None: shapes for which nimble_lstm_seq_preferred says so run as one launch
    (nimble_lstm_seq_pre_dyn), others by nimble_lstm_loop_preferred through nimble_lstm_loop_dyn, whose
    own recovery launch stands behind it, so that nothing is waited for and the third value is False (it is
    not known then) as for steps; True: every shape nimble_lstm_seq_supported accepts runs as one launch (others
    raise); False: none.  After a one-launch run the call waits for the stream and reads the loop's give-up word;
    if the loop gave up, or neither was taken, the steps run one by one through
    nimble_lstm_gates_pre_dyn.  All three give the same bits.
    workspace: of the one-launch run; the others need none or bring their own.
    Two loops find their places on the GPU beside each other; programs that run more at once ask for steps (False)."""
    (T, B, H), _ = nb.lstm_seq_shape(tuple(pre.shape), tuple(h0.shape), tuple(c0.shape), tuple(w_h.shape))
    dev = h0.device
    h_seq = _alloc((T, B, H), nb.BF16, dev)
    c_out = _alloc((B, H), nb.F32, dev)
    pp, wp, hp, cp = _ptr(pre, _F32, "pre"), _ptr(w_h, _BF, "w_h"), _ptr(h0, _BF, "h0"), _ptr(c0, _F32, "c0")
    if T == 0:
        c_out.copy_(c0)
        return h_seq, c_out, False
    supported = nb.lstm_seq_supported(B, H)
    if one_launch and not supported:
        raise nb.NimbleError(-3, f"the one-launch token loop does not run B={B}, H={H}")
    if one_launch is None:
        one_launch = nb.lstm_seq_preferred(B, H)
        # 128 steps of 3 rows at H = 1024 took 748 us as eager steps (projection included), 215 in the loop.  An eager step
        # takes its caller 5 us: 2 steps of 20 rows at H = 512 22.6 us, 20.0 in the loop (one 17.4 / 20.1); 12 of 256 96.9 / 87.4
        # (8 65.5 / 68.2)
        if not one_launch and nb.lstm_loop_preferred(T + 5, B, 0, H):
            ws = torch.empty(nb.lstm_loop_workspace_bytes(B, 0, H), dtype=torch.uint8, device=dev)
            if cp % 16:  # (any alignment of c0 will do here, as for steps)
                c_out.copy_(c0)
                cp = c_out.data_ptr()
            nb.nimble_lstm_loop_dyn(0, pp, wp, 0, hp, cp, h_seq.data_ptr(), c_out.data_ptr(), T, B, 0, H, ws.data_ptr(),
                                    ws.numel(), min(max_polls, LSTM_LOOP_MAX_POLLS), _stream())
            return h_seq, c_out, False
    if supported and one_launch:
        need = nb.lstm_seq_workspace_bytes(B, H)
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        nb.nimble_lstm_seq_pre_dyn(pp, wp, hp, cp, h_seq.data_ptr(), c_out.data_ptr(), T, B, H,
                                   _ptr(workspace, torch.uint8, "workspace"), workspace.numel(), max_polls, _stream())
        if not nb.nimble_lstm_seq_status(workspace.data_ptr(), _stream()):
            return h_seq, c_out, True
    st = _stream()
    c_out.copy_(c0)
    for t in range(T):
        nb.nimble_lstm_gates_pre_dyn(pre[t].data_ptr(), (h0 if t == 0 else h_seq[t - 1]).data_ptr(), wp,
                                     c_out.data_ptr(), c_out.data_ptr(), h_seq[t].data_ptr(), B, H, st)
    return h_seq, c_out, False


def lstm_sequence(xs: torch.Tensor, w_x: torch.Tensor, w_h: torch.Tensor, bias: torch.Tensor, h0: torch.Tensor,
                  c0: torch.Tensor, **kw) -> Tuple[torch.Tensor, torch.Tensor, bool]:
    """A whole sequence xs [T, B, Ix] through the cell: the inputs' share of the gates for all T*B tokens in one
    dense call (M = T*B dynamic, f32 output), then the token loop (lstm_sequence_pre).  w_x [4H, Ix] and
    w_h [4H, H] are the two halves of the fused weight (split_lstm_weight)."""
    if not kw:
        r = _host_calls.lstm_sequence(xs, w_x, w_h, bias, h0, c0, LSTM_SEQ_MAX_POLLS)
        if isinstance(r, tuple):
            return r
        if r is not None:  # the loop gave up
            return lstm_sequence_pre(r, w_h, h0, c0, one_launch=False)
    T, B, Ix = xs.shape
    pre = dense(xs.view(T * B, Ix), w_x, bias, nb.EPI_BIAS, nb.F32)
    return lstm_sequence_pre(pre.view(T, B, w_x.shape[0]), w_h, h0, c0, **kw)


def split_lstm_weight(w: torch.Tensor, Ix: int) -> Tuple[torch.Tensor, torch.Tensor]:
    """One-time split of the fused weight [4H, Ix+H] into contiguous input and recurrent halves."""
    return w[:, :Ix].contiguous(), w[:, Ix:].contiguous()


class LstmSequenceGraph:
    """The token loop of one sequence, captured once per batch size B as a HIP graph and replayed: where
    nimble_lstm_loop_preferred says so the loop is one launch (with a recovery launch behind it that ends at once
    unless the loop's bounded waits ran out), else `steps` launches of the fused LSTM cell, with the same bits.  The graph
    holds kernel launches only (state is cleared by a fill kernel outside it).  The dynamic extent
    B is fixed per graph; a server keeps one graph per batch size it has seen.

    run() starts from zero.  `graph` itself goes on from what hs[0] and c hold, so that a program which takes a long sequence
    in parts puts the last h into hs[0], leaves c as it is and replays it.

    Two such loops find their places on the GPU beside each other.  Of three or more that replay at the same time some
    can run out of their waits, which costs milliseconds: four of 64 rows at H = 512 took 0.4 ms for 64 steps, and 17 in
    the one round of 17 where that happened; as launches per step (one_launch=False) 0.5."""

    def __init__(self, w: torch.Tensor, bias: torch.Tensor, B: int, steps: int, Ix: int, H: int,
                 project_inputs: bool = False, one_launch: Optional[bool] = None):
        """project_inputs: compute the inputs' share of the gates for all tokens in one dense
        call (M = steps * B) ahead of the loop, so each step streams only the recurrent half
        of the weight.
        one_launch: None: the loop in one launch where that is preferred (nimble_lstm_loop_preferred); True: where it is
        supported, other shapes raise;
        False: a launch per step, for programs that replay three or more of these graphs at once."""
        dev = w.device
        (self.B, self.H), _ = nb.lstm_shape((B, Ix), (B, H), (B, H), tuple(w.shape))
        self.steps, self.Ix = steps, Ix
        self.w, self.bias = w, bias
        self.project_inputs = project_inputs
        if project_inputs:
            self.w_x, self.w_h = split_lstm_weight(w, Ix)
            self.pre = torch.empty((steps, B, 4 * H), dtype=torch.float32, device=dev)
        self.xs = torch.zeros((steps, B, Ix), dtype=torch.bfloat16, device=dev)
        self.hs = torch.zeros((steps + 1, B, H), dtype=torch.bfloat16, device=dev)  # hs[0] = h_0
        self.c = torch.zeros((B, H), dtype=torch.float32, device=dev)
        # one fill clears both (c seen as bf16: all of one type): 128 steps of 37 rows at H = 512 186.1 -> 184.5 us, 32 of one
        # row 57.8 -> 56.5
        self._first_state = [self.hs[0], self.c.view(torch.bfloat16)]
        loop_ix = 0 if project_inputs else Ix
        self.workspace = None
        supported = (project_inputs or Ix > 0) and nb.lstm_loop_supported(B, loop_ix, H)
        if one_launch and not supported:
            raise nb.NimbleError(-3, f"the one-launch token loop does not run B={B}, Ix={loop_ix}, H={H}")
        if one_launch or (one_launch is None and supported and nb.lstm_loop_preferred(steps, B, loop_ix, H)):
            self.workspace = torch.empty(nb.lstm_loop_workspace_bytes(B, loop_ix, H), dtype=torch.uint8, device=dev)
        # one eager pass so that nothing is lazily initialised during capture
        self._enqueue()
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self._enqueue()

    def _enqueue(self) -> None:
        st = _stream()
        if self.project_inputs:
            dense(self.xs.view(self.steps * self.B, self.Ix), self.w_x, self.bias, nb.EPI_BIAS, nb.F32,
                  out=self.pre.view(self.steps * self.B, 4 * self.H))
        if self.workspace is not None:
            w = self.w_h if self.project_inputs else self.w
            nb.nimble_lstm_loop_dyn(self.xs.data_ptr(), self.pre.data_ptr() if self.project_inputs else 0, w.data_ptr(),
                                    self.bias.data_ptr(), self.hs.data_ptr(), self.c.data_ptr(), self.hs[1:].data_ptr(),
                                    self.c.data_ptr(), self.steps, self.B, 0 if self.project_inputs else self.Ix, self.H,
                                    self.workspace.data_ptr(), self.workspace.numel(), LSTM_LOOP_MAX_POLLS, st)
            return
        if self.project_inputs:
            for t in range(self.steps):
                nb.nimble_lstm_gates_pre_dyn(self.pre[t].data_ptr(), self.hs[t].data_ptr(), self.w_h.data_ptr(),
                                             self.c.data_ptr(), self.c.data_ptr(), self.hs[t + 1].data_ptr(),
                                             self.B, self.H, st)
            return
        for t in range(self.steps):
            nb.nimble_lstm_gates_dyn(self.xs[t].data_ptr(), self.hs[t].data_ptr(), self.w.data_ptr(),
                                     self.bias.data_ptr(), self.c.data_ptr(), self.c.data_ptr(),
                                     self.hs[t + 1].data_ptr(), self.B, self.Ix, self.H, 0, 0, st)

    def run(self, xs: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Run the sequence from h_0 = c_0 = 0; returns (all h_t [steps,B,H], final c)."""
        if xs is not None:
            self.xs.copy_(xs)
        torch._foreach_zero_(self._first_state)
        self.graph.replay()
        return self.hs[1:], self.c
