"""Performance cases of the 8-bit and the grouped products: quantize_rows, dense_i8, grouped_dense, grouped_dense_i8.

The layer sizes are those of the BERT-large feed-forward block in ``workloads.py`` (1024 -> 4096 -> 1024) and of the wide layers of
``bench.py``, and generic odd ones; the token counts are one token, small batches and the ragged batch of 32 sentences (8177 tokens
on average), twice that where every token goes to two experts.  ``run`` computes an operator in its plain form from elementary
torch operations, or, where ``own`` is true, calls the library.
"""
import math

import torch

own = False

D, F = 1024, 4096   # BERT-large feed-forward block
TOKENS = 8177       # tokens of a ragged batch of 32 sentences of up to 512


def listed():
    return [
        # one token's activations on the way into an 8-bit layer
        {"name": "quantize_token", "kind": "quantize", "M": 1, "K": F, "dtype": "bf16"},
        # the hidden activations of a whole batch
        {"name": "quantize_batch", "kind": "quantize", "M": TOKENS, "K": F, "dtype": "bf16"},
        # laying out f32 weights of a layer with odd extents (rows padded by the operator)
        {"name": "quantize_weights", "kind": "quantize", "M": 1001, "K": 1003, "dtype": "f32"},
        # one token through the first layer of the block
        {"name": "dense_i8_token", "kind": "dense_i8", "M": 1, "N": F, "K": D, "epilogue": "bias", "out": "bf16"},
        # a small batch through the second layer
        {"name": "dense_i8_small", "kind": "dense_i8", "M": 200, "N": D, "K": F, "epilogue": "bias", "out": "bf16"},
        # f32 logits of a layer whose extents are nobody's multiple
        {"name": "dense_i8_odd", "kind": "dense_i8", "M": 515, "N": 1001, "K": 1040, "epilogue": "none", "out": "f32"},
        # the ragged batch through the first layer
        {"name": "dense_i8_batch", "kind": "dense_i8", "M": TOKENS, "N": F, "K": D, "epilogue": "bias_gelu", "out": "bf16"},
        # four tokens at two experts each: the weights of the experts that are hit stream from memory
        {"name": "grouped_token", "kind": "grouped", "rows": 8, "E": 16, "live": 6, "spare": 0, "N": F, "K": D,
         "epilogue": "bias_gelu", "out": "bf16"},
        # odd extents, empty experts, rows behind the last expert's that stay as they were
        {"name": "grouped_odd", "kind": "grouped", "rows": 515, "E": 7, "live": 5, "spare": 13, "N": 1001, "K": 1000,
         "epilogue": "none", "out": "f32"},
        # a batch at two experts each, first layer of the experts
        {"name": "grouped_batch", "kind": "grouped", "rows": 2 * TOKENS, "E": 8, "live": 8, "spare": 0, "N": F, "K": D,
         "epilogue": "bias_gelu", "out": "bf16"},
        # sixteen rows over many small experts in 8 bits, second layer
        {"name": "grouped_i8_token", "kind": "grouped_i8", "rows": 16, "E": 64, "live": 13, "spare": 0, "N": D, "K": F,
         "epilogue": "bias", "out": "bf16"},
        # a batch over 32 experts in 8 bits, second layer; unevenly filled
        {"name": "grouped_i8_batch", "kind": "grouped_i8", "rows": 2 * TOKENS, "E": 32, "live": 31, "spare": 0, "N": D, "K": F,
         "epilogue": "bias", "out": "bf16"},
    ]


MOST_OPS = 2 * 2 * TOKENS * F * D        # of the largest listed product
MOST_WEIGHTS = 64 * D * F                # elements of the largest listed stack of experts
MOST_VALUES = TOKENS * F                 # elements of the largest listed activation


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _extent(rng, lo, hi, unit):
    """Mostly a multiple of 128, else of `unit`, now and then any number."""
    n = _log(rng, lo, hi)
    p = rng.random()
    step = 128 if p < 0.6 else unit if p < 0.9 else 1
    return max(1, n // step) * step


def draw(rng):
    kind = rng.choice(("quantize", "dense_i8", "grouped", "grouped_i8"))
    if kind == "quantize":
        K = _extent(rng, 128, 8192, 8)
        return {"kind": kind, "M": _log(rng, 1, min(2 * TOKENS, MOST_VALUES // K)), "K": K, "dtype": rng.choice(("bf16", "bf16", "f32"))}
    epilogue, out = rng.choice((("none", "bf16"), ("none", "f32"), ("bias", "bf16"), ("bias", "f32"), ("bias_gelu", "bf16")))
    K = _extent(rng, 128, 8192, 16)
    N = _extent(rng, 128, 8192, 8)
    if kind == "dense_i8":
        return {"kind": kind, "M": _log(rng, 1, min(2 * TOKENS, MOST_OPS // (2 * N * K))), "N": N, "K": K, "epilogue": epilogue,
                "out": out}
    E = _log(rng, 1, max(1, min(64, MOST_WEIGHTS // (N * K))))
    rows = _log(rng, 1, min(2 * TOKENS, MOST_OPS // (2 * N * K)))
    live = rng.randint(max(1, min(E, rows) // 4), min(E, rows))
    return {"kind": kind, "rows": rows, "E": E, "live": live, "spare": rng.choice((0, 0, rng.randint(1, 64))), "N": N, "K": K,
            "epilogue": epilogue, "out": out}


# ---------------------------------------------------------------------------------------------- inputs
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, std):
    return torch.empty(shape, device="cuda").normal_(0, std, generator=g)


def _codes(g, shape):
    """8-bit codes as they come from normal values whose largest is some three times their spread."""
    return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(0, 42, generator=g).round_().clamp_(-127, 127).to(torch.int8)


def _stacked_codes(g, E, N, K):
    return torch.cat([_codes(g, (1, N, K)) for _ in range(E)])


def _scales(g, shape, size):
    return torch.empty(shape, device="cuda").uniform_(0.5 * size, 1.5 * size, generator=g)


def _group_sizes(g, rows, E, live):
    """`live` of the E experts get at least a row each; the others' shares fall off unevenly, as a router leaves them."""
    share = torch.rand(live, device="cuda", generator=g, dtype=torch.float64) ** 2 + 0.1
    cuts = torch.round(torch.cumsum(share, 0) / share.sum() * (rows - live)).long()
    n = torch.diff(cuts, prepend=cuts.new_zeros(1)) + 1
    sizes = torch.zeros(E, dtype=torch.int64, device="cuda")
    sizes[torch.randperm(E, device="cuda", generator=g)[:live]] = n
    return sizes


def prepare(case, seed):
    g = _generator(seed)
    kind = case["kind"]
    state = {"case": case}
    if kind == "quantize":
        x = _normal(g, (case["M"], case["K"]), 1.0)
        x *= torch.exp(_normal(g, (1, case["K"]), 0.5))                                  # channels of different size
        x[torch.rand(case["M"], device="cuda", generator=g) < (0.05 if case["M"] > 1 else 0)] = 0   # padding tokens
        state["x"] = x.to(_DTYPES[case["dtype"]])
        return state
    N, K = case["N"], case["K"]
    if kind == "dense_i8":
        state["x"], state["w"] = _codes(g, (case["M"], K)), _codes(g, (N, K))
        state["x_scale"], state["w_scale"] = _scales(g, (case["M"],), 0.02), _scales(g, (N,), 0.0005)
        state["bias"] = None if case["epilogue"] == "none" else _normal(g, (N,), 0.1).to(torch.bfloat16)
        return state
    E, rows, spare = case["E"], case["rows"], case["spare"]
    sizes = _group_sizes(g, rows, E, case["live"])
    state["offsets"] = torch.cat([sizes.new_zeros(1), torch.cumsum(sizes, 0)])
    state["capacity"] = int(sizes.max())      # rows that a program which pads its experts sets aside for each
    if kind == "grouped":
        state["x"] = _normal(g, (rows + spare, K), 1.0).to(torch.bfloat16)
        state["w"] = torch.cat([_normal(g, (1, N, K), 0.02).to(torch.bfloat16) for _ in range(E)])
    else:
        state["x"], state["w"] = _codes(g, (rows + spare, K)), _stacked_codes(g, E, N, K)
        state["x_scale"], state["w_scale"] = _scales(g, (rows + spare,), 0.02), _scales(g, (E, N), 0.0005)
    state["bias"] = None if case["epilogue"] == "none" else _normal(g, (E, N), 0.1).to(torch.bfloat16)
    state["out"] = torch.full((rows + spare, N), 0.25, device="cuda", dtype=_DTYPES[case["out"]])
    return state


# ---------------------------------------------------------------------------------------------- one pass
def _finish(y, bias, case):
    if bias is not None:
        y = y + bias
    if case["epilogue"] == "bias_gelu":
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y.to(_DTYPES[case["out"]])


def _quantize(state):
    x = state["x"].double()
    top = x.abs().amax(1, keepdim=True)
    q = torch.where(top > 0, torch.round(127 * x / top), 0.0).float()   # (64 bits: values at the border of two codes)
    scale = top.float() / 127
    return torch.nn.functional.pad(q * scale, (0, -x.shape[1] % 128)), scale[:, 0]


def _dense_i8(state):
    case = state["case"]
    y = state["x"].float() @ state["w"].float().t()
    y = y * state["x_scale"][:, None] * state["w_scale"]
    return _finish(y, None if state["bias"] is None else state["bias"].float(), case)


def _grouped(state):
    case, x, w, offsets, capacity = state["case"], state["x"], state["w"], state["offsets"], state["capacity"]
    E, N, K = w.shape
    row = torch.arange(x.shape[0], device=x.device)
    group = torch.searchsorted(offsets[1:], row, right=True)
    inside = group < E
    group = group.clamp(max=E - 1)
    slot = torch.where(inside, group * capacity + row - offsets[group], E * capacity)   # (one more slot for rows of no group)
    padded = torch.zeros((E * capacity + 1, K), device=x.device)
    padded[slot] = x.float()
    y = torch.bmm(padded[:-1].view(E, capacity, K), w.float().transpose(1, 2)).view(E * capacity, N)
    y = y[slot.clamp(max=E * capacity - 1)]
    if case["kind"] == "grouped_i8":
        y = y * state["x_scale"][:, None] * state["w_scale"][group]
    y = _finish(y, None if state["bias"] is None else state["bias"].float()[group], case)
    return torch.where(inside[:, None], y, state["out"])


def _own(state):
    import paper_2006_03031_amd as nb
    from paper_2006_03031_amd import runtime as rt
    case = state["case"]
    if case["kind"] == "quantize":
        q, scale = rt.quantize_rows(state["x"])
        return torch.mul(q, scale[:, None]), scale
    epilogue = {"none": nb.EPI_NONE, "bias": nb.EPI_BIAS, "bias_gelu": nb.EPI_BIAS_GELU_ERF}[case["epilogue"]]
    out = {"bf16": nb.BF16, "f32": nb.F32}[case["out"]]
    if case["kind"] == "dense_i8":
        return rt.dense_i8(state["x"], state["x_scale"], state["w"], state["w_scale"], state["bias"], epilogue, out)
    if case["kind"] == "grouped":
        return rt.grouped_dense(state["x"], state["w"], state["bias"], state["offsets"], epilogue, out, out=state["out"])
    return rt.grouped_dense_i8(state["x"], state["x_scale"], state["w"], state["w_scale"], state["bias"], state["offsets"], epilogue,
                               out, out=state["out"])


def run(state):
    if own:
        return _own(state)
    return {"quantize": _quantize, "dense_i8": _dense_i8, "grouped": _grouped, "grouped_i8": _grouped}[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------------------------- work and the exact results
def work(case):
    kind = case["kind"]
    if kind == "quantize":
        M, K = case["M"], case["K"]
        return {"bytes": M * K * (2 if case["dtype"] == "bf16" else 4) + M * (K + -K % 128) * 4 + 4 * M, "flops": 4 * M * K}
    N, K = case["N"], case["K"]
    out = 2 if case["out"] == "bf16" else 4
    rows, stacks, live = (case["M"], 1, 1) if kind == "dense_i8" else (case["rows"], case["E"], case["live"])
    size = 2 if kind == "grouped" else 1
    moved = size * (rows * K + live * N * K) + rows * N * out
    if kind != "grouped":
        moved += 4 * (rows + live * N)
    if case["epilogue"] != "none":
        moved += 2 * live * N
    if kind != "dense_i8":
        moved += 8 * (stacks + 1)
    return {"bytes": moved, "flops": 2 * rows * N * K}


def exact(case, seed):
    state = prepare(case, seed)
    x = state["x"].to(torch.float64)
    if case["kind"] == "quantize":
        top = x.abs().max(dim=1).values
        v = 127.0 * x / torch.where(top == 0, torch.ones_like(top), top)[:, None]
        low = torch.floor(v)
        part = v - low
        q = low + ((part > 0.5) | ((part == 0.5) & (torch.remainder(low, 2) == 1))).double()
        wide = torch.zeros((x.shape[0], x.shape[1] + -x.shape[1] % 128), dtype=torch.float64, device=x.device)
        wide[:, :x.shape[1]] = q * (top / 127.0)[:, None]
        return wide, top / 127.0
    if case["kind"] == "dense_i8":
        groups = [(0, case["M"], state["w"], state.get("w_scale"), state["bias"])]
        y = torch.empty((case["M"], case["N"]), dtype=torch.float64, device=x.device)
    else:
        ends = state["offsets"].tolist()
        groups = [(ends[e], ends[e + 1], state["w"][e], state["w_scale"][e] if "w_scale" in state else None,
                   None if state["bias"] is None else state["bias"][e]) for e in range(case["E"])]
        y = state["out"].double()
    for lo, hi, w, w_scale, bias in groups:
        if lo == hi:
            continue
        part = torch.matmul(x[lo:hi], w.double().t().contiguous())
        if w_scale is not None:
            part *= state["x_scale"][lo:hi, None].double() * w_scale.double()[None, :]
        if bias is not None:
            part += bias.double()
        if case["epilogue"] == "bias_gelu":
            part = part * torch.special.ndtr(part)
        y[lo:hi] = part
    return y
