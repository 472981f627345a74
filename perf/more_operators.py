"""Performance cases of the paged cache and what stands around it: rotary, cache_write, cache_read, paged_attention.

Head counts and widths are those of the BERT layers in ``workloads.py`` (16 or 12 heads of 64, each with keys of its own) and
generic ones whose query heads share keys (32 heads of 128 over 8); the token counts are one token, a token for each of many
sequences, chunks of a prompt, and the ragged batch of 32 sentences of up to 512.  ``run`` computes an operator in its plain form
from elementary torch operations, or, where ``own`` is true, calls the library.

A batch is described by three tensors on the GPU: ``offsets`` [S + 1] (rows offsets[s] .. offsets[s + 1] - 1 are the new tokens of
sequence s), ``lengths`` [S] (its tokens with the new ones, which are the last) and ``pages`` [S, W] (the pages that hold them).
"""
import math

import torch

own = False


def listed():
    return [
        # the queries of one token, far into a long context
        {"name": "rotary_token", "kind": "rotary", "T": 1, "H": 16, "D": 64, "rot": 64, "interleaved": False, "far": 120000},
        # a batch of prompts, half of each head rotated in neighbouring pairs, the heads read out of wider rows
        {"name": "rotary_batch", "kind": "rotary", "T": 8177, "H": 32, "D": 128, "rot": 64, "interleaved": True, "far": 4000},
        # serving: a new token of each of 64 sequences into a cache of 8 bits, keys and queries rotated on the way
        {"name": "write_tokens", "kind": "write", "S": 64, "idle": 3, "new": 1, "old": 90, "H": 32, "G": 8, "D": 128, "page": 16,
         "bits": 8, "rot": 128, "interleaved": False},
        # prompts of a ragged batch into a cache of bf16
        {"name": "write_batch", "kind": "write", "S": 32, "idle": 0, "new": 512, "old": 0, "H": 16, "G": 16, "D": 64, "page": 32,
         "bits": 16, "rot": 64, "interleaved": False},
        # a few sequences of odd length read back
        {"name": "read_odd", "kind": "read", "S": 5, "idle": 1, "new": 333, "old": 0, "G": 12, "D": 64, "page": 16, "bits": 16,
         "out": "bf16"},
        # long sequences of a cache of 8 bits read back
        {"name": "read_long", "kind": "read", "S": 8, "idle": 0, "new": 8192, "old": 0, "G": 8, "D": 128, "page": 64, "bits": 8,
         "out": "bf16"},
        # one token of one short sequence: latency
        {"name": "attention_token", "kind": "attention", "S": 1, "idle": 0, "new": 1, "old": 776, "H": 16, "G": 16, "D": 64,
         "page": 16, "bits": 16, "window": 0},
        # one token of one long sequence
        {"name": "attention_long", "kind": "attention", "S": 1, "idle": 0, "new": 1, "old": 131000, "H": 32, "G": 8, "D": 128,
         "page": 16, "bits": 16, "window": 0},
        # serving: a token of each of 64 sequences of uneven length, 8 bits
        {"name": "attention_tokens", "kind": "attention", "S": 64, "idle": 3, "new": 1, "old": 8191, "H": 32, "G": 8, "D": 128,
         "page": 32, "bits": 8, "window": 0},
        # chunks of several prompts beside what they have in the cache, a window over it
        {"name": "attention_chunks", "kind": "attention", "S": 7, "idle": 1, "new": 77, "old": 4001, "H": 12, "G": 4, "D": 64,
         "page": 16, "bits": 8, "window": 1000},
        # the prompts of a ragged batch
        {"name": "attention_batch", "kind": "attention", "S": 32, "idle": 0, "new": 512, "old": 0, "H": 16, "G": 16, "D": 64,
         "page": 32, "bits": 16, "window": 0},
        # a chunk of a long prompt
        {"name": "attention_prompt", "kind": "attention", "S": 1, "idle": 0, "new": 2048, "old": 14336, "H": 32, "G": 8, "D": 128,
         "page": 64, "bits": 16, "window": 0},
    ]


MOST_PAIRS = 32 * 2048 * 15360          # (query head, query, key) of the largest listed attention
MOST_CACHE = 64 * 4200 * 8 * 128        # elements of keys in the largest listed cache, by its mean length
MOST_MOVED = 8 * 4608 * 8 * 128         # elements of keys that the largest listed call writes or reads back


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _heads(rng):
    G = rng.choice((1, 2, 4, 8, 12, 16))
    return G * rng.choice([m for m in (1, 2, 3, 4, 8) if G * m <= 48]), G


def draw(rng):
    kind = rng.choice(("rotary", "write", "read", "attention", "attention"))
    D = rng.choice((64, 128))
    rot = rng.choice((D, D, D // 2, D // 4))
    inter = rng.random() < 0.4
    H, G = _heads(rng)
    if kind == "rotary":
        return {"kind": kind, "T": _log(rng, 1, 8177 * 32 * 128 // (H * D)), "H": H, "D": D, "rot": rot, "interleaved": inter,
                "far": _log(rng, 1, 130000)}
    page, bits = rng.choice((16, 32, 64, 128)), rng.choice((8, 16))
    idle = rng.choice((0, 0, 1, 3))
    if kind in ("write", "read"):
        S = _log(rng, 1, 64)
        new = _log(rng, 1, max(1, min(8192, MOST_MOVED // (G * D * S))))
        if kind == "read":
            return {"kind": kind, "S": S, "idle": idle, "new": new, "old": 0, "G": G, "D": D, "page": page, "bits": bits,
                    "out": rng.choice(("bf16", "f32"))}
        new = max(1, min(new, MOST_MOVED // ((H + 2 * G) * D * S)))
        return {"kind": kind, "S": S, "idle": idle, "new": new, "old": rng.choice((0, rng.randint(1, 100))), "H": H, "G": G, "D": D,
                "page": page, "bits": bits, "rot": rng.choice((rot, rot, 0)), "interleaved": inter}
    S = _log(rng, 1, 64)
    new = 1 if rng.random() < 0.5 else _log(rng, 2, 2048)
    most = min(131072, MOST_PAIRS // (H * S * new), MOST_CACHE // (G * D * S))
    new = max(1, min(new, most))
    total = _log(rng, new, max(new, most))
    return {"kind": kind, "S": S, "idle": idle, "new": new, "old": total - new, "H": H, "G": G, "D": D, "page": page, "bits": bits,
            "window": rng.choice((0, 0, _log(rng, 1, 4096)))}


# ---------------------------------------------------------------------------------------------- inputs
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0, std, generator=g)


def _sequences(case):
    """(tokens before, new tokens) of each sequence: uneven, from a few to the largest, and `idle` places without any."""
    S = case["S"]
    return [(round(case["old"] * (i + 1) / S), max(1, round(case["new"] * (S - i) / S))) for i in range(S)] + [(0, 0)] * case["idle"]


def _table(far, rot):
    """cos and sin of the angles of each position and pair, [positions, rot / 2, 2]: frequencies stretched for contexts eight times
    the trained ones, the slow ones in full, the fast ones not at all."""
    f = 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    turns = 4096.0 * f / (2 * math.pi)
    keep = ((turns - 1.0) / 31.0).clamp(0, 1)
    f = f * keep + f / 8.0 * (1 - keep)
    angle = torch.arange(far, dtype=torch.float64, device="cuda")[:, None] * f
    return (torch.stack((torch.cos(angle), torch.sin(angle)), 2) * 1.2).float()


def prepare(case, seed):
    g = _generator(seed)
    state = {"case": case}
    if case["kind"] == "rotary":
        T, H, D = case["T"], case["H"], case["D"]
        rows = _normal(g, (T, H + 2, D)).to(torch.bfloat16)
        state["x"] = rows[:, :H]                                             # (a layer's queries, in front of its keys and values)
        start = torch.randint(0, case["far"], (1,), device="cuda", generator=g)
        state["positions"] = (start + torch.arange(T, device="cuda")) % case["far"]
        state["table"] = _table(case["far"], case["rot"])
        return state
    G, D, page = case["G"], case["D"], case["page"]
    S = case["S"] + case["idle"]
    sizes = torch.tensor(_sequences(case), device="cuda")[torch.randperm(S, device="cuda", generator=g)]
    old, new = sizes[:, 0], sizes[:, 1]
    lengths = old + new
    state["offsets"] = torch.cat([new.new_zeros(1), torch.cumsum(new, 0)])
    state["lengths"] = lengths
    W = (case["old"] + case["new"] + page - 1) // page + 1
    used = (lengths + page - 1) // page
    live = torch.arange(W, device="cuda") < used[:, None]
    count = int(used.sum())
    order = torch.randperm(count + 2, device="cuda", generator=g)[:count]    # (pages in no order, and two that nobody has)
    pages = torch.full((S, W), -1, device="cuda", dtype=torch.int32)
    pages[live] = order.to(torch.int32)
    state["pages"] = pages
    T = int(state["offsets"][-1])
    state["rows"] = T
    shape = (count + 2, G, page, D)
    if case["bits"] == 16:
        state["k"], state["v"] = (torch.cat([_normal(g, (n,) + shape[1:]).to(torch.bfloat16) for n in _parts(shape[0])]) for _ in "kv")
        state["k_scale"] = state["v_scale"] = None
    else:
        state["k"], state["v"] = (torch.randint(-127, 128, shape, device="cuda", dtype=torch.int8, generator=g) for _ in "kv")
        state["k_scale"], state["v_scale"] = (torch.empty(shape[:3], device="cuda").uniform_(0.008, 0.024, generator=g) for _ in "kv")
    if case["kind"] == "write":
        H = case["H"]
        rows = _normal(g, (T, H + 2 * G, D)).to(torch.bfloat16)              # a layer's queries, keys and values in one row
        state["new_q"], state["new_k"], state["new_v"] = rows[:, :H], rows[:, H:H + G], rows[:, H + G:]
        state["table"] = _table(case["old"] + case["new"], case["rot"]) if case["rot"] else None
    if case["kind"] == "attention":
        state["q"] = _normal(g, (T, case["H"], D)).to(torch.bfloat16)
    state["longest"], state["most_new"] = int(lengths.max()), int(new.max())
    return state


def _parts(n, step=1024):
    return [min(step, n - i) for i in range(0, n, step)]


# ---------------------------------------------------------------------------------------------- one pass
def _rotated(x, rows, interleaved):
    """The first 2 P elements of each head of x [T, H, D] turned by the rows' angles [T, P, 2]."""
    P = rows.shape[1]
    c, s = rows[:, None, :, 0], rows[:, None, :, 1]
    a, b = (x[..., 0:2 * P:2], x[..., 1:2 * P:2]) if interleaved else (x[..., :P], x[..., P:2 * P])
    a, b = a * c - b * s, b * c + a * s
    front = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((front, x[..., 2 * P:]), -1)


def _rotary(state):
    case = state["case"]
    return _rotated(state["x"].float(), state["table"][state["positions"]], case["interleaved"]).to(torch.bfloat16)


def _places(state):
    """Of each row: its sequence, its position, and where in the cache it lies."""
    offsets, pages = state["offsets"], state["pages"]
    row = torch.arange(state["rows"], device=offsets.device)
    s = torch.searchsorted(offsets[1:], row, right=True)
    position = state["lengths"][s] - offsets[1:][s] + row
    page = state["case"]["page"]
    return position, pages[s, position // page].long(), position % page


def _held(x):
    """Rows as 8-bit codes and a scale each: (codes, scales)."""
    top = x.abs().amax(-1, keepdim=True)
    return torch.where(top > 0, torch.round(127 * x / top), 0.0).to(torch.int8), (top.float() / 127)[..., 0]


def _write(state):
    case = state["case"]
    position, page, slot = _places(state)
    q, k, v = state["new_q"].double(), state["new_k"].double(), state["new_v"].double()   # (64 bits: values at the border of two codes)
    if case["rot"]:
        rows = state["table"][position].double()
        q, k = _rotated(q, rows, case["interleaved"]), _rotated(k, rows, case["interleaved"])
    q = q.to(torch.bfloat16)
    if case["bits"] == 16:
        state["k"][page, :, slot] = k.to(torch.bfloat16)
        state["v"][page, :, slot] = v.to(torch.bfloat16)
        return q, state["k"], state["v"]
    for name, x in (("k", k), ("v", v)):
        codes, scales = _held(x)
        state[name][page, :, slot] = codes
        state[name + "_scale"][page, :, slot] = scales
    return q, state["k"] * state["k_scale"][..., None], state["v"] * state["v_scale"][..., None]


def _read(state):
    _, page, slot = _places(state)
    out = []
    for name in "kv":
        x = state[name][page, :, slot].float()
        if state["case"]["bits"] == 8:
            x = x * state[name + "_scale"][page, :, slot][..., None]
        out.append(x.to(_DTYPES[state["case"]["out"]]))
    return tuple(out)


def _attention(state):
    """Every sequence padded to the longest, its queries to the most that one has."""
    case, q = state["case"], state["q"]
    G, D, page = case["G"], case["D"], case["page"]
    offsets, lengths, pages = state["offsets"], state["lengths"], state["pages"]
    S, N, L, g = lengths.shape[0], state["most_new"], state["longest"], case["H"] // case["G"]
    j = torch.arange(L, device=q.device)
    at = pages[:, j // page].clamp(min=0).long(), j % page
    k, v = state["k"][at[0], :, at[1]].float(), state["v"][at[0], :, at[1]].float()        # [S, L, G, D]
    if case["bits"] == 8:
        k = k * state["k_scale"][at[0], :, at[1]][..., None]
        v = v * state["v_scale"][at[0], :, at[1]][..., None]
    new = offsets[1:] - offsets[:-1]
    i = torch.arange(N, device=q.device)
    there = i < new[:, None]                                                               # [S, N]
    row = (offsets[:-1, None] + i).clamp(max=q.shape[0] - 1)
    position = (lengths - new)[:, None] + i
    seen = j <= position[..., None]
    if case["window"]:
        seen = seen & (j > position[..., None] - case["window"])
    x = q[row].float().view(S, N, G, g, D).permute(0, 2, 3, 1, 4).reshape(S * G, g * N, D)
    scores = torch.bmm(x, k.permute(0, 2, 3, 1).reshape(S * G, D, L)).view(S, G, g, N, L) * D ** -0.5
    del k
    scores.masked_fill_(~(seen & there[..., None])[:, None, None], -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True).clamp(min=-3e38))
    del scores
    total = p.sum(-1, keepdim=True)
    v = torch.where((j < lengths[:, None])[..., None, None], v, 0.0)
    o = torch.bmm(p.view(S * G, g * N, L), v.permute(0, 2, 1, 3).reshape(S * G, L, D)).view(S, G, g, N, D)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(S, N, case["H"], D)
    return o[there].to(torch.bfloat16)


def _own(state):
    import paper_2006_03031_amd as nb
    from paper_2006_03031_amd import runtime as rt
    case = state["case"]
    if case["kind"] == "rotary":
        return rt.rotary(state["x"], state["positions"], state["table"], interleaved=case["interleaved"])
    if "handle" not in state:   # (a program keeps it beside the tensors)
        state["handle"] = (rt.PagedCache(state["k"], state["v"], state["k_scale"], state["v_scale"]),
                           rt.Sequences(state["offsets"], state["lengths"], state["pages"]))
    cache, sequences = state["handle"]
    if case["kind"] == "write":
        q = rt.cache_write(cache, state["new_k"], state["new_v"], sequences, q=state["new_q"], table=state["table"],
                           interleaved=case["interleaved"])
        if case["bits"] == 16:
            return q, state["k"], state["v"]
        return q, state["k"] * state["k_scale"][..., None], state["v"] * state["v_scale"][..., None]
    if case["kind"] == "read":
        return rt.cache_read(cache, sequences, state["rows"], {"bf16": nb.BF16, "f32": nb.F32}[case["out"]])
    return rt.paged_attention(state["q"], cache, sequences, window=case["window"])


def run(state):
    if own:
        return _own(state)
    return {"rotary": _rotary, "write": _write, "read": _read, "attention": _attention}[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------------------------- work and the exact results
def work(case):
    D = case["D"]
    if case["kind"] == "rotary":
        T, H = case["T"], case["H"]
        return {"bytes": 4 * T * H * D + T * (8 + 4 * case["rot"]), "flops": 3 * T * H * case["rot"]}
    sizes = _sequences(case)
    G = case["G"]
    new = sum(n for _, n in sizes)
    held = 2 * D if case["bits"] == 16 else D + 4                 # bytes of a key or a value of one head
    entries = sum((o + n + case["page"] - 1) // case["page"] for o, n in sizes)
    batch = 8 * (2 * len(sizes) + 1)
    if case["kind"] == "write":
        H = case["H"]
        moved = new * (2 * D * (2 * H + 2 * G) + 2 * G * held + 4 * case["rot"]) + batch + 4 * new
        return {"bytes": moved, "flops": new * (3 * (H + G) * case["rot"] + (4 * G * D * 2 if case["bits"] == 8 else 0))}
    if case["kind"] == "read":
        out = 2 if case["out"] == "bf16" else 4
        return {"bytes": new * 2 * G * (held + D * out) + batch + 4 * entries, "flops": new * 2 * G * D if case["bits"] == 8 else 0}
    H, w = case["H"], case["window"]
    pairs = read = 0
    for o, n in sizes:
        first = max(0, o + 1 - w) if w else 0
        read += o + n - first if n else 0
        pairs += sum(min(p + 1, w) if w else p + 1 for p in range(o, o + n))
    return {"bytes": 4 * new * H * D + 2 * read * G * held + batch + 4 * entries, "flops": 4 * D * H * pairs}


def exact(case, seed):
    state = prepare(case, seed)
    f64 = torch.float64

    def turned(x, position):      # element by element of the rotation's definition
        P = case["rot"] // 2
        y = x.clone()
        t = state["table"][position].to(f64)
        for i in range(P):
            a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + P)
            c, s = t[:, i, 0].unsqueeze(1), t[:, i, 1].unsqueeze(1)
            y[:, :, a] = c * x[:, :, a] - s * x[:, :, b]
            y[:, :, b] = s * x[:, :, a] + c * x[:, :, b]
        return y

    if case["kind"] == "rotary":
        return turned(state["x"].to(f64), state["positions"])
    ends, lengths = state["offsets"].tolist(), state["lengths"].tolist()
    page = case["page"]

    def slots(s, first, last):    # of positions first .. last - 1 of sequence s
        p = torch.arange(first, last, device=state["pages"].device)
        return state["pages"][s].long()[torch.div(p, page, rounding_mode="floor")], torch.remainder(p, page)

    def stored(name, s, first, last):
        a, b = slots(s, first, last)
        x = state[name][a, :, b].to(f64)
        return x if case["bits"] == 16 else x * state[name + "_scale"][a, :, b].to(f64).unsqueeze(2)

    spans = [(s, lengths[s] - (ends[s + 1] - ends[s]), lengths[s]) for s in range(len(lengths)) if ends[s + 1] > ends[s]]
    if case["kind"] == "read":
        return tuple(torch.cat([stored(name, *span) for span in spans]) for name in "kv")
    if case["kind"] == "write":
        position = torch.cat([torch.arange(a, b, device="cuda") for _, a, b in spans])
        q, k, v = (state[n].to(f64) for n in ("new_q", "new_k", "new_v"))
        if case["rot"]:
            q, k = turned(q, position), turned(k, position)
        page_of, slot_of = (torch.cat(x) for x in zip(*[slots(*span) for span in spans]))
        out = [q]
        for name, x in (("k", k), ("v", v)):
            whole = state[name].to(f64)
            if case["bits"] == 8:
                whole = whole * state[name + "_scale"].to(f64).unsqueeze(3)
                top = torch.max(torch.abs(x), dim=2, keepdim=True).values
                t = 127.0 * x / torch.where(top == 0, torch.ones_like(top), top)
                low = torch.floor(t)
                up = (t - low > 0.5) | ((t - low == 0.5) & (torch.remainder(low, 2) == 1))
                x = (low + up.to(f64)) * top / 127.0
            whole[page_of, :, slot_of] = x
            out.append(whole)
        return tuple(out)
    H, D, g = case["H"], case["D"], case["H"] // case["G"]
    out = torch.zeros((state["rows"], H, D), dtype=f64, device="cuda")
    for s, first, last in spans:
        low = max(0, first + 1 - case["window"]) if case["window"] else 0
        k, v = stored("k", s, low, last), stored("v", s, low, last)
        p = torch.arange(first, last, device="cuda").unsqueeze(1)
        key = torch.arange(low, last, device="cuda").unsqueeze(0)
        hidden = key > p
        if case["window"]:
            hidden |= p - key >= case["window"]
        for h in range(H):
            x = state["q"][ends[s]:ends[s + 1], h].to(f64) / math.sqrt(D)
            w = torch.matmul(x, k[:, h // g].t().contiguous())
            w[hidden] = -math.inf
            out[ends[s]:ends[s + 1], h] = torch.matmul(torch.softmax(w, 1), v[:, h // g].contiguous())
    return out
