"""A paged cache and its batches for the tests, and the operators' formulas in 64 bits on the CPU."""
import math

import torch

BF = torch.bfloat16


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


class Batch:
    """sizes: (tokens before, new rows) of each sequence; ahead, behind: rows of no sequence."""

    def __init__(self, sizes, page, seed=0, ahead=0, behind=0, spare_pages=2, extra_columns=1):
        g = torch.Generator().manual_seed(seed)
        self.sizes, self.page, self.ahead, self.behind = sizes, page, ahead, behind
        self.offsets = torch.tensor([ahead] + [ahead + sum(n for _, n in sizes[:i + 1]) for i in range(len(sizes))])
        self.lengths = torch.tensor([max(0, o + n) for o, n in sizes], dtype=torch.int64)
        used = [(int(l) + page - 1) // page for l in self.lengths]
        self.count = sum(used) + spare_pages
        order = torch.randperm(self.count, generator=g).tolist()
        self.pages = torch.full((len(sizes), max([0] + used) + extra_columns), -1, dtype=torch.int32)
        for s, n in enumerate(used):
            for i in range(n):
                self.pages[s, i] = order.pop()
        self.rows = int(self.offsets[-1]) + behind

    def slots(self, s, positions):
        """(page, slot) of positions of sequence s."""
        p = torch.as_tensor(positions)
        return self.pages[s].long()[p // self.page], p % self.page

    def each(self):
        """(sequence, row, position) of every row."""
        for s, (o, n) in enumerate(self.sizes):
            for i in range(n):
                yield s, int(self.offsets[s]) + i, int(self.lengths[s]) - n + i

    def on_gpu(self):
        from paper_2006_03031_amd import runtime as rt
        return rt.Sequences(self.offsets.cuda(), self.lengths.cuda(), self.pages.cuda())


def random_cache(batch, G, D, int8, seed=1):
    """(k, v, k_scale, v_scale) on the CPU."""
    g = torch.Generator().manual_seed(seed)
    shape = (batch.count, G, batch.page, D)
    if not int8:
        return tuple(torch.randn(shape, generator=g).to(BF) for _ in range(2)) + (None, None)
    codes = tuple(torch.randint(-127, 128, shape, generator=g).to(torch.int8) for _ in range(2))
    return codes + tuple(torch.rand(shape[:3], generator=g) * 0.02 + 0.005 for _ in range(2))


def to_gpu(cache):
    from paper_2006_03031_amd import runtime as rt
    return rt.PagedCache(*(None if t is None else t.cuda() for t in cache))


def values(cache, which):
    x, scale = cache[which].double(), cache[2 + which]
    return x if scale is None else x * scale.double()[..., None]


def attention(q, cache, batch, window=0, alpha=None, weight_step=None):
    """(o, bound): the formula in 64 bits, and how far the kernel may be off in each element: half a step of bf16 for the result, another,
    relative to sum_j w_j |v_j|, for the probabilities' rounding, and for the weights' own errors twice those of the scores, whose D products
    are added in f32, and 2^-18 for exp2, the running sums and the joins.  exp2 of less than -126, and a probability below 2^-126 once it is
    rounded to bf16, may be taken as 0, a weight of at most 2^-126 either time (the weights' sum is at least about 1): 2^-125 sum_j |v_j|.
    weight_step: what the probabilities' rounding may take instead; in two bf16 it is half a step of half a step, and what the second loses
    below 2^-126 at most 2^-125 too."""
    T, H, D = q.shape
    weight_step = half_step(BF) if weight_step is None else weight_step
    G = cache[0].shape[1]
    alpha = D ** -0.5 if alpha is None else alpha
    k_all, v_all = values(cache, 0), values(cache, 1)
    o = torch.zeros(T, H, D, dtype=torch.float64)
    bound = torch.zeros_like(o)
    for s, row, p in batch.each():
        low = max(0, p - window + 1) if window else 0
        if p < low:
            continue
        page, slot = batch.slots(s, torch.arange(low, p + 1))
        k, v = k_all[page, :, slot], v_all[page, :, slot]                                  # [L, G, D]
        for h in range(H):
            x = q[row, h].double()
            terms = k[:, h // (H // G)] * x
            w = torch.softmax(alpha * terms.sum(1), 0)
            vh = v[:, h // (H // G)]
            o[row, h] = w @ vh
            scores_off = (D + 4) * 2.0 ** -24 * alpha * float(terms.abs().sum(1).max())
            bound[row, h] = half_step(BF) * o[row, h].abs() + (weight_step + 2 * scores_off + 2.0 ** -18) * (w @ vh.abs()) + \
                2.0 ** -124 * vh.abs().sum(0)
    return o, bound


def angles(positions, rot, base=10000.0, factor=1.0, trained=0.0, low=1.0, high=32.0, magnitude=1.0):
    t = torch.zeros(positions, rot // 2, 2, dtype=torch.float64)
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        keep = min(1.0, max(0.0, (trained * f / (2 * math.pi) - low) / (high - low))) if trained else 0.0
        f = f * keep + f / factor * (1 - keep)
        a = torch.arange(positions, dtype=torch.float64) * f
        t[:, i, 0], t[:, i, 1] = magnitude * torch.cos(a), magnitude * torch.sin(a)
    return t


def turned(x, rows, interleaved):
    """(y, size): heads x [T, H, D] turned by rows [T, R, 2] in 64 bits, and the sum of the magnitudes that each element is made of."""
    x, rows = x.double(), rows.double()
    y, size = x.clone(), x.abs()
    R = rows.shape[1]
    for i in range(R):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R)
        c, s = rows[:, i, 0, None], rows[:, i, 1, None]
        y[:, :, a], y[:, :, b] = x[:, :, a] * c - x[:, :, b] * s, x[:, :, b] * c + x[:, :, a] * s
        size[:, :, a] = (x[:, :, a] * c).abs() + (x[:, :, b] * s).abs()
        size[:, :, b] = (x[:, :, b] * c).abs() + (x[:, :, a] * s).abs()
    return y, size


def quantized(x):
    """(codes, scales) of rows x [..., D] in 64 bits: exactly rounded codes, ties to even; scales in f32."""
    top = x.abs().amax(-1, keepdim=True)
    finite = torch.isfinite(x).all(-1, keepdim=True)
    codes = torch.where(finite & (top > 0), torch.round(127.0 * x / torch.where(top > 0, top, 1.0)), 0.0)
    scales = torch.where(finite, top.float() / 127, math.nan)[..., 0]
    return codes.to(torch.int8), scales
