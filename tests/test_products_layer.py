"""A layer of experts in 8 bits, end to end, against the layer in float64 from the operands before they are quantised.

The error that the roundings make is predicted from the operands: a code is off by an even spread over its step (a 127th of its row's largest
value; a variance of step^2 / 12), the hidden rows by a spread of at most 2^-8 of the value for bf16, GELU passes at most 1.13 of an error on,
and errors of weights and rows that are drawn at random add up as their squares.  Over some 75000 results the root of the mean square
is known to a few per cent, and one and a half times the predicted one is allowed (it is 2.1 % of the results' own).
A layer of zeros, one with two experts swapped, with rows that are one off and with a scale that is 5 % off miss that: tested without a GPU."""
import math

import pytest

import paper_2006_03031_amd as nb

torch = pytest.importorskip("torch")

T, E, D, F = 150, 6, 256, 640


def _operands():
    g = torch.Generator().manual_seed(11)

    def normal(shape, std=1.0):
        return (torch.randn(shape, generator=g) * std).bfloat16()
    x, w1, w2 = normal((T, D)), normal((E, F, D), D ** -0.5), normal((E, D, F), F ** -0.5)
    b1, b2 = normal((E, F), 0.1), normal((E, D), 0.1)
    chosen = torch.stack([torch.randperm(E - 1, generator=g)[:2] for _ in range(T)])   # the last expert gets none
    order = torch.argsort(chosen.flatten(), stable=True)
    sizes = torch.bincount(chosen.flatten(), minlength=E)
    return x[order // 2].contiguous(), w1, w2, b1, b2, torch.cat([sizes.new_zeros(1), sizes.cumsum(0)])


def _quantised(x):
    """The values that the codes of the rows stand for, in float64."""
    top = x.double().abs().amax(-1, keepdim=True)
    return torch.round(127 * x.double() / top) * (top / 127)


def _gelu(v):
    return 0.5 * v * torch.special.erfc(-v * math.sqrt(0.5))


def _layer_and_limit(rows, w1, w2, b1, b2, offsets):
    y, square = torch.zeros((rows.shape[0], D), dtype=torch.float64), torch.zeros((rows.shape[0], D), dtype=torch.float64)
    cuts = offsets.tolist()

    def spread(v):      # variance of the codes' errors, a row's the same
        return (v.abs().amax(1, keepdim=True) / 127) ** 2 / 12
    for e in range(E):
        part = slice(cuts[e], cuts[e + 1])
        x, a, b = rows[part].double(), w1[e].double(), w2[e].double()
        if not x.shape[0]:
            continue
        h = _gelu(x @ a.t() + b1[e].double())
        of_h = 1.13 ** 2 * (spread(x) * (a ** 2).sum(1) + (x ** 2).sum(1, keepdim=True) * spread(a).t()) + (2.0 ** -8 * h) ** 2 / 3 + spread(h)
        y[part] = h @ b.t() + b2[e].double()
        square[part] = of_h @ (b ** 2).t() + (h ** 2).sum(1, keepdim=True) * spread(b).t()
    return y, 1.5 * square.mean().sqrt()


def _within(got, y, limit):
    return bool(((got.double() - y) ** 2).mean().sqrt() <= limit)


def test_what_the_limit_lets_through():
    rows, w1, w2, b1, b2, offsets = _operands()
    y, limit = _layer_and_limit(rows, w1, w2, b1, b2, offsets)
    cuts = offsets.tolist()

    def emulated(order, scale=1.0):
        out = torch.zeros_like(y)
        for e in range(E):
            part, o = slice(cuts[e], cuts[e + 1]), order[e]
            if cuts[e] < cuts[e + 1]:
                h = _gelu(_quantised(rows[part]) @ _quantised(w1[o]).t() + b1[o].double()).bfloat16()
                out[part] = scale * (_quantised(h) @ _quantised(w2[o]).t()) + b2[o].double()
        return out
    assert _within(emulated(range(E)), y, limit)
    assert not _within(torch.zeros_like(y), y, limit)
    assert not _within(emulated([1, 0, 2, 3, 4, 5]), y, limit)
    assert not _within(emulated(range(E), 0.95), y, limit)
    assert not _within(emulated(range(E)).roll(1, 0), y, limit)


@pytest.mark.gpu
def test_a_layer_of_experts_in_8_bits():
    from paper_2006_03031_amd import runtime as rt
    rows, w1, w2, b1, b2, offsets = _operands()
    y, limit = _layer_and_limit(rows, w1, w2, b1, b2, offsets)
    (w1q, s1), (w2q, s2) = rt.quantize_rows(w1.view(E * F, D).cuda()), rt.quantize_rows(w2.view(E * D, F).cuda())
    off = offsets.cuda()
    h = rt.grouped_dense_i8(*rt.quantize_rows(rows.cuda()), w1q.view(E, F, -1), s1.view(E, F), b1.cuda(), off, nb.EPI_BIAS_GELU_ERF)
    got = rt.grouped_dense_i8(*rt.quantize_rows(h), w2q.view(E, D, -1), s2.view(E, D), b2.cuda(), off, nb.EPI_BIAS, nb.F32)
    assert _within(got.cpu(), y, limit)
