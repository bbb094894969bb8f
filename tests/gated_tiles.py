"""Blocks that take every tile of the gated feed-forward kernels, and what their results may be off by, entry by entry and by norm.

TILES: type, m, d, f, d_out, activations, then the planner's choices: tile of h, tile of y and the splits of its sum, tile of da
and db, tile of the gradients and the splits of dx, of dWg and dWu, and of dWd (0 to 3: the largest to the smallest).

expected() works in torch's 64 bits, on any device.  The entries' tolerances are those that test_gpu_gated.py derives.  By norm,
errors of many entries add as squares, which tells fp32's three parts from two:

- a sum of K terms, in steps of 16 of q products each (6 in fp32, 1 in bf16), rounds its running sum, whose mean square grows to that
  of the whole, q K / 16 times by half a step 2^-24 at most: sqrt(q K / 32) 2^-24 of sqrt(sum x^2 w^2), which is what random terms sum
  to.  A sum in s splits has K / s terms in each, and s more roundings.
- fp32's parts leave out some 2^-26 of a product, less than these.
- an activation is off by 2^-21 (|a| + 1) at most, evenly: a third of its square; so are roundings to bf16, 2^-8, or fp32, 2^-24.
- an operand's error passes on by the slopes, its square by their squares.

A part of an operand that is lost is 2^-16 / sqrt(3) of 1.5 as a mean, and shows: test_gated_tiles.py plants it.
"""
import math

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}

TILES = [
    ("bf16", 24, 18, 19, 7, ("silu", "gelu", "relu"), (3, 2, 1, 3, 2, 1, 1, 1)),
    ("bf16", 2_583, 17, 1_547, 5, ("silu",), (2, 3, 3, 2, 2, 6, 5, 10)),
    ("bf16", 5_053, 17, 1_422, 6, ("gelu",), (0, 3, 1, 0, 3, 5, 9, 9)),
    ("bf16", 5_845, 19, 2_537, 5, ("relu",), (0, 2, 5, 0, 3, 1, 1, 1)),
    ("bf16", 44_027, 74, 141, 70, ("silu",), (2, 1, 1, 2, 1, 1, 63, 63)),
    ("bf16", 275, 23, 6_061, 969, ("gelu",), (3, 1, 11, 3, 0, 45, 1, 1)),
    ("bf16", 21, 414, 3_781, 417, ("relu",), (3, 3, 7, 3, 1, 14, 1, 1)),
    ("bf16", 11_751, 29, 205, 849, ("silu",), (3, 0, 1, 3, 0, 1, 46, 23)),
    ("bf16", 301, 28, 7_535, 1_613, ("gelu",), (3, 0, 14, 2, 2, 27, 1, 1)),
    ("bf16", 8_193, 602, 1_024, 41, ("silu", "gelu", "relu"), (2, 3, 1, 2, 0, 1, 5, 5)),
    ("bf16", 50_001, 256, 1_024, 256, ("silu", "gelu", "relu"), (0, 0, 1, 0, 0, 1, 26, 26)),
    ("bf16", 9_001, 130, 1_030, 200, ("relu",), (2, 2, 1, 2, 2, 1, 7, 7)),
    ("f32", 21, 23, 17, 11, ("silu", "gelu", "relu"), (3, 2, 1, 3, 2, 1, 1, 1)),
    ("f32", 7_625, 19, 941, 81, ("silu", "gelu", "relu"), (1, 3, 1, 1, 3, 7, 29, 29)),
    ("f32", 731, 21, 2_915, 6, ("relu",), (1, 2, 11, 3, 2, 22, 2, 2)),
    ("f32", 16_889, 95, 17, 563, ("gelu",), (3, 1, 1, 3, 1, 1, 63, 63)),
    ("f32", 25, 1_139, 2_059, 2_297, ("silu",), (3, 3, 8, 3, 1, 16, 1, 1)),
    ("f32", 2_401, 101, 1_241, 250, ("gelu",), (1, 1, 4, 3, 3, 1, 1, 1)),
    ("f32", 2_459, 21, 5_499, 105, ("silu", "gelu", "relu"), (1, 1, 21, 1, 2, 20, 5, 5)),
    ("f32", 30_001, 200, 700, 100, ("relu",), (1, 1, 1, 1, 1, 1, 31, 31)),
    ("f32", 8_193, 256, 1_024, 256, ("relu",), (1, 1, 1, 3, 2, 1, 10, 10)),
    ("f32", 4_097, 602, 1_024, 41, ("silu", "gelu", "relu"), (1, 2, 4, 3, 1, 3, 6, 6)),
]


def activation(a, act):
    """act(a) and its slope."""
    import torch
    if act == "silu":
        g = torch.sigmoid(a)
        return a * g, g + a * g * (1.0 - g)
    if act == "gelu":
        g = 0.5 * torch.erfc(-a / math.sqrt(2.0))
        return a * g, g + a * torch.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
    return torch.clamp(a, min=0.0), (a > 0).to(a.dtype)


class Value:
    """A matrix in 64 bits, what its entries are off by at the most, and the mean square of that."""

    def __init__(self, value, off=None, square=None):
        self.value, self.off, self.square = value, off, square


def product(x, w, dtype, splits=1):
    k = x.value.shape[1]
    q, e = (6, 2.0 ** -20) if dtype == "f32" else (1, 0.0)
    value, s = x.value @ w.value, x.value.abs() @ w.value.abs()
    xx, ww = x.value ** 2, w.value ** 2
    off = (2 * k * 2.0 ** -23 + e) * s
    square = (q * (k / splits) / 32 + (splits if splits > 1 else 0)) * 2.0 ** -48 * (xx @ ww)
    for a, b, sq in ((x, w, ww), (w, x, xx)):
        if a.off is not None:
            left = a is x
            off = off + (a.off @ b.value.abs() if left else b.value.abs() @ a.off)
            square = square + (a.square @ sq if left else sq @ a.square)
    return Value(value, off, square)


def rounded(v, dtype):
    """... and rounded to the type (fp32's parts hold all of it)."""
    step = HALF_STEP[dtype] + 2.0 ** -23
    v.off = v.off + step * v.value.abs()
    v.square = v.square + step ** 2 / 3 * v.value ** 2
    return v


def t(v):
    return Value(v.value.t(), None if v.off is None else v.off.t(), None if v.square is None else v.square.t())


def expected(x, wg, wu, wd, dy, act, dtype, splits=(1, 1, 1, 1), sides=False):
    """{name: Value} of y, dx, dwg, dwu and dwd; `sides`: ReLU's slope is right however near a is to 0."""
    import torch
    x, wg, wu, wd, dy = (Value(v.double()) for v in (x, wg, wu, wd, dy))
    a, b = product(x, wg, dtype), product(x, wu, dtype)
    value, slope = activation(a.value, act)
    near = 2.0 ** -21 * (a.value.abs() + 1)
    v = Value(value, 1.13 * a.off + 2 * near, (slope * slope).clamp(max=1.13 ** 2) * a.square + near ** 2 / 3)
    s = Value(slope, 0.8 * a.off + 2 * near, 0.64 * a.square + near ** 2 / 3)
    if act == "relu":
        jump = torch.zeros_like(slope, dtype=torch.bool) if sides else a.value.abs() <= a.off
        sure = torch.zeros_like(jump) if sides else a.value.abs() <= 4 * a.square.sqrt()
        s = Value(slope, jump.double(), sure.double())

    def times(p, r):
        return Value(p.value * r.value, p.off * r.value.abs() + p.value.abs() * r.off, p.square * r.value ** 2 + p.value ** 2 * r.square)
    h = rounded(times(v, b), dtype)
    dh = product(dy, t(wd), dtype)
    da, db = rounded(times(times(dh, b), s), dtype), rounded(times(dh, v), dtype)
    both = Value(torch.cat([da.value, db.value], 1), torch.cat([da.off, db.off], 1), torch.cat([da.square, db.square], 1))
    out = dict(y=product(h, wd, dtype, splits[0]), dx=product(both, t(Value(torch.cat([wg.value, wu.value], 1))), dtype, splits[1]),
               dwg=product(t(x), da, dtype, splits[2]), dwu=product(t(x), db, dtype, splits[2]), dwd=product(t(h), dy, dtype, splits[3]))
    for r in out.values():
        rounded(r, dtype)
        r.off = r.off * (1 + 2.0 ** -6) + 1e-37
    return out
