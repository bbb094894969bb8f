"""Gated feed-forward blocks and their backward pass, against numpy in 64 bits.

Tolerances follow the arithmetic, entry by entry.  A product's sum of K terms is off by (2 K 2^-23 + e) S, S the sum of its
terms' magnitudes, e = 2^-20 for fp32's six part products and 0 for bf16's exact ones, and by what its operands are off
by.  The activations' largest slopes are below 1.13, their slopes' own below 0.8 (ReLU's jumps at 0); each is evaluated
within 2^-20 (|a| + 1): exp takes an argument off by 2^-24 |a|, and a^2 g (1 - g) < 0.5.  h, da and db are
rounded to bf16 (fp32's parts are within e), outputs to their type.  Second-order terms: 2^-6 of it all.
"""
import math

import numpy as np
import pytest

from test_gpu_embedding import HALF_STEP, f64, matrix, torch_type, unit_end, wide
from test_gpu_parity import G, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu

U = 2.0 ** -23


def activation(a, act):
    if act == "silu":
        g = 1.0 / (1.0 + np.exp(-a))
        return a * g, g + a * g * (1.0 - g)
    if act == "gelu":
        g = 0.5 * (1.0 + np.vectorize(math.erf)(a / math.sqrt(2.0)))
        return a * g, g + a * np.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
    return np.where(a > 0, a, 0.0), (a > 0).astype(np.float64)


def product(x, ex, w, ew, e):
    """x w and what it is off by, for operands off by ex and ew."""
    k = x.shape[1]
    s = np.abs(x) @ np.abs(w)
    off = (2 * k * U + e) * s
    if ex is not None:
        off = off + ex @ np.abs(w)
    if ew is not None:
        off = off + np.abs(x) @ ew
    return x @ w, off


def reference(x, wg, wu, wd, dy, act, dtype, sides=False):
    """{name: (value, tolerance)} of y, dx, dwg, dwu, dwd; `sides`: ReLU's slope is right however near a is to 0."""
    e = 2.0 ** -20 if dtype == "f32" else 0.0
    mid = HALF_STEP["bf16"] if dtype == "bf16" else 0.0
    a, ea = product(x, None, wg, None, e)
    b, eb = product(x, None, wu, None, e)
    v, s = activation(a, act)
    near = 2.0 ** -20 * (np.abs(a) + 1)
    ev = 1.13 * ea + near
    es = 0.8 * ea + near if act != "relu" else (np.abs(a) <= (0.0 if sides else ea)) * 1.0
    h = v * b
    eh = np.abs(v) * eb + np.abs(b) * ev + (mid + U) * np.abs(h)
    out = {}

    def done(name, got):
        value, off = got
        out[name] = (value, off * (1 + 2.0 ** -6) + (HALF_STEP[dtype] + U) * np.abs(value) + 1e-37)
    done("y", product(h, eh, wd, None, e))
    if dy is not None:
        dh, edh = product(dy, None, wd.T, None, e)
        da, db = dh * b * s, dh * v
        eda = edh * np.abs(b * s) + np.abs(dh * s) * eb + np.abs(dh * b) * es + (mid + 2 * U) * np.abs(da)
        edb = edh * np.abs(v) + np.abs(dh) * ev + (mid + 2 * U) * np.abs(db)
        done("dx", product(np.hstack([da, db]), np.hstack([eda, edb]), np.hstack([wg, wu]).T, None, e))
        done("dwg", product(x.T, None, da, eda, e))
        done("dwu", product(x.T, None, db, edb, e))
        done("dwd", product(h.T, eh.T, dy, None, e))
    return out


def empty(rows, cols, dtype):
    import torch
    return torch.full((rows + 1, unit_end(cols, dtype) + unit_end(1, dtype)), -7.0, dtype=torch_type(dtype), device="cuda")[:, :cols]


def block(m, d, f, o, dtype, seed, extra=1):
    x, dy = matrix(m, d, dtype, seed, extra), matrix(m, o, dtype, seed + 1, extra)
    wg, wu, wd = (matrix(r, c, dtype, seed + 2 + i, extra * i) for i, (r, c) in enumerate(((d, f), (d, f), (f, o))))
    for w, k in ((wg, d), (wu, d), (wd, f)):
        w.mul_(1.0 / math.sqrt(k))
    return x, wg, wu, wd, dy


def saved_for(G, m, f, dtype):
    import torch
    return torch.full((G.gated_ffn_saved(m, f, dtype),), 0xFF, dtype=torch.uint8, device="cuda")


def check(G, x, wg, wu, wd, dy, act, dtype, grads=("dx", "dwg", "dwu", "dwd"), sides=False):
    """Runs both passes and compares every output."""
    m, d = x.shape
    f, o = wd.shape
    got = dict(y=empty(m, o, dtype))
    alone = empty(m, o, dtype)
    G.gated_ffn(x, wg, wu, wd, alone, act=act)
    saved = saved_for(G, m, f, dtype) if grads else None
    if grads:
        G.gated_ffn(x, wg, wu, wd, got["y"], act=act, saved=saved)
        shapes = dict(dx=(m, d), dwg=(d, f), dwu=(d, f), dwd=(f, o))
        got.update({n: empty(*shapes[n], dtype) for n in grads})
        G.gated_ffn_backward(x, wg, wu, wd, dy, saved, act=act, **{n: got[n] for n in grads})
    else:
        got["y"].copy_(alone)
        wide(got["y"]).copy_(wide(alone))
    G.sync()
    want = reference(f64(x), f64(wg), f64(wu), f64(wd), f64(dy) if grads else None, act, dtype, sides)
    got["alone"], want["alone"] = alone, want["y"]
    for n, t in got.items():
        value, tol = want[n]
        r, c = value.shape
        worst = (np.abs(f64(t)[:r] - value) / tol).max() if r else 0.0
        assert worst <= 1.0, (n, worst)
        b = wide(t).float().cpu()
        end = unit_end(c, dtype)
        assert (b[:r, c:end] == 0).all() and (b[:, end:] == -7).all() and (b[r:] == -7).all(), n
    return got


SHAPES = [(1, 1, 1, 1), (1, 8, 16, 8), (2, 5, 3, 7), (3, 40, 72, 41), (7, 64, 130, 16), (17, 100, 33, 9), (33, 31, 96, 64),
          (64, 128, 128, 128), (65, 72, 200, 5), (130, 602, 257, 41), (200, 33, 64, 300), (257, 16, 520, 129), (1000, 24, 40, 8),
          (1, 1100, 2300, 70), (4, 2050, 1025, 33), (5, 64, 96, 24), (8, 40, 1030, 9), (9, 1024, 70, 16)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,d,f,o", SHAPES)
def test_both_passes(G, m, d, f, o, dtype):
    act = ("silu", "gelu", "relu")[(m + f) % 3]
    say("gated", m, d, f, o, dtype, act)
    check(G, *block(m, d, f, o, dtype, m + d + f), act, dtype)


@pytest.mark.parametrize("m,d,f,o", [(40, 64, 700, 24), (300, 333, 1000, 41), (3000, 130, 520, 70)])
def test_relu_is_on_the_right_side_of_zero(G, m, d, f, o):
    """Every hidden column has a row whose a nearly cancels, to less than what a sum in fp32 is off by; none is 0."""
    import torch
    x, wg, wu, wd, dy = block(m, d, f, o, "f32", 60)
    at = np.arange(f) * 7 % m
    x[:, d - 1] = 1.0 + x[:, d - 1].abs()
    full = f64(x)
    rest = np.einsum("cd,dc->c", full[at, :-1], f64(wg)[:-1])
    wg[d - 1] = torch.from_numpy(-rest / full[at, -1]).to(wg)
    a = np.einsum("cd,dc->c", full[at], f64(wg))
    assert (a != 0).all() and (np.abs(a) < 2.0 ** -22 * np.abs(full[at]).max()).all()
    say("gated relu sides", m, d, f, o)
    check(G, x, wg, wu, wd, dy, "relu", "f32", sides=True)


@pytest.mark.parametrize("m", [5, 70, 500])
def test_relu_with_columns_and_rows_that_are_nearly_dead(G, m):
    """Hidden columns of zeros, and columns and rows 2^-40 of the others: their signs are those of their own sizes."""
    x, wg, wu, wd, dy = block(m, 130, 300, 40, "f32", 70)
    wg[:, 3::7] = 0
    wg[:, 5::7] *= 2.0 ** -40
    x[1::9] *= 2.0 ** -40
    x[2::9] = 0
    say("gated relu dead", m)
    check(G, x, wg, wu, wd, dy, "relu", "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_activations(G, act, dtype):
    """From values whose activation vanishes to ones that it leaves as they are, on the tiles and on few rows."""
    for m in (3, 90):
        say("gated act", act, dtype, m)
        x, wg, wu, wd, dy = block(m, 24, 64, 32, dtype, 5)
        wg[:, :16].mul_(30.0)
        wg[:, 16:32].mul_(1e-3)
        check(G, x, wg, wu, wd, dy, act, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,d,f,o", [(2500, 128, 512, 72), (4000, 264, 392, 250), (900, 700, 1100, 520)])
def test_large_tiles(G, m, d, f, o, dtype):
    """Enough rows and columns for the larger tiles and for sums that are cut; ragged ones among them."""
    say("gated large", m, d, f, o, dtype)
    check(G, *block(m, d, f, o, dtype, 11), "silu", dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_of_the_weights(G, dtype):
    """Every matrix has a stride of its own, Wg and Wu too; rows and outputs in views of wider buffers."""
    say("gated strides", dtype)
    for m in (2, 70, 600):
        x, wg, wu, wd, dy = block(m, 72, 136, 40, dtype, 3, extra=2)
        assert wg.stride(0) != wu.stride(0) != wd.stride(0)
        check(G, x, wg, wu, wd, dy, "silu", dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("grads", [("dx",), ("dwg",), ("dwu",), ("dwd",), ("dwg", "dwu", "dwd"), ("dx", "dwd")], ids="+".join)
def test_what_is_asked_for(G, grads, dtype):
    say("gated outputs", grads, dtype)
    check(G, *block(70, 44, 100, 24, dtype, 3), "silu", dtype, grads=grads)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows(G, dtype):
    """m = 0: the forward pass does nothing, the weights' gradients are zero."""
    import torch
    say("gated no rows", dtype)
    x, wg, wu, wd, dy = block(4, 40, 72, 17, dtype, 3)
    saved = torch.zeros(0, dtype=torch.uint8, device="cuda")
    y = empty(2, 17, dtype)
    G.gated_ffn(x[:0], wg, wu, wd, y, saved=saved)
    dwg, dwu, dwd = empty(40, 72, dtype), empty(40, 72, dtype), empty(72, 17, dtype)
    G.gated_ffn_backward(x[:0], wg, wu, wd, dy[:0], saved, dwg=dwg, dwu=dwu, dwd=dwd)
    G.sync()
    assert (wide(y) == -7).all()
    for t, r in ((dwg, 40), (dwu, 40), (dwd, 72)):
        assert (t[:r] == 0).all() and (wide(t)[r:] == -7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m", [4, 150])
def test_rows_do_not_meet(G, m, dtype):
    """A row of NaN or infinities shows in its own answers and in the weights' gradients alone."""
    import torch
    say("gated nan rows", dtype, m)
    x, wg, wu, wd, dy = block(m, 40, 100, 24, dtype, 3)

    def run(x, dy):
        y, dx, saved = empty(m, 24, dtype), empty(m, 40, dtype), saved_for(G, m, 100, dtype)
        G.gated_ffn(x, wg, wu, wd, y, saved=saved)
        G.gated_ffn_backward(x, wg, wu, wd, dy, saved, dx=dx)
        return y[:m].clone(), dx[:m].clone()
    clean = run(x, dy)
    others = [i for i in range(m) if i != 1]
    for value in (float("nan"), float("inf")):
        xx, dd = x.clone(), dy.clone()
        xx[1], dd[1] = value, value
        for got in (run(xx, dy), run(x, dd)):
            for a, b in zip(got, clean):
                assert torch.equal(a[others], b[others])
        y, dx = run(xx, dd)
        assert torch.isnan(y[1]).any() and torch.isnan(dx[1]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_against_differences(G, dtype):
    """The loss sum(y * dy) of fp32, along single entries; steps of 2^-6 leave a curvature of 2^-12 of the entry's own, which the
    tolerance is far above, and rounding 2^-20 / 2^-6 of the terms; bf16's gradients are compared with fp32's differences."""
    import torch
    say("gated differences", dtype)
    m, d, f, o = 5, 12, 20, 6
    x, wg, wu, wd, dy = block(m, d, f, o, dtype, 9, extra=0)
    saved = saved_for(G, m, f, dtype)
    y = empty(m, o, dtype)
    grads = dict(dx=empty(m, d, dtype), dwg=empty(d, f, dtype), dwu=empty(d, f, dtype), dwd=empty(f, o, dtype))
    G.gated_ffn(x, wg, wu, wd, y, saved=saved)
    G.gated_ffn_backward(x, wg, wu, wd, dy, saved, **grads)
    t = {n: v.float().contiguous() for n, v in dict(x=x, wg=wg, wu=wu, wd=wd).items()}
    per = {n: torch.zeros((v.shape[0], unit_end(v.shape[1], "f32")), device="cuda") for n, v in t.items()}
    t32 = {n: per[n][:, :v.shape[1]] for n, v in t.items()}
    for n, v in t.items():
        t32[n].copy_(v)
    yy = torch.zeros((m, unit_end(o, "f32")), device="cuda")[:, :o]
    for name, at in (("x", (0, 0)), ("x", (4, 11)), ("wg", (3, 7)), ("wg", (11, 19)), ("wu", (0, 1)), ("wu", (11, 0)), ("wd", (19, 5)), ("wd", (2, 0))):
        old, value = t32[name][at].item(), []
        for step in (2.0 ** -6, -2.0 ** -6):
            t32[name][at] = old + step
            G.gated_ffn(t32["x"], t32["wg"], t32["wu"], t32["wd"], yy)
            value.append((yy.double() * dy.double()).sum().item())
        t32[name][at] = old
        got = grads["d" + name][at].item()
        assert got == pytest.approx((value[0] - value[1]) / 2.0 ** -5, abs=2.0 ** -7 if dtype == "bf16" else 2.0 ** -9, rel=2.0 ** -6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,d,f,o", [(3, 48, 96, 24), (50, 44, 100, 41), (700, 130, 300, 72)])
def test_workspace_and_saved_are_guarded(G, m, d, f, o, dtype):
    """Sizes of exactly what is asked for, garbage in them, canaries behind; the same bits from a workspace of torch's, and again."""
    import torch
    say("gated workspace", m, d, f, o, dtype)
    x, wg, wu, wd, dy = block(m, d, f, o, dtype, 3)
    need = [G.gated_ffn_workspace(m, d, f, o, dtype), G.gated_ffn_backward_workspace(m, d, f, o, dtype)]
    keep = G.gated_ffn_saved(m, f, dtype)
    res = []
    for fill in (0, 0xFF, None):
        ws = [torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda") for n in need]
        saved = torch.full((keep + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
        if fill is not None:
            for w, n in zip(ws, need):
                w[:n] = fill
            saved[:keep] = fill
        given = [w[:n] for w, n in zip(ws, need)] if fill is not None else [None, None]
        y, grads = empty(m, o, dtype), dict(dx=empty(m, d, dtype), dwg=empty(d, f, dtype), dwu=empty(d, f, dtype), dwd=empty(f, o, dtype))
        G.gated_ffn(x, wg, wu, wd, y, saved=saved[:keep], workspace=given[0])
        G.gated_ffn_backward(x, wg, wu, wd, dy, saved[:keep], workspace=given[1], **grads)
        assert all((w[n:] == 0x5A).all() for w, n in zip(ws + [saved], need + [keep]))
        res.append([y, *grads.values()])
        for w, n, call in ((need[0], 0, lambda b: G.gated_ffn(x, wg, wu, wd, y, workspace=b)),
                           (need[1], 1, lambda b: G.gated_ffn_backward(x, wg, wu, wd, dy, saved[:keep], workspace=b, **grads))):
            if w > 0:
                with pytest.raises(G.GnnavError):
                    call(ws[n][:w - 1])
        with pytest.raises(G.GnnavError):
            G.gated_ffn(x, wg, wu, wd, y, saved=saved[:keep - 1])
    for other in res[1:]:
        assert all(torch.equal(wide(a), wide(b)) for a, b in zip(res[0], other))


def test_argument_types(G):
    import torch
    x, wg, wu, wd, dy = block(4, 8, 16, 8, "f32", 1, extra=0)
    y, saved = torch.zeros((4, 8), device="cuda"), saved_for(G, 4, 16, "f32")
    for bad in (lambda: G.gated_ffn(x, wg.bfloat16(), wu, wd, y), lambda: G.gated_ffn(x, wg, wu[:, :8], wd, y),
                lambda: G.gated_ffn(x, wg[:4], wu, wd, y), lambda: G.gated_ffn(x, wg, wu, wd[:8], y),
                lambda: G.gated_ffn(x, wg, wu, wd, y[:3]), lambda: G.gated_ffn(x, wg, wu, wd, y[:, :4]),
                lambda: G.gated_ffn(x, wg, wu, wd, y, act="tanh"), lambda: G.gated_ffn(x, wg, wu, wd, y, saved=saved.float()),
                lambda: G.gated_ffn(x.half(), wg, wu, wd, y), lambda: G.gated_ffn(x, wg.t(), wu, wd, y),
                lambda: G.gated_ffn_backward(x, wg, wu, wd, dy[:2], saved), lambda: G.gated_ffn_backward(x, wg, wu, wd, dy, saved, dx=x[:2]),
                lambda: G.gated_ffn_backward(x, wg, wu, wd, dy, saved, dwd=wg)):
        with pytest.raises(ValueError):
            bad()
