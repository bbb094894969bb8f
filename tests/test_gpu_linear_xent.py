"""Softmax cross entropy over many classes without the logits, against numpy in 64 bits.

Tolerances follow the arithmetic.  With S_iv = sum_k |h_ik w_vk| a logit is off by
ez = (2 d 2^-23 + e) S, e = 2^-20 for fp32's six part products and 0 for bf16's
exact ones (2^-23: the matrix cores' sums may truncate).  exp takes an argument off by
2^-22 |z - lse|, and is off by 2^-22 itself; a sum of exponentials by its terms
and 2^-15 at most for 512 roundings in a row.  So log-sum-exp and the row's loss are off by
2 ez + 2^-15 (+ rounding of the value), and p by the relative rp = 2 ez + 2^-15 + 2^-22
(1 + |z - lse|).  bf16 rounds p - [v = y] once more by 2^-8 of it.  The gradients' products are
sums of K terms as the logits are; the result is rounded to the type.  exp of less than
2^-126, the smallest normal number, is zero: an error of p below 2^-126.  (At m = 5, 3,000 classes, d = 602
5,036 of 9,000 p lie below it, and setting just those to zero in the 64-bit reference moves
dw by 1.12009 of a tolerance without that term, digit for digit what the kernel's dw is off by.)
"""
import numpy as np
import pytest

from test_gpu_embedding import HALF_STEP, f64, matrix, torch_type, unit_end, wide
from test_gpu_parity import G, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu


def reference(h, w, y, ignore, dtype):
    """(loss, row losses, dh, dw) in 64 bits and the bounds of each."""
    m, d = h.shape
    v = w.shape[0]
    out = y == ignore
    bad = ~out & ((y < 0) | (y >= v))
    live = ~out & ~bad
    x = np.where(live[:, None], h, 0.0)
    z, s = x @ w.T, np.abs(x) @ np.abs(w).T
    top = z.max(axis=1, keepdims=True)
    lse = top[:, 0] + np.log(np.exp(z - top).sum(axis=1))
    rows = np.arange(m)
    yy = np.where(live, y, 0)
    row = np.where(live, lse - z[rows, yy], np.where(bad, np.nan, 0.0))
    count = int((~out).sum())
    loss = row.sum() / count if count else 0.0
    e = 2.0 ** -20 if dtype == "f32" else 0.0
    ez = ((2 * d * 2.0 ** -23 + e) * s).max(axis=1)
    row_tol = 2 * ez + 2.0 ** -15 + 2.0 ** -22 * (np.abs(lse) + np.abs(z[rows, yy]))
    loss_tol = np.where(live, row_tol, 0.0).sum() / max(count, 1) + 2.0 ** -23 * abs(np.nan_to_num(loss))
    p = np.exp(z - lse[:, None]) * live[:, None]
    rp = (2 * ez + 2.0 ** -15)[:, None] + 2.0 ** -22 * (1 + np.abs(z - lse[:, None]))
    ep = p * rp
    p1 = p.copy()
    p1[rows[live], y[live]] -= 1.0
    ep = ep + (HALF_STEP["bf16"] if dtype == "bf16" else 2.0 ** -22) * np.abs(p1) + 2.0 ** -24 * (p1 < 0) + 2.0 ** -126
    n = max(count, 1)

    def product(a, ea, b):
        k = a.shape[1]
        want = a @ b / n
        tol = (ea @ np.abs(b) + (2 * k * 2.0 ** -23 + e) * (np.abs(a) @ np.abs(b))) / n
        return want, tol * (1 + 2.0 ** -20) + (HALF_STEP[dtype] + 2.0 ** -22) * np.abs(want) + 1e-38
    dh, dh_tol = product(p1, ep, w)
    dw, dw_tol = product(p1.T, ep.T, x)
    return (loss, row, dh, dw), (loss_tol, row_tol, dh_tol, dw_tol)


def check(G, h, w, y, dtype, ignore=-1, what=("row", "dh", "dw"), stream=None):
    import torch
    m, d = h.shape
    v = w.shape[0]
    loss = torch.full((1,), -7.0, device="cuda")
    row = torch.full((m + 3,), -7.0, device="cuda") if "row" in what else None

    def empty(rows):
        return torch.full((rows + 1, unit_end(d, dtype) + unit_end(1, dtype)), -7.0, dtype=torch_type(dtype),
                          device="cuda")[:, :d]
    dh = empty(m) if "dh" in what else None
    dw = empty(v) if "dw" in what else None
    yd = torch.from_numpy(np.asarray(y, np.int32)).cuda()
    G.linear_xent(h, w, yd, loss, row_loss=row, dh=dh, dw=dw, ignore_label=ignore)
    G.sync()
    want, tol = reference(f64(h), f64(w), np.asarray(y), ignore, dtype)
    got_loss = loss.item()
    if np.isnan(want[0]):
        assert np.isnan(got_loss)
    else:
        assert abs(got_loss - want[0]) <= tol[0], (got_loss, want[0], tol[0])
    if row is not None:
        r = f64(row)
        assert (r[m:] == -7).all()
        bad = np.isnan(want[1])
        assert np.array_equal(np.isnan(r[:m]), bad)
        assert (np.abs(r[:m] - want[1]) <= tol[1])[~bad].all()
    for g, x, t, rows in ((dh, want[2], tol[2], m), (dw, want[3], tol[3], v)):
        if g is None:
            continue
        got = f64(g)[:rows]
        worst = (np.abs(got - x) / t).max() if rows else 0.0
        assert worst <= 1.0, (worst, rows)
        b = wide(g).float().cpu()
        end = unit_end(d, dtype)
        assert (b[:rows, d:end] == 0).all() and (b[:, end:] == -7).all() and (b[rows:] == -7).all()
    return loss, row, dh, dw


SHAPES = [(1, 1, 1), (1, 5, 3), (3, 300, 8), (2, 256, 16), (31, 255, 40), (32, 257, 64), (33, 512, 65), (64, 1000, 100),
          (100, 777, 128), (128, 256, 129), (129, 700, 130), (200, 2000, 250), (257, 513, 300), (5, 3000, 602),
          (130, 260, 520)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v,d", SHAPES)
def test_loss_and_gradients(G, m, v, d, dtype):
    say("xent", m, v, d, dtype)
    rng = np.random.default_rng(m + v + d)
    h, w = matrix(m, d, dtype, m + 1, extra=1), matrix(v, d, dtype, v + 2, extra=1)
    y = rng.integers(0, v, m)
    y[rng.random(m) < 0.2] = -1
    check(G, h, w, y, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v,d", [(150, 33_001, 200), (300, 17_000, 400), (60, 33_001, 70)])
def test_loss_and_gradients_of_many_classes(G, m, v, d, dtype):
    """Enough classes for the products' largest tiles."""
    say("xent many classes", m, v, d, dtype)
    rng = np.random.default_rng(m + v + d)
    h, w = matrix(m, d, dtype, m + 1, extra=1), matrix(v, d, dtype, v + 2, extra=1)
    y = rng.integers(0, v, m)
    y[rng.random(m) < 0.2] = -1
    check(G, h, w, y, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", [(), ("row",), ("dh",), ("dw",), ("row", "dw")], ids=str)
def test_what_is_asked_for(G, what, dtype):
    say("xent outputs", what, dtype)
    for m in (7, 140):
        h, w = matrix(m, 48, dtype, 1), matrix(600, 48, dtype, 2)
        check(G, h, w, np.arange(m) * 4 % 600, dtype, what=what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m", [20, 150])
def test_rows_that_do_not_count(G, m, dtype):
    """Padded rows hold NaN and infinities; nothing of them reaches a result."""
    import torch
    say("xent padded rows", m, dtype)
    v, d = 500, 72
    h, w = matrix(m, d, dtype, 1), matrix(v, d, dtype, 2)
    y = np.arange(m) % v
    y[m // 2:] = -100
    clean = check(G, h, w, y, dtype, ignore=-100)
    for value in (float("nan"), float("inf"), -float("inf"), 3e38):
        hh = h.clone()
        hh[m // 2:] = value
        loss, row, dh, dw = (torch.full_like(t, -3.0) for t in clean)
        yd = torch.from_numpy(y.astype(np.int32)).cuda()
        G.linear_xent(hh, w, yd, loss, row_loss=row[:m], dh=dh, dw=dw, ignore_label=-100)
        assert torch.equal(loss, clean[0]) and torch.equal(row[:m], clean[1][:m])
        assert torch.equal(dh[:m], clean[2][:m]) and torch.equal(dw[:v], clean[3][:v])
        assert (dh[m // 2:m] == 0).all() and (row[m // 2:m] == 0).all()
    # an ignored label may be a class
    check(G, h, w, np.where(np.arange(m) % 3 == 0, 4, np.arange(m) % v), dtype, ignore=4)
    # no row counts, and no row at all
    loss, row, dh, dw = check(G, h, w, np.full(m, -1), dtype)
    assert loss.item() == 0 and (dh[:m] == 0).all() and (dw[:v] == 0).all()
    dw2, loss2 = torch.full((v, d), 3.0, dtype=w.dtype, device="cuda"), torch.full((1,), 3.0, device="cuda")
    G.linear_xent(h[:0], w, torch.zeros(0, dtype=torch.int32, device="cuda"), loss2, dw=dw2)
    assert loss2.item() == 0 and (dw2 == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_labels_outside_the_classes(G, dtype):
    say("xent bad labels", dtype)
    h, w = matrix(40, 32, dtype, 1), matrix(300, 32, dtype, 2)
    y = np.arange(40) * 7
    y[3], y[39], y[20] = 300, -2, 2 ** 31 - 1
    loss, row, dh, dw = check(G, h, w, y, dtype)
    assert np.isnan(loss.item()) and (dh[[3, 39, 20]] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_and_equal_logits(G, dtype):
    """Logits of several hundred, a confident row, all classes equal: no overflow, exact ties."""
    import torch
    say("xent large logits", dtype)
    m, v, d = 50, 900, 64
    h, w = matrix(m, d, dtype, 1), matrix(v, d, dtype, 2)
    h.mul_(16.0)
    check(G, h, w, np.arange(m), dtype)
    h.zero_()
    loss, row, dh, dw = check(G, h, w, np.arange(m), dtype)
    assert row[0].item() == pytest.approx(np.log(v), rel=1e-6)
    h[:, 0] = -1.0
    w[:, 0] = 1e30                  # every logit -1e30
    w[:, 1:] = 0
    loss, row, dh, dw = (torch.zeros(1, device="cuda"), torch.zeros(m, device="cuda"), torch.zeros_like(h), torch.zeros_like(w))
    G.linear_xent(h, w, torch.arange(m, dtype=torch.int32, device="cuda"), loss, row_loss=row, dh=dh, dw=dw)
    assert row[0].item() == pytest.approx(np.log(v), rel=1e-6) and torch.isfinite(dw).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinite_and_nan_inputs(G, dtype):
    """A class whose logits are all -inf has no share in anything (bf16; fp32's part products make NaN of
    an infinite entry, which every row then shows); a NaN row spoils its own loss and dw, no other row's dh."""
    import torch
    say("xent infinities", dtype)
    m, v, d = 40, 700, 24
    h, w = matrix(m, d, dtype, 1), matrix(v, d, dtype, 2)
    h[:, 0] = 1.0
    w[300:640, 0] = -float("inf")   # a whole tile of classes and more
    y = torch.arange(m, dtype=torch.int32, device="cuda")
    loss, row, dh, dw = (torch.zeros(1, device="cuda"), torch.zeros(m, device="cuda"), torch.zeros_like(h), torch.zeros_like(w))
    G.linear_xent(h, w, y, loss, row_loss=row)
    keep = torch.cat([w[:300], w[640:]])
    loss2, row2 = torch.zeros(1, device="cuda"), torch.zeros(m, device="cuda")
    G.linear_xent(h, keep, y, loss2, row_loss=row2)
    if dtype == "f32":
        assert torch.isnan(row).all() and torch.isnan(loss).all()
    else:
        assert torch.allclose(row, row2, rtol=1e-5, atol=1e-5) and torch.isfinite(loss).all()
    w = matrix(v, d, dtype, 2)
    h[5, 3] = float("nan")
    G.linear_xent(h, w, y, loss, row_loss=row, dh=dh, dw=dw)
    nan = torch.isnan(row)
    assert nan.nonzero().flatten().tolist() == [5] and torch.isnan(loss).all()
    assert torch.isnan(dh[5]).all() and torch.isfinite(dh[:5]).all() and torch.isfinite(dh[6:]).all()


@pytest.mark.parametrize("dtype,m,v,d", [("f32", 4000, 70_001, 16), ("bf16", 8100, 90_001, 24), ("bf16", 8000, 80_001, 264),
                                         ("f32", 70_001, 300, 40), ("bf16", 70_001, 300, 40)])
def test_several_pieces_of_classes(G, dtype, m, v, d):
    """More classes than a piece holds, the last piece ragged; in 64 bits on the device."""
    import torch
    say("xent pieces", dtype, m, v, d)
    h, w = matrix(m, d, dtype, 1), matrix(v, d, dtype, 2)
    y = torch.randint(0, v, (m,), device="cuda")
    y[::7] = -1
    loss, row, dh, dw = (torch.zeros(1, device="cuda"), torch.zeros(m, device="cuda"),
                         torch.zeros((m, d), dtype=h.dtype, device="cuda"), torch.zeros((v, d), dtype=h.dtype, device="cuda"))
    G.linear_xent(h, w, y.int(), loss, row_loss=row, dh=dh, dw=dw)
    keep = y >= 0
    x, ww = h.double() * keep[:, None], w.double()
    z = x @ ww.t()
    lse = torch.logsumexp(z, 1)
    at = torch.arange(m, device="cuda")
    want = torch.where(keep, lse - z[at, y.clamp(min=0)], 0.0)
    # 2 ez + 2^-15 + rounding, ez <= (2 d 2^-23 + 2^-20) max sum |h w| <= 2^-17 * 60
    assert (row.double() - want).abs().max().item() <= 2 * 60 * 2.0 ** -17 + 2.0 ** -15
    p = torch.exp(z - lse[:, None])
    p[at, y.clamp(min=0)] -= 1
    p *= keep[:, None] / keep.sum()
    # by the norm: p within 2^-8 (bf16) or 2^-9 of 2 ez (fp32), random over the terms, and the output's rounding
    bound = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -9
    for got, ref in ((dh, p @ ww), (dw, p.t() @ x)):
        assert torch.linalg.norm(got.double() - ref).item() <= bound * torch.linalg.norm(ref).item()
    again = torch.zeros_like(dw), torch.zeros_like(dh)
    G.linear_xent(h, w, y.int(), loss, dh=again[1], dw=again[0])
    assert torch.equal(again[0], dw) and torch.equal(again[1], dh)      # the same bits on every run


def test_gradients_against_differences(G):
    """fp32 loss differences along one entry; step 1e-2 leaves a curvature of 1e-4 of the loss, rounding 1e-5 / 2e-2."""
    import torch
    m, v, d = 12, 90, 20
    h, w = matrix(m, d, "f32", 1), matrix(v, d, "f32", 2)
    h.mul_(0.5)
    y = torch.arange(m, dtype=torch.int32, device="cuda") * 5
    loss, dh, dw = torch.zeros(1, device="cuda"), torch.zeros((m, d), device="cuda"), torch.zeros((v, d), device="cuda")
    G.linear_xent(h, w, y, loss, dh=dh, dw=dw)
    dh0, dw0 = dh.clone(), dw.clone()
    for t, g, at in ((h, dh0, (0, 0)), (h, dh0, (11, 19)), (w, dw0, (0, 3)), (w, dw0, (55, 7)), (w, dw0, (89, 19))):
        old, value = t[at].item(), []
        for step in (1e-2, -1e-2):
            t[at] = old + step
            G.linear_xent(h, w, y, loss)
            value.append(loss.item())
        t[at] = old
        assert (value[0] - value[1]) / 2e-2 == pytest.approx(g[at].item(), abs=3e-4)


def test_workspace_is_guarded(G):
    """A workspace of exactly the size asked for, canaries behind it, garbage in it."""
    import torch
    for dtype in ("f32", "bf16"):
        for m, v, d, grads in ((5, 700, 40, True), (5, 700, 40, False), (200, 1300, 100, True), (200, 1300, 300, False)):
            need = G.linear_xent_workspace(m, v, d, dtype, grads)
            ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
            h, w = matrix(m, d, dtype, 1), matrix(v, d, dtype, 2)
            y = torch.arange(m, dtype=torch.int32, device="cuda")
            res = []
            for given in (ws[:need], None):
                loss, dh, dw = torch.zeros(1, device="cuda"), matrix(m, d, dtype, 3), matrix(v, d, dtype, 3)
                G.linear_xent(h, w, y, loss, dh=dh if grads else None, dw=dw if grads else None, workspace=given)
                res.append((loss, dh, dw))
            assert all(torch.equal(a, b) for a, b in zip(*res)) and (ws[need:] == 0xFF).all()
            with pytest.raises(G.GnnavError):
                G.linear_xent(h, w, y, loss, dh=dh if grads else None, workspace=ws[:need // 2])


def test_argument_types(G):
    import torch
    h, w, y, one = (torch.zeros((4, 8), device="cuda"), torch.zeros((6, 8), device="cuda"),
                    torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda"))
    for bad in (lambda: G.linear_xent(h, w.bfloat16(), y, one), lambda: G.linear_xent(h, w[:, :4], y, one),
                lambda: G.linear_xent(h, w, y.long(), one), lambda: G.linear_xent(h, w, y[:3], one),
                lambda: G.linear_xent(h, w, y, one.double()), lambda: G.linear_xent(h, w, y, one, dh=h[:2]),
                lambda: G.linear_xent(h, w, y, one, dw=h), lambda: G.linear_xent(h, w, y, one, row_loss=one)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v,d", [(1, 20_001, 96), (2, 129, 200), (4, 40_000, 373), (9, 1_000, 64), (16, 70_003, 33),
                                   (17, 5_000, 1_030), (32, 60_001, 128), (32, 300_001, 16), (20, 524_289, 72), (33, 20_001, 129), (50, 60_000, 40), (64, 131_073, 64)])
def test_few_rows(G, m, v, d, dtype):
    """At most 64 rows: several blocks of classes a workgroup, columns that end inside a block's."""
    say("xent few rows", m, v, d, dtype)
    rng = np.random.default_rng(m + v + d)
    h, w = matrix(m, d, dtype, m + 1, extra=1), matrix(v, d, dtype, v + 2, extra=1)
    y = rng.integers(0, v, m)
    if m > 2:
        y[0], y[1], y[m - 1] = -1, v - 1, 0
    for what in (("row", "dh", "dw"), ("dh",), ("dw",)):
        check(G, h, w, y, dtype, what=what)


@pytest.mark.parametrize("m,v", [(17, 8_400_000), (40, 1_050_000)])
def test_few_rows_of_very_many_classes(G, m, v):
    """More logits than are kept: the classes are taken in pieces, or by the tiles."""
    say("xent very many classes", m, v)
    d = 8
    h, w = matrix(m, d, "bf16", 1, extra=1), matrix(v, d, "bf16", 2, extra=1)
    check(G, h, w, np.arange(m) * (v // m - 1), "bf16", what=("row", "dh", "dw"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v,d", [(20, 140_000, 40), (50, 70_000, 130), (130, 1300, 100), (290, 40_000, 200)])
def test_garbage_in_the_workspace(G, m, v, d, dtype):
    """NaN in every byte of a workspace of the size asked for, and canaries behind it: the same bits as with zeros."""
    import torch
    say("xent garbage", m, v, d, dtype)
    h, w = matrix(m, d, dtype, 1), matrix(v, d, dtype, 2)
    y = (torch.arange(m, dtype=torch.int32, device="cuda") * 17) % v
    need = G.linear_xent_workspace(m, v, d, dtype, True)
    res = []
    for fill in (0, 0xFF):
        ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
        ws[:need] = fill
        loss, row, dh, dw = torch.zeros(1, device="cuda"), torch.zeros(m, device="cuda"), matrix(m, d, dtype, 3), matrix(v, d, dtype, 3)
        G.linear_xent(h, w, y, loss, row_loss=row, dh=dh, dw=dw, workspace=ws[:need])
        assert (ws[need:] == 0x5A).all()
        res.append((loss, row, dh, dw))
    assert all(torch.equal(a, b) and torch.isfinite(b).all() for a, b in zip(*res))
