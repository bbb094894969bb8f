"""Cross entropy over many classes where logits are infinite, huge or all alike and
where rows do not count, on each of its paths: the kernels for few rows (40), rows
held in registers (bf16, at most 256 columns), and the tiles.
"""
import numpy as np
import pytest

from test_gpu_embedding import HALF_STEP, f64, matrix, torch_type
from test_gpu_linear_xent import check, reference
from test_gpu_parity import G, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu

PATHS = [(40, 24), (70, 24), (150, 24), (70, 300), (150, 300)]   # rows, columns


def outputs(m, v, d, dtype):
    import torch
    t = torch_type(dtype)
    return (torch.full((1,), 3.0, device="cuda"), torch.full((m,), 3.0, device="cuda"),
            torch.full((m, (d + 7) // 8 * 8), 3.0, dtype=t, device="cuda")[:, :d],
            torch.full((v, (d + 7) // 8 * 8), 3.0, dtype=t, device="cuda")[:, :d])


@pytest.mark.parametrize("ignored", [False, True])
@pytest.mark.parametrize("m,d", PATHS)
def test_classes_of_minus_infinity(G, m, d, ignored):
    """bf16: classes whose logits are -inf in every row that counts have p = 0: the gradients are those of the other
    classes alone, and theirs zero, whatever rows do not count.  (dh of the column that holds the infinity is 0 * inf.)"""
    import torch
    say("xent -inf classes", m, d, ignored)
    v, a, b = 900, 300, 640
    h, w = matrix(m, d, "bf16", 1), matrix(v, d, "bf16", 2)
    h[:, 0] = 1.0
    w[a:b, 0] = -float("inf")
    y = np.arange(m) * 3 % a
    if ignored:
        y[::3] = -1
    yd = torch.from_numpy(y.astype(np.int32)).cuda()
    loss, row, dh, dw = outputs(m, v, d, "bf16")
    G.linear_xent(h, w, yd, loss, row_loss=row, dh=dh, dw=dw)
    keep = np.r_[0:a, b:v]
    want, tol = reference(f64(h), f64(w)[keep], y, -1, "bf16")
    assert abs(loss.item() - want[0]) <= tol[0] and (np.abs(f64(row) - want[1]) <= tol[1]).all()
    assert (np.abs(f64(dh) - want[2]) <= tol[2])[:, 1:].all()
    assert (np.abs(f64(dw)[keep] - want[3]) <= tol[3]).all()
    assert (dw[a:b] == 0).all()
    alone = outputs(m, v, d, "bf16")
    G.linear_xent(h, w, yd, alone[0], dw=alone[3])
    assert torch.equal(alone[3], dw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,d", PATHS)
def test_no_row_counts_and_classes_are_infinite(G, m, d, dtype):
    """No row that counts: loss and gradients are zero, whatever w holds."""
    import torch
    say("xent nothing counts", m, d, dtype)
    v = 700
    for value in (float("inf"), -float("inf"), float("nan")):
        h, w = matrix(m, d, dtype, 1), matrix(v, d, dtype, 2)
        w[5], w[300:640, 0] = value, value
        h[m // 2:] = float("nan")
        loss, row, dh, dw = outputs(m, v, d, dtype)
        G.linear_xent(h, w, torch.full((m,), -1, dtype=torch.int32, device="cuda"), loss, row_loss=row, dh=dh, dw=dw)
        assert all((t == 0).all() for t in (loss, row, dh, dw))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,d", PATHS)
def test_labels_outside_the_classes(G, m, d, dtype):
    say("xent bad labels", m, d, dtype)
    h, w = matrix(m, d, dtype, 1), matrix(300, d, dtype, 2)
    y = np.arange(m) * 7 % 300
    y[3], y[m - 1], y[20], y[21] = 300, -2, 2 ** 31 - 1, -1
    loss, row, dh, dw = check(G, h, w, y, dtype)
    assert np.isnan(loss.item()) and (dh[[3, m - 1, 20, 21]] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,d", PATHS)
def test_rows_of_nan_and_infinity(G, m, d, dtype):
    """A counted row of NaN or infinities spoils its own loss and dh, and dw, but no other row's loss or dh."""
    import torch
    say("xent nan rows", m, d, dtype)
    v = 700
    for value in (float("nan"), float("inf")):
        h, w = matrix(m, d, dtype, 1), matrix(v, d, dtype, 2)
        y = torch.arange(m, dtype=torch.int32, device="cuda")
        clean, spoilt = outputs(m, v, d, dtype), outputs(m, v, d, dtype)
        G.linear_xent(h, w, y, clean[0], row_loss=clean[1], dh=clean[2], dw=clean[3])
        h[m - 3, 3] = value
        G.linear_xent(h, w, y, spoilt[0], row_loss=spoilt[1], dh=spoilt[2], dw=spoilt[3])
        others = [i for i in range(m) if i != m - 3]
        assert torch.isnan(spoilt[1][m - 3]) and torch.isnan(spoilt[0]).all() and torch.isnan(spoilt[2][m - 3]).all()
        assert torch.equal(spoilt[1][others], clean[1][others]) and torch.equal(spoilt[2][others], clean[2][others])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,d", PATHS)
@pytest.mark.parametrize("base", [0.0, 2.0 ** 8, 2.0 ** 14, 2.0 ** 20, -2.0 ** 20, 2.0 ** 100], ids=str)
def test_logits_far_from_zero(G, m, d, dtype, base):
    """Adding the same number to all of a row's logits changes no p.

    h holds |base|^(1/2) and 1, w +-|base|^(1/2) and -k, k = 0 .. 3 (0 at 2^100): the logits base - k are exact in fp32, so p is off by its own arithmetic alone: 2^-15 and 2^-22 (1 + |z - lse|) of it, as
    test_gpu_linear_xent.py derives, its rounding (bf16), and the sums over 1 to m rows and the result's rounding.
    """
    import torch
    say("xent far logits", m, d, dtype, base)
    v = 900
    t = dict(dtype=torch_type(dtype), device="cuda")
    h, w = torch.zeros((m, (d + 7) // 8 * 8), **t)[:, :d], torch.zeros((v, (d + 7) // 8 * 8), **t)[:, :d]
    k = np.arange(v) % (4 if abs(base) < 2.0 ** 30 else 1)
    h[:, 0], h[:, 1] = abs(base) ** 0.5, 1.0
    w[:, 0] = float(np.copysign(abs(base) ** 0.5, base))
    w[:, 1] = -torch.from_numpy(k.astype(np.float32)).cuda().to(t["dtype"])
    y = np.arange(m) * 5 % v
    y[1] = -1
    loss, row, dh, dw = outputs(m, v, d, dtype)
    G.linear_xent(h, w, torch.from_numpy(y.astype(np.int32)).cuda(), loss, row_loss=row, dh=dh, dw=dw)
    z = -k.astype(float)
    lse = np.log(np.exp(z).sum())
    live, p = y >= 0, np.exp(z - lse)
    n = live.sum()
    want = np.where(live, lse - z[np.where(live, y, 0)], 0.0)
    assert (np.abs(f64(row) - want) <= 2.0 ** -15 + 2.0 ** -20).all()
    assert abs(loss.item() - want.sum() / n) <= 2.0 ** -15 + 2.0 ** -20
    # column 1 of h is 1: dw there is the sum of p - [v = y] over the rows that count, divided by their number
    hits = np.bincount(y[live], minlength=v)
    got = f64(dw)[:, 1]
    exact = p - hits / n
    ep = p * (2.0 ** -15 + 2.0 ** -22 * (1 + np.abs(z - lse)))
    ep = ep + (HALF_STEP["bf16"] if dtype == "bf16" else 2.0 ** -22) * (p + hits / n) + 2.0 ** -24 * hits / n
    tol = ep + (2 * m * 2.0 ** -23 + 2.0 ** -20) * (p + hits / n) + (HALF_STEP[dtype] + 2.0 ** -22) * np.abs(exact)
    worst = (np.abs(got - exact) / tol).max()
    assert worst <= 1.0
    # dh's column 1: sum_v p_v (-k_v) + k_y, of one row
    x = np.where(live, (-p * k).sum() + k[np.where(live, y, 0)], 0.0) / n
    size = (p * k).sum() + k[np.where(live, y, 0)]
    rel = 2.0 ** -15 + 2.0 ** -19 + (HALF_STEP["bf16"] if dtype == "bf16" else 2.0 ** -22) + 2 * v * 2.0 ** -23 + 2.0 ** -20
    worst = (np.abs(f64(dh)[:, 1] - x) / (rel * size / n + (HALF_STEP[dtype] + 2.0 ** -22) * np.abs(x) + 1e-30)).max()
    assert worst <= 1.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,d", PATHS)
def test_large_logits(G, m, d, dtype):
    """Logits of several hundred and thousand, confident rows: no overflow."""
    say("xent large logits", m, d, dtype)
    for scale in (16.0, 256.0):
        h, w = matrix(m, d, dtype, 1), matrix(900, d, dtype, 2)
        h.mul_(scale)
        y = np.arange(m)
        y[::5] = -1
        check(G, h, w, y, dtype)


def test_sums_of_many_equal_terms(G):
    """bf16, a million classes, no gradients: logits 0 at two classes of each 512 (one for each half of a wavefront), all
    others ln t with t = 0.45 of a step above a multiple of 2^-10, which a sum past 8,192 that takes them one by one loses
    each time.  A row's sum may round 384 times along a wavefront's run of tiles, 17 times in a tile and 128 times where
    runs are joined: (384 + 17 + 128) 2^-24 of it; exp2's argument and result are off by 2^-22 (1 + |z|); a few roundings
    of the result."""
    import torch
    m, v, d = 4096, (1 << 20) - 300, 16
    say("xent long sums", m, v, d)
    t = (717 + 0.45) * 2.0 ** -10
    hi = torch.tensor(np.log(t), dtype=torch.float64).bfloat16()
    lo = torch.tensor(np.log(t) - hi.item(), dtype=torch.float64).bfloat16()
    h, w = torch.zeros((m, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((v, d), dtype=torch.bfloat16, device="cuda")
    h[:, :2] = 1.0
    w[:, 0], w[:, 1] = hi.item(), lo.item()
    w[::512] = 0.0
    w[4::512] = 0.0
    zeros = len(range(0, v, 512)) + len(range(4, v, 512))
    loss, row = torch.zeros(1, device="cuda"), torch.zeros(m, device="cuda")
    G.linear_xent(h, w, torch.zeros(m, dtype=torch.int32, device="cuda"), loss, row_loss=row)
    want = np.log(zeros + (v - zeros) * np.exp(hi.double().item() + lo.double().item()))
    tol = (384 + 17 + 128) * 2.0 ** -24 + 2.0 ** -22 * (2 + abs(np.log(t))) + 2.0 ** -22 * want
    off = np.abs(f64(row) - want).max()
    say("off by", off, "of", tol)
    assert off <= tol


@pytest.mark.parametrize("dtype,m,v,d", [("f32", 70, 157_300, 1_000), ("bf16", 70, 230_001, 2_050)])
def test_weights_packed_twice(G, dtype, m, v, d):
    """Packed weights of more than 896 MiB are not kept between the passes: each packs its pieces, the last one ragged.
    In a workspace of the size asked for, every byte NaN; against 64 bits on the device.  Bounds as of
    test_several_pieces_of_classes: ez by the largest sum of |h w|, gradients by the norm."""
    import torch
    say("xent packed twice", dtype, m, v, d)
    gen = torch.Generator(device="cuda").manual_seed(5)
    ld = (d + 7) // 8 * 8
    t = dict(dtype=torch_type(dtype), device="cuda")
    h = torch.randn((m, ld), generator=gen, device="cuda").to(t["dtype"])[:, :d]
    w = (torch.randn((v, ld), generator=gen, device="cuda") / d ** 0.5).to(t["dtype"])[:, :d]
    y = (torch.arange(m, device="cuda") * 2_237) % v
    y[-1], y[::7] = v - 1, -1
    loss, row, dh, dw = outputs(m, v, d, dtype)
    need = G.linear_xent_workspace(m, v, d, dtype, True)
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    G.linear_xent(h, w, y.int(), loss, row_loss=row, dh=dh, dw=dw, workspace=ws[:need])
    assert (ws[need:] == 0xFF).all()
    keep = y >= 0
    x = h.double() * keep[:, None]
    z, biggest, step = torch.empty((m, v), dtype=torch.float64, device="cuda"), 0.0, 16_384
    for a in range(0, v, step):
        piece = w[a:a + step].double()
        z[:, a:a + step] = x @ piece.t().contiguous()
        biggest = max(biggest, (x.abs() @ piece.abs().t().contiguous()).max().item())
    lse = torch.logsumexp(z, 1)
    at = torch.arange(m, device="cuda")
    want = torch.where(keep, lse - z[at, y.clamp(min=0)], 0.0)
    ez = (2 * d * 2.0 ** -23 + (2.0 ** -20 if dtype == "f32" else 0.0)) * biggest
    assert (row.double() - want).abs().max().item() <= 2 * ez + 2.0 ** -15 + 2.0 ** -18
    assert abs(loss.item() - want.sum().item() / keep.sum().item()) <= 2 * ez + 2.0 ** -15 + 2.0 ** -18
    p = torch.exp(z - lse[:, None])
    p[at, y.clamp(min=0)] -= 1
    p *= keep[:, None] / keep.sum()
    want_dh = torch.zeros((m, d), dtype=torch.float64, device="cuda")
    bound = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -9
    for a in range(0, v, step):
        q = p[:, a:a + step].contiguous()
        want_dh += q @ w[a:a + step].double()
        ref = q.t().contiguous() @ x
        assert torch.linalg.norm(dw[a:a + step].double() - ref).item() <= bound * torch.linalg.norm(ref).item(), a
    assert torch.linalg.norm(dh.double() - want_dh).item() <= bound * torch.linalg.norm(want_dh).item()


@pytest.mark.parametrize("m,v,d", [(1, 20_001, 96), (1, 300, 24), (3, 9_000, 200), (30, 5_000, 300), (64, 3_001, 130), (17, 600_001, 40)])
def test_gradients_of_few_bf16_rows_are_rounded_once(G, m, v, d):
    """Up to 64 rows, p - [v = y] is multiplied in two bf16 parts, 2^-8 of 2^-8 off at most: sums this short would show one
    of 2^-8.  What is left is p's own error (as test_gpu_linear_xent.py derives), the sums' and the result's."""
    say("xent few rows, rounding", m, v, d)
    rng = np.random.default_rng(m + v + d)
    h, w = matrix(m, d, "bf16", m + 1), matrix(v, d, "bf16", v + 2)
    y = rng.integers(0, v, m)
    if m > 2:
        y[1] = -1
    import torch
    loss, row, dh, dw = outputs(m, v, d, "bf16")
    G.linear_xent(h, w, torch.from_numpy(y.astype(np.int32)).cuda(), loss, row_loss=row, dh=dh, dw=dw)
    x, ww, live, rows = f64(h), f64(w), y >= 0, np.arange(m)
    x[~live] = 0
    z, s = x @ ww.T, np.abs(x) @ np.abs(ww).T
    lse = np.log(np.exp(z - z.max(axis=1, keepdims=True)).sum(axis=1)) + z.max(axis=1)
    ez = (2 * d * 2.0 ** -23 * s).max(axis=1)
    p = np.exp(z - lse[:, None]) * live[:, None]
    ep = p * ((2 * ez + 2.0 ** -15)[:, None] + 2.0 ** -22 * (1 + np.abs(z - lse[:, None])))
    p[rows[live], y[live]] -= 1
    ep += 2.0 ** -16 * np.abs(p) + 2.0 ** -24 * (p < 0) + 2.0 ** -126
    n = live.sum()

    def worst(got, a, ea, b):
        want = a @ b / n
        tol = (ea @ np.abs(b) + 2 * a.shape[1] * 2.0 ** -23 * (np.abs(a) @ np.abs(b))) / n
        return (np.abs(f64(got) - want) / (tol * (1 + 2.0 ** -20) + (HALF_STEP["bf16"] + 2.0 ** -22) * np.abs(want) + 1e-38)).max()
    assert worst(dw, p.T, ep.T, x) <= 1.0
    assert worst(dh, p, ep, ww) <= 1.0
