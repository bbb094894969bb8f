"""Distillation from a teacher's top logits with the labels' cross entropy, against numpy in 64 bits.

Tolerances follow the arithmetic.  exp takes an argument x = (z - M) / T off by 2^-23 |x| (bf16's path another 2^-23 |x| for
log2 e), which moves it by the same part of itself, and is off by 2^-22; a class beyond x = -87 may count as 0.  A
sum of C exponentials rounds at most (C / 64 + 32) 2^-24 of it in a thread's and a workgroup's additions.  So p is off by
rp = 2^-21 (|x| + |x|_mean + 2) + (C / 64 + 32) 2^-24 of itself, |x|_mean that of the row under p, and the log of the sum by
as much; q likewise over its k entries.  dlogits add their parts and round once; the loss sums k terms.
"""
import numpy as np
import pytest

from test_gpu_embedding import HALF_STEP, f64, matrix, torch_type, unit_end, wide
from test_gpu_parity import G, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def softmax(x, there):
    """softmax over the places that are there (rows of none: zeros), its log, and the relative tolerance of either."""
    x = np.where(there, x, -np.inf)
    top = x.max(axis=1, keepdims=True, initial=-np.inf)
    top = np.where(np.isfinite(top), top, 0.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.exp(x - top)
        s = e.sum(axis=1, keepdims=True)
        p = e / np.where(s == 0, 1.0, s)
        logs = np.where(there, x - top, 0.0) - np.log(np.where(s == 0, 1.0, s))
    far = np.where(np.isfinite(x), np.abs(x - top), 0.0)
    r = 2.0 ** -21 * (far + (p * far).sum(axis=1, keepdims=True) + 2) + (x.shape[1] / 64 + 32) * U
    return p, logs, r


def reference(z, ids, t, temp, alpha, labels, ignore, dtype):
    m, c = z.shape
    k = ids.shape[1]
    rows = np.arange(m)
    there = (ids >= 0) & (t > -np.inf)
    has, wrong = there.any(axis=1), (there & (ids >= c)).any(axis=1)
    if alpha == 0:
        has[:] = wrong[:] = False
    if labels is None or alpha == 1:
        labels = np.full(m, ignore)
    counted = labels != ignore
    off = counted & ((labels < 0) | (labels >= c))
    A, B = max(int(has.sum()), 1), max(int(counted.sum()), 1)
    q, log_q, rq = softmax(t / temp, there)
    p, log_p, rp = softmax(z / temp, np.ones((m, c), bool))
    p1, log_p1, rp1 = softmax(z, np.ones((m, c), bool))
    at = np.where(there & (ids < c), ids, 0)
    lp, rl = log_p[rows[:, None], at], rp[rows[:, None], at]
    with np.errstate(invalid="ignore"):
        term = np.where(there & (q > 0), q * (log_q - lp), 0.0)
        tol = np.where(there & (q > 0), q * (rq * (1 + np.abs(log_q - lp)) + rl) + 2.0 ** -21 * np.abs(q) * (np.abs(log_q) + np.abs(lp)), 0.0)
    kd = temp ** 2 * term.sum(axis=1)
    ekd = temp ** 2 * (tol.sum(axis=1) + (k / 64 + 16) * U * np.abs(term).sum(axis=1)) + 2.0 ** -22 * np.abs(kd)
    kd = np.where(wrong, np.nan, np.where(has, kd, 0.0))
    y = np.where(counted & ~off, labels, 0)
    ce = -log_p1[rows, y]
    ece = rp1[rows, y] + 2.0 ** -21 * (np.abs(ce) + np.abs(z[rows, y] - z.max(axis=1)))
    ce = np.where(off, np.nan, np.where(counted, ce, 0.0))
    ekd, ece = np.where(has, ekd, 0.0), np.where(counted, ece, 0.0)
    row, erow = alpha * kd + (1 - alpha) * ce, alpha * ekd + (1 - alpha) * ece
    first, second = kd.sum() / A, ce.sum() / B
    e1, e2 = ekd.sum() / A + 2.0 ** -23 * np.nansum(np.abs(kd)) / A, ece.sum() / B + 2.0 ** -23 * np.nansum(np.abs(ce)) / B
    loss = np.array([alpha * first + (1 - alpha) * second, first, second])
    eloss = np.array([alpha * e1 + (1 - alpha) * e2 + 2.0 ** -22 * np.nan_to_num(abs(loss[0])), e1, e2]) + 1e-38
    target, etarget = np.zeros((m, c)), np.zeros((m, c))
    np.add.at(target, (rows[:, None], at), np.where(there, q, 0.0))
    np.add.at(etarget, (rows[:, None], at), np.where(there, q * (rq + k * U), 0.0))
    onehot = np.zeros((m, c))
    onehot[rows, y] = 1.0
    wk, wc = alpha * temp / A * (has & ~wrong), (1 - alpha) / B * (counted & ~off)
    dz = wk[:, None] * (p - target) + wc[:, None] * (p1 - onehot)
    edz = wk[:, None] * (p * rp + etarget + 4 * U * (p + target)) + wc[:, None] * (p1 * rp1 + 4 * U * (p1 + onehot))
    edz = edz + (HALF_STEP[dtype] + 2 * U) * np.abs(dz) + 1e-37
    return dict(loss=(loss, eloss), row=(row, erow * (1 + 2.0 ** -10) + 2.0 ** -22 * np.abs(np.nan_to_num(row)) + 1e-38), dz=(dz, edz))


def check(G, z, ids, t, temp=1.0, alpha=1.0, labels=None, ignore=-1, what=("row", "dz"), inplace=False):
    import torch
    m, c = z.shape
    dtype = "bf16" if z.dtype == torch.bfloat16 else "f32"
    want = reference(f64(z), np.asarray(ids), np.asarray(t, np.float64), temp, alpha, None if labels is None else np.asarray(labels), ignore, dtype)
    loss = torch.full((3,), -7.0, device="cuda")
    row = torch.full((m + 3,), -7.0, device="cuda") if "row" in what else None
    if inplace:
        dz = z
    else:
        dz = torch.full((m + 1, unit_end(c, dtype) + unit_end(1, dtype)), -7.0, dtype=torch_type(dtype), device="cuda")[:, :c] if "dz" in what else None
    G.distill(z, torch.from_numpy(np.asarray(ids, np.int32)).cuda(), torch.from_numpy(np.asarray(t, np.float32)).cuda(), loss, temperature=temp,
              alpha=alpha, labels=None if labels is None else torch.from_numpy(np.asarray(labels, np.int32)).cuda(), ignore_label=ignore,
              row_loss=row, dlogits=dz)
    G.sync()

    def near(got, name):
        value, tol = want[name]
        nan = np.isnan(value)
        assert np.array_equal(np.isnan(got), nan), name
        with np.errstate(invalid="ignore"):
            worst = np.where(nan | (got == value), 0.0, np.abs(got - value) / tol).max(initial=0.0)
        assert worst <= 1.0, (name, worst)
    near(f64(loss), "loss")
    if row is not None:
        near(f64(row)[:m], "row")
        assert (row[m:] == -7).all()
    if dz is not None:
        near(f64(dz)[:m], "dz")
        b, end = wide(dz).float().cpu(), unit_end(c, dtype)
        assert (b[:m, c:end] == 0).all()
        if not inplace:
            assert (b[:, end:] == -7).all() and (b[m:] == -7).all()
    return loss, row, dz


def aligned(m, c, dtype, value=0.0):
    import torch
    return torch.full((m, unit_end(c, dtype)), value, dtype=torch_type(dtype), device="cuda")[:, :c]


def teacher(m, c, k, seed, spread=2.0):
    """k distinct classes a row (as many as there are, then none) and logits in fp32."""
    rng = np.random.default_rng(seed)
    n = min(k, c)
    ids = np.full((m, k), -1, np.int32)
    for i in range(m):
        ids[i, :n] = rng.choice(c, n, replace=False)
    return ids, np.where(ids >= 0, rng.normal(0, spread, (m, k)), -np.inf).astype(np.float32)


SHAPES = [(1, 1, 1), (1, 5, 3), (3, 41, 8), (70, 41, 41), (5, 64, 1), (9, 100, 64), (130, 257, 20), (20, 1_000, 130), (33, 2_049, 50),
          (6, 5_000, 256), (3, 20_001, 64), (2, 70_003, 100), (300, 17, 4), (1_000, 6, 2), (1, 169_000, 32), (200, 12_001, 9)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,c,k", SHAPES)
def test_loss_and_gradient(G, m, c, k, dtype):
    say("distill", m, c, k, dtype)
    rng = np.random.default_rng(m + c + k)
    z = matrix(m, c, dtype, m + 1, extra=1)
    z.mul_(3.0)
    ids, t = teacher(m, c, k, c)
    labels = rng.integers(0, c, m)
    labels[rng.random(m) < 0.3] = -1
    check(G, z, ids, t, temp=2.0, alpha=0.7, labels=labels)
    check(G, z, ids, t, temp=1.0, alpha=0.5, labels=labels)
    check(G, z, ids, t, temp=0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [41, 1_000, 40_000])
@pytest.mark.parametrize("temp", [4.0, 3.0, 0.25])
def test_temperatures_beside_labels(G, c, temp, dtype):
    """Exponentials at the temperature and at 1, from one another or each by itself."""
    m, k = 30, 12
    z = matrix(m, c, dtype, 80).mul_(4.0)
    ids, t = teacher(m, c, k, 81)
    labels = np.random.default_rng(82).integers(0, c, m).astype(np.int32)
    say("distill temperatures", c, temp, dtype)
    check(G, z, ids, t, temp=temp, alpha=0.4, labels=labels)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [41, 3_000, 40_000])
def test_what_is_asked_for_and_in_place(G, c, dtype):
    say("distill outputs", c, dtype)
    m = 20
    z = matrix(m, c, dtype, 2)
    ids, t = teacher(m, c, 10, 5)
    labels = np.arange(m) % c
    for what in ((), ("row",), ("dz",)):
        check(G, z, ids, t, 3.0, 0.4, labels, what=what)
    check(G, z, ids, t, 3.0, 0.0, labels)             # the labels alone
    check(G, z, ids, t, 3.0, 1.0, labels)             # the teacher alone, labels or not
    import torch
    loss = torch.zeros(3, device="cuda")
    G.distill(z, None, None, loss, alpha=0.0, labels=torch.from_numpy(labels.astype(np.int32)).cuda())
    assert loss[1].item() == 0 and loss[0].item() == loss[2].item() > 0
    check(G, matrix(m, c, dtype, 2), ids, t, 3.0, 0.4, labels, inplace=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [41, 5_000])
def test_rows_that_do_not_count(G, c, dtype):
    """Rows without entries or labels: parts of zero, not in the means; those with neither may hold anything."""
    import torch
    say("distill padded rows", c, dtype)
    m, k = 30, 6
    z = matrix(m, c, dtype, 1)
    ids, t = teacher(m, c, k, 2)
    labels = np.arange(m) % c
    ids[::3] = -1                  # no entry
    t[1] = -np.inf                 # none either
    ids[2, 2:] = -1                # some
    t[4, 0] = -np.inf
    labels[::2] = -100
    clean = check(G, z, ids, t, 2.0, 0.5, labels, ignore=-100)
    for value in (float("nan"), float("inf"), -float("inf")):
        zz = matrix(m, c, dtype, 1)
        zz[::6] = value
        loss, row, dz = torch.full_like(clean[0], -3.0), torch.full_like(clean[1], -3.0), aligned(m, c, dtype, -3.0)
        G.distill(zz, torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), loss, temperature=2.0, alpha=0.5,
                  labels=torch.from_numpy(labels.astype(np.int32)).cuda(), ignore_label=-100, row_loss=row[:m], dlogits=dz)
        assert torch.equal(loss, clean[0]) and torch.equal(row[:m], clean[1][:m]) and torch.equal(dz[:m], clean[2][:m])
        assert (dz[:m:6] == 0).all() and (row[:m:6] == 0).all()
    # no row counts, and no row at all
    loss, row, dz = check(G, z, np.full((m, k), -1), t, 2.0, 0.5, np.full(m, -1))
    assert (loss == 0).all() and (dz[:m] == 0).all()
    loss = torch.full((3,), 5.0, device="cuda")
    G.distill(z[:0], torch.zeros((0, k), dtype=torch.int32, device="cuda"), torch.zeros((0, k), device="cuda"), loss)
    assert (loss == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [41, 4_000])
def test_same_class_twice_and_classes_outside(G, c, dtype):
    """Shares of one class add up; a class or a label outside makes its part NaN and its gradient zero."""
    import torch
    say("distill repeats", c, dtype)
    m, k = 12, 9
    z = matrix(m, c, dtype, 1)
    ids, t = teacher(m, c, k, 2)
    ids[:, 5:] = ids[:, :1]
    labels = ids[:, 0].copy()
    check(G, z, ids, t, 2.0, 0.6, labels)
    ids[3, 2], ids[7, 0], labels[5], labels[7] = c, 2 ** 31 - 1, c, -2
    loss, row, dz = check(G, z, ids, t, 2.0, 0.6, labels)
    assert torch.isnan(loss).all() and torch.isnan(row[[3, 5, 7]]).all() and (dz[7] == 0).all() and torch.isfinite(dz[:m]).all()
    check(G, z, ids, t, 2.0, 1.0)
    check(G, z, ids, t, 2.0, 0.0, labels)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", [41, 30_000])
def test_masked_and_large_logits(G, c, dtype):
    """Classes of -inf (and of the type's lowest value) have no share; logits far from zero and far apart; a confident row."""
    import torch
    say("distill masked", c, dtype)
    m, k = 8, 4
    z = matrix(m, c, dtype, 1)
    ids, t = teacher(m, c, k, 2)
    ids[:] = np.arange(k)
    z[0, k:] = -float("inf")
    z[1, k + 1::2] = torch.finfo(z.dtype).min
    z[2].add_(1e4 if dtype == "f32" else 256.0)
    z[3].sub_(1e6 if dtype == "f32" else 1024.0)
    z[4].mul_(40.0)
    t[5] = [200.0, 0.0, -200.0, 100.0]
    labels = np.zeros(m, int)
    check(G, z, ids, t, 2.0, 0.5, labels)
    # an entry, or a label, whose logit is masked: an infinite loss, a finite gradient; a row of -inf alone: NaN
    z[6, 0] = -float("inf")
    z[7] = -float("inf")
    loss, row, dz = torch.zeros(3, device="cuda"), torch.zeros(m, device="cuda"), aligned(m, c, dtype)
    G.distill(z, torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), loss, temperature=2.0, alpha=0.5,
              labels=torch.from_numpy(labels.astype(np.int32)).cuda(), row_loss=row, dlogits=dz)
    assert torch.isfinite(row[:6]).all() and torch.isposinf(row[6]).all() and torch.isnan(row[7]).all()
    assert torch.isfinite(dz[:7]).all() and torch.isnan(dz[7]).all() and (dz[0, k:] == 0).all()
    # NaN in one row stays there
    z = matrix(m, c, dtype, 1)
    z[2, c - 1] = float("nan")
    G.distill(z, torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), loss, row_loss=row, dlogits=dz)
    nan = torch.isnan(row)
    assert nan.nonzero().flatten().tolist() == [2] and torch.isnan(dz[2]).all() and torch.isfinite(dz[:2]).all() and torch.isfinite(dz[3:]).all()


def test_gradients_against_differences(G):
    """fp32 loss differences along one entry: a step of 2^-5 leaves a curvature of 2^-10 / 6 of it, rounding 2^-20 / 2^-5."""
    import torch
    m, c, k = 6, 50, 5
    z = matrix(m, c, "f32", 3)
    ids, t = teacher(m, c, k, 4)
    labels = torch.arange(m, dtype=torch.int32, device="cuda")
    args = (torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda())
    loss, dz = torch.zeros(3, device="cuda"), aligned(m, c, "f32")
    G.distill(z, *args, loss, temperature=2.0, alpha=0.6, labels=labels, dlogits=dz)
    for at in ((0, 0), (0, int(ids[0, 0])), (3, int(ids[3, 4])), (5, 49), (2, 2)):
        old, value = z[at].item(), []
        for step in (2.0 ** -5, -2.0 ** -5):
            z[at] = old + step
            G.distill(z, *args, loss, temperature=2.0, alpha=0.6, labels=labels)
            value.append(loss[0].item())
        z[at] = old
        assert (value[0] - value[1]) / 2.0 ** -4 == pytest.approx(dz[at].item(), abs=2.0 ** -12, rel=2.0 ** -10)


def test_workspace_is_guarded(G):
    import torch
    for dtype, m, c, k in (("f32", 5, 700, 4), ("bf16", 300, 41, 8), ("f32", 2, 100_000, 64)):
        need = G.distill_workspace(m, c, k, dtype)
        z = matrix(m, c, dtype, 1)
        ids, t = teacher(m, c, k, 2)
        res = []
        for fill in (0, 0xFF):
            ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
            ws[:need] = fill
            loss, row, dz = torch.zeros(3, device="cuda"), torch.zeros(m, device="cuda"), aligned(m, c, dtype)
            G.distill(z, torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), loss, row_loss=row, dlogits=dz, workspace=ws[:need])
            assert (ws[need:] == 0x5A).all()
            res.append((loss, row, dz))
        assert all(torch.equal(a, b) for a, b in zip(*res))
        with pytest.raises(G.GnnavError):
            G.distill(z, torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), loss, workspace=ws[:need - 1])


def test_argument_types(G):
    import torch
    z, ids, t, loss = (torch.zeros((4, 8), device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda"),
                       torch.zeros(3, device="cuda"))
    for bad in (lambda: G.distill(z, ids.long(), t, loss), lambda: G.distill(z, ids, t.bfloat16(), loss), lambda: G.distill(z, ids[:3], t[:3], loss),
                lambda: G.distill(z, ids, t[:, :1], loss), lambda: G.distill(z, ids, t, loss[:2]), lambda: G.distill(z, ids, t, loss, labels=ids[:, 0].long()),
                lambda: G.distill(z, ids, t, loss, dlogits=z[:2]), lambda: G.distill(z, ids, t, loss, dlogits=z.bfloat16()),
                lambda: G.distill(z, ids, t, loss, row_loss=loss), lambda: G.distill(z.half(), ids, t, loss)):
        with pytest.raises(ValueError):
            bad()
