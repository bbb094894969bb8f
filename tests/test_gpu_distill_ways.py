"""Distillation's edges on every way that its exponentials are had: one a logit (the teacher alone, the labels alone, both at
T = 1), two (T = 3), powers of those at T (T = 2, 4); by classes, in teams of 16 lanes to four wavefronts, and in strips.

References and tolerances are those of test_gpu_distill.py.
"""
import numpy as np
import pytest

from test_gpu_distill import aligned, check, teacher
from test_gpu_embedding import matrix
from test_gpu_parity import G, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu

WAYS = [(1.0, 1.0, False), (0.5, 1.0, False), (3.0, 1.0, True), (1.0, 0.0, True), (1.0, 0.5, True), (2.0, 0.5, True), (4.0, 0.5, True), (3.0, 0.4, True)]
CLASSES = [41, 200, 1_000, 5_000, 40_000]


def call(G, z, ids, t, temp, alpha, labels, ignore=-1):
    import torch
    m, c = z.shape
    dtype = "bf16" if z.dtype == torch.bfloat16 else "f32"
    loss, row, dz = torch.full((3,), -3.0, device="cuda"), torch.full((m,), -3.0, device="cuda"), aligned(m, c, dtype, -3.0)
    G.distill(z, torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), loss, temperature=temp, alpha=alpha,
              labels=None if labels is None else torch.from_numpy(labels.astype(np.int32)).cuda(), ignore_label=ignore, row_loss=row, dlogits=dz)
    return loss, row, dz


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", CLASSES)
@pytest.mark.parametrize("temp,alpha,with_labels", WAYS)
def test_rows_that_do_not_count_hold_anything(G, c, dtype, temp, alpha, with_labels):
    """Whatever the rows without entries and label hold, and those whose entries and labels are outside the classes: gradients of zero."""
    import torch
    say("distill uncounted", c, dtype, temp, alpha, with_labels)
    m, k = 20, 6
    ids, t = teacher(m, c, k, 2)
    labels = np.arange(m) % c if with_labels else None
    ids[::5] = -1
    if with_labels:
        labels[::5] = -100
    clean = check(G, matrix(m, c, dtype, 1), ids, t, temp, alpha, labels, ignore=-100)
    most = torch.finfo(clean[2].dtype).max
    for value in (100.0, 1e4, most, -most, float("inf"), -float("inf"), float("nan")):
        z = matrix(m, c, dtype, 1)
        z[::5] = value
        z[5, ::3] = 0.0
        loss, row, dz = call(G, z, ids, t, temp, alpha, labels, ignore=-100)
        assert torch.equal(loss, clean[0]) and torch.equal(row, clean[1][:m]) and torch.equal(dz, clean[2][:m]), value
        assert (dz[::5] == 0).all() and (row[::5] == 0).all()
    ids[3, 1] = c
    if with_labels:
        labels[3] = c
    z = matrix(m, c, dtype, 1)
    z[3] = 1e4
    loss, row, dz = call(G, z, ids, t, temp, alpha, labels, ignore=-100)
    assert torch.isnan(loss[0]) and torch.isnan(row[3]) and (dz[3] == 0).all() and torch.isfinite(dz).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", CLASSES)
@pytest.mark.parametrize("temp,alpha,with_labels", WAYS)
def test_masked_classes_beside_low_logits(G, c, dtype, temp, alpha, with_labels):
    """Long runs of classes of -inf have p = 0 however low the others are; a row of -inf alone and one with a NaN are NaN everywhere."""
    import torch
    say("distill masked runs", c, dtype, temp, alpha, with_labels)
    m, k = 9, 4
    ids, t = teacher(m, c, k, 2)
    ids[:] = np.arange(k)
    labels = np.zeros(m, int) if with_labels else None
    z = matrix(m, c, dtype, 1)
    for row, low in enumerate((50.0, 100.0, 200.0, 1e3, 1e6 if dtype == "f32" else 4096.0)):
        z[row].sub_(low)
        z[row, k:] = -float("inf")
    z[5].sub_(300.0)
    z[5, c // 2:] = -float("inf")
    z[6].sub_(300.0)
    z[6, k + 1:] = torch.finfo(z.dtype).min
    z[6, c // 2:] = -float("inf")
    z[7].sub_(500.0)
    z[7, k + 4:c - 2] = -float("inf")
    dz = check(G, z, ids, t, temp, alpha, labels)[2]
    assert (dz[:5, k:] == 0).all() and (dz[5:7, c // 2:] == 0).all()
    z[0] = -float("inf")
    z[1, c - 1] = float("nan")
    again = call(G, z, ids, t, temp, alpha, labels)[2]
    assert torch.isnan(again[:2]).all() and torch.isfinite(again[2:]).all()
