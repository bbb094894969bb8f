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
