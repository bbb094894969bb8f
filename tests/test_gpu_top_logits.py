"""The k largest logits of each row, against a stable sort: values and classes are exact."""
import numpy as np
import pytest

from test_gpu_embedding import matrix, torch_type
from test_gpu_parity import G, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu


def reference(z, k):
    """numpy [m, v] in fp32: NaN first, then falling, equal ones by class; -inf and -1 past the classes."""
    m, v = z.shape
    values, ids = np.full((m, k), -np.inf, np.float32), np.full((m, k), -1, np.int32)
    bits = np.ascontiguousarray(z, np.float32).view(np.int32).astype(np.int64)
    key = np.where(np.isnan(z), 1 << 40, np.where(bits < 0, -(bits & 0x7fffffff), bits))
    order = np.argsort(-key, axis=1, kind="stable")[:, :k]
    values[:, :order.shape[1]], ids[:, :order.shape[1]] = np.take_along_axis(z, order, 1), order
    return values, ids


def check(G, logits, k, workspace=None):
    import torch
    m = logits.shape[0]
    values = torch.full((m + 1, k), -7.0, device="cuda")
    ids = torch.full((m + 1, k), -7, dtype=torch.int32, device="cuda")
    G.top_logits(logits, values[:m], ids[:m], workspace=workspace)
    G.sync()
    want, at = reference(logits.float().cpu().numpy(), k)
    assert np.array_equal(ids[:m].cpu().numpy(), at)
    assert np.array_equal(values[:m].cpu().numpy(), want, equal_nan=True)
    assert (values[m:] == -7).all() and (ids[m:] == -7).all()


SHAPES = [(1, 1, 1), (1, 2, 5), (3, 7, 7), (5, 41, 8), (70, 41, 1), (300, 41, 41), (9, 64, 64), (4, 65, 64), (6, 200, 100),
          (3, 500, 129), (2, 511, 256), (8, 513, 256), (1, 5_000, 64), (2, 20_001, 33), (5, 70_003, 128), (130, 3_001, 50),
          (1, 169_000, 256), (600, 1_000, 16), (33, 12, 12), (2_000, 17, 3),
          (9_000, 9, 8), (43_000, 41, 7), (30_000, 64, 2), (70_000, 70, 13), (110_000, 200, 15), (3_000, 100, 90)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v,k", SHAPES)
def test_random_logits(G, m, v, k, dtype):
    """bf16 logits hold many equal ones."""
    say("top", m, v, k, dtype)
    check(G, matrix(m, v, dtype, m + v + k, extra=1), k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v,k", [(41, 8), (41, 41), (3_000, 20), (9_001, 64), (30_000, 200)])
def test_orders(G, v, k, dtype):
    """Rising, falling, all equal, two values, few distinct ones, one large value at the end."""
    import torch
    say("top orders", v, k, dtype)
    z = matrix(8, v, dtype, 3)
    n = torch.arange(v, device="cuda", dtype=torch.float32)
    for i, row in enumerate((n, -n, 0 * n + 2.5, (n % 2), -(n % 7), (n == v - 1).float(), torch.where(n % 3 == 0, -torch.inf, n % 11),
                             torch.where(n < v - 3, -torch.inf, n))):
        z[i].copy_(row)
    check(G, z, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v,more", [(50, 0), (100, 0), (5_000, 0), (20, 20_000)])
def test_special_values(G, v, more, dtype):
    """NaN first, infinities, zeros of either sign by class, rows of -inf alone."""
    import torch
    say("top special", v, more, dtype)
    z = matrix(6 + more, v, dtype, 4)
    z[0, 7], z[0, 3], z[0, 13] = float("nan"), float("nan"), float("inf")
    z[1] = -float("inf")
    z[2].clamp_(max=0.0)
    z[2, ::2] = -0.0
    z[2, 1::4] = 0.0
    z[3] = float("nan")
    z[4, 5:] = -float("inf")
    z[5].mul_(1e-38 if dtype == "bf16" else 1e-40)      # subnormal ones keep their order
    check(G, z, 10 if not more else 6)


def test_workspace_is_guarded(G):
    import torch
    for m, v, k in ((1, 169_000, 64), (3, 40_000, 7), (5, 30, 4)):
        need = G.top_logits_workspace(m, v, k, "f32")
        ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
        z = matrix(m, v, "f32", 5)
        check(G, z, k, workspace=ws[:need])
        assert (ws[need:] == 0xFF).all()
        if need:
            with pytest.raises(G.GnnavError):
                check(G, z, k, workspace=ws[:need - 1])


def test_argument_types(G):
    import torch
    z, values, ids = torch.zeros((4, 8), device="cuda"), torch.zeros((4, 2), device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    for bad in (lambda: G.top_logits(z, values, ids.long()), lambda: G.top_logits(z, values[:3], ids[:3]),
                lambda: G.top_logits(z, values, ids[:, :1]), lambda: G.top_logits(z.half(), values, ids),
                lambda: G.top_logits(z, values.bfloat16(), ids)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(G.GnnavError):
        G.top_logits(z, torch.zeros((4, 257), device="cuda"), torch.zeros((4, 257), dtype=torch.int32, device="cuda"))
    with pytest.raises(G.GnnavError):
        G.top_logits(torch.zeros((4, 9), device="cuda"), values, ids)      # rows off the 16-byte boundaries
    G.top_logits(z[:0], values[:0], ids[:0])
