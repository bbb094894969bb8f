"""The bounds of the cross entropy's workspace that the header states, over small and huge sizes (the query runs on the host)."""
import random

import paper_2404_09544_amd as G

MIB = 1 << 20


def most(m, v, d, dtype, grads):
    planes = 1 if dtype == "bf16" else 3
    slack = 16 * 256
    if m <= 32 or (m <= 64 and v <= 1 << 20):
        rows, width = 64, (d + 127) // 128 * 128
        return 4 * (v + 256) + (32 if m <= 32 else 256) * MIB + max(33 * MIB, 2 * rows * width * 4) * grads + 64 * rows + slack
    rows, width = (m + 255) // 256 * 256, (d + 255) // 256 * 256
    h = rows * width * 2 * planes
    parts = 128 * rows * width * 4 * grads
    w = max(896 * MIB, 256 * width * 2 * planes)
    p = max(1024 * MIB, 256 * rows * 2 * planes) * grads
    return h + parts + w + p + max((64 if grads else 512) * MIB, 56 * rows) + 56 * rows + slack


def test_stated_bounds():
    rng = random.Random(3)
    cases = [(1_500_000, 1_000_000, 16, "f32", 1), (5_000_000, 300, 16, "f32", 1), (128, 300, 1 << 20, "f32", 1),
             (64, 1 << 20, 1 << 20, "bf16", 1), (32, 2 ** 31 - 1, 8, "bf16", 1), (64, (1 << 20) + 1, 64, "f32", 0)]
    for _ in range(3000):
        cases.append((int(2 ** rng.uniform(0, 24)), int(2 ** rng.uniform(0, 30.9)), int(2 ** rng.uniform(0, 20)),
                      rng.choice(["f32", "bf16"]), rng.randint(0, 1)))
    for m, v, d, dtype, grads in cases:
        need = G.linear_xent_workspace(m, v, d, dtype, bool(grads))
        assert 0 < need <= most(m, v, d, dtype, grads), (m, v, d, dtype, grads, need)
