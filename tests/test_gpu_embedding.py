"""Lookup in a trained table and its gradient, against plain numpy in 64 bits.

The lookup is one fp32 product and one rounding per element: exact.  The
gradient is a sum of k rows in fp32 in any order, times the scale, rounded to the
row's type: off by at most (k + 2) 2^-24 of the sum of magnitudes, and
half a step of the type (fp32 2^-24, bf16 2^-8).
"""
import numpy as np
import pytest

from test_gpu_parity import G, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def torch_type(dtype):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


def matrix(rows, d, dtype, seed, extra=0, pad=float("nan")):
    """A [rows, d] device view in a wider buffer whose padding holds NaN."""
    import torch
    per = 16 // (2 if dtype == "bf16" else 4)
    ld = (d + per - 1) // per * per + extra * per
    gen = torch.Generator().manual_seed(seed)
    t = torch.full((rows, ld), pad, dtype=torch.float32)
    t[:, :d] = torch.randn((rows, d), generator=gen)
    return t.to(torch_type(dtype)).cuda()[:, :d]


def f64(t):
    return t.detach().double().cpu().numpy()


def wide(t):
    """The whole buffer that a view's rows lie in."""
    return t.as_strided((t.shape[0], t.stride(0)), (t.stride(0), 1))


def unit_end(d, dtype):
    per = 16 // (2 if dtype == "bf16" else 4)
    return (d + per - 1) // per * per


LOOKUPS = [(1, 1, 1), (1, 3, 5), (5, 7, 4), (63, 100, 17), (257, 50, 64), (1000, 31, 100), (300, 200, 256),
           (513, 129, 602), (40, 9, 1030), (70_001, 5000, 32)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,rows,d", LOOKUPS)
@pytest.mark.parametrize("scale", [1.0, 0.3])
def test_lookup_is_exact(G, n, rows, d, dtype, scale):
    import torch
    say("lookup", n, rows, d, dtype, scale)
    table = matrix(rows, d, dtype, n + d, extra=1)
    out = torch.full((n + 2, unit_end(d, dtype) + unit_end(1, dtype)), -7.0, dtype=torch_type(dtype), device="cuda")[:, :d]
    rng = np.random.default_rng(n)
    ids = rng.integers(0, rows, n).astype(np.int32)
    if n > 4:
        ids[1], ids[2], ids[3] = -1, rows, np.iinfo(np.int32).max
    G.embedding(table, torch.from_numpy(ids).cuda(), out, scale=scale)
    G.sync()
    t = table.float().cpu()
    want = torch.zeros((n, d))
    ok = torch.from_numpy((ids >= 0) & (ids < rows))
    want[ok] = t[torch.from_numpy(ids[ok.numpy()]).long()] * torch.tensor(scale, dtype=torch.float32)
    assert torch.equal(out[:n].cpu(), want.to(torch_type(dtype)))
    w = wide(out).float().cpu()
    assert (w[:n, d:unit_end(d, dtype)] == 0).all()          # up to the next 16 bytes: zeros
    assert (w[:, unit_end(d, dtype):] == -7).all() and (w[n:] == -7).all()


def test_lookup_reads_its_count_on_the_device(G):
    import torch
    table, ids = matrix(20, 8, "f32", 1), torch.arange(16, dtype=torch.int32, device="cuda") % 20
    for count in (0, 5, 16, 99, -3):
        out = torch.full((16, 8), -7.0, device="cuda")
        G.embedding(table, ids, out, n_ids_dev=torch.tensor([count], dtype=torch.int32, device="cuda"))
        k = min(16, max(0, count))
        assert torch.equal(out[:k], table[:k]) and (out[k:] == -7).all()


def test_lookup_offsets_past_32_bits(G):
    """Rows at byte offsets beyond 4 GiB of a wide table."""
    import torch
    table = torch.zeros((70_000, 16_384), dtype=torch.float32, device="cuda")   # 4.6 GB
    table[:, 0] = torch.arange(70_000, device="cuda", dtype=torch.float32)
    table[:, 16_383] = table[:, 0]
    ids = torch.tensor([69_999, 0, 65_537, 32_768], dtype=torch.int32, device="cuda")
    out = torch.zeros((4, 16_384), device="cuda")
    G.embedding(table, ids, out, scale=2.0)
    assert out[:, 0].tolist() == [2.0 * i for i in ids.tolist()] and torch.equal(out[:, 0], out[:, 16_383])
    grad = torch.zeros_like(table)
    G.embedding_backward(out, ids, grad, scale=0.5)
    assert torch.equal(grad[ids.long(), 16_383], table[ids.long(), 0]) and grad.sum(dtype=torch.float64) == table[ids.long()].sum(dtype=torch.float64)


def make_ids(kind, n, rows, rng):
    if kind == "uniform":
        return rng.integers(0, rows, n).astype(np.int32)
    if kind == "same":
        return np.full(n, rows // 2, np.int32)
    if kind == "few":
        return rng.integers(0, min(rows, 3), n).astype(np.int32)
    if kind == "skew":
        return np.minimum(np.exp(rng.random(n) * np.log(rows + 1.0)) - 1, rows - 1).astype(np.int32)
    if kind == "runs":      # ids in order, runs of 64 and 63 and 65
        return np.minimum(np.repeat(np.arange(rows), [63 + i % 3 for i in range(rows)])[:n], rows - 1).astype(np.int32)
    assert kind == "bad"
    ids = rng.integers(-2, rows + 3, n)
    return ids.astype(np.int32)


GRADS = [("uniform", 1, 1, 1), ("uniform", 1, 9, 8), ("uniform", 300, 1000, 17), ("same", 700, 5, 64),
         ("few", 1000, 40_000, 100), ("bad", 4096, 777, 33), ("skew", 4096, 70_000, 4), ("same", 4096, 3, 300),
         ("uniform", 4097, 3000, 64), ("same", 4097, 1, 8), ("same", 10_007, 9, 100), ("few", 9000, 3, 602),
         ("bad", 6000, 1000, 5), ("bad", 5000, 1, 12), ("runs", 6400, 110, 32), ("skew", 50_000, 20_000, 128),
         ("skew", 70_000, 300, 1030), ("uniform", 30_000, 1_500_000, 8), ("uniform", 20_001, 1025, 48),
         ("uniform", 8000, 1023, 260), ("uniform", 8000, 1024, 20), ("skew", 1_200_000, 5000, 4)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,n,rows,d", GRADS)
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(G, kind, n, rows, d, dtype, accumulate):
    import torch
    say("embedding gradient", kind, n, rows, d, dtype, accumulate)
    rng = np.random.default_rng(n + rows + d)
    ids = make_ids(kind, n, rows, rng)
    dout = matrix(n, d, dtype, n + d, extra=1)
    grads = []
    for _ in range(2):
        g = matrix(rows, d, dtype, d, extra=1, pad=-7.0)     # what was there
        old = f64(g) if accumulate else np.zeros((rows, d))
        G.embedding_backward(dout, torch.from_numpy(ids).cuda(), g, scale=0.75, accumulate=accumulate)
        grads.append(g)
    G.sync()
    x = f64(dout)
    ok = (ids >= 0) & (ids < rows)
    want, mags, count = np.zeros((rows, d)), np.zeros((rows, d)), np.zeros(rows)
    np.add.at(want, ids[ok], x[ok])
    np.add.at(mags, ids[ok], np.abs(x[ok]))
    np.add.at(count, ids[ok], 1)
    want = 0.75 * want + old
    got = f64(grads[0])
    tol = (count + 4)[:, None] * 2.0 ** -24 * (0.75 * mags + np.abs(old)) + HALF_STEP[dtype] * np.abs(want)
    assert (np.abs(got - want) <= tol).all(), float(np.max(np.abs(got - want) - tol))
    assert torch.equal(grads[0].contiguous(), grads[1].contiguous())              # the same bits on every run
    w = wide(grads[0]).float().cpu()
    end = unit_end(d, dtype)
    assert (w[:, end:] == -7).all()
    if accumulate:
        same = torch.from_numpy(count == 0)
        assert torch.equal(grads[0].cpu()[same], matrix(rows, d, dtype, d, extra=1).cpu()[same])
    else:
        assert (w[:, d:end] == 0).all()


@pytest.mark.parametrize("n", [900, 9000])
def test_gradient_reads_its_count_on_the_device(G, n):
    """Rows behind the count, NaN among them, take no part; a count of zero gives zeros."""
    import torch
    rng = np.random.default_rng(n)
    ids = rng.integers(0, 500, n).astype(np.int32)
    idd = torch.from_numpy(ids).cuda()
    for count in (0, 1, n // 3, n - 1, n, n + 7, -1):
        k = min(n, max(0, count))
        dout = matrix(n, 20, "f32", 3)
        dout[k:] = float("nan")
        g = torch.full((500, 20), 5.0, device="cuda")
        G.embedding_backward(dout, idd, g, n_ids_dev=torch.tensor([count], dtype=torch.int32, device="cuda"))
        short = torch.full((500, 20), 5.0, device="cuda")
        if k:
            G.embedding_backward(dout[:k], idd[:k], short)
        else:
            short.zero_()
        # another count takes another cut of the sums: equal within their rounding
        assert torch.allclose(g, short, rtol=1e-5, atol=1e-5), count


def test_gradient_keeps_infinities_and_nan_to_their_rows(G):
    import torch
    for n in (200, 6000):
        ids = torch.arange(n, dtype=torch.int32, device="cuda") % 50
        dout = torch.ones((n, 12), device="cuda")
        dout[3, 1], dout[104, 2], dout[57, 5] = float("inf"), float("nan"), -float("inf")
        ids[100:150] = -1
        g = torch.zeros((50, 12), device="cuda")
        G.embedding_backward(dout, ids, g)
        bad = ~torch.isfinite(g)
        assert bad.nonzero().tolist() == [[3, 1], [7, 5]]     # row 104's id is left out


def test_gradient_against_differences(G):
    """d/dtable of sum(out * c) for out = scale * table[ids]: linear, so the difference is exact up to rounding."""
    import torch
    table, ids = matrix(40, 16, "f32", 5), torch.randint(0, 40, (200,), dtype=torch.int32, device="cuda")
    c = matrix(200, 16, "f32", 6)
    g = torch.zeros((40, 16), device="cuda")
    G.embedding_backward(c, ids, g, scale=1.5)
    out = torch.zeros((200, 16), device="cuda")
    for r, k in ((int(ids[0]), 3), (int(ids[7]), 15), (int(ids[199]), 0)):
        value = []
        for step in (2.0, -2.0):
            t = table.clone()
            t[r, k] += step
            G.embedding(t, ids, out, scale=1.5)
            value.append((out.double() * c.double()).sum().item())
        assert (value[0] - value[1]) / 4.0 == pytest.approx(g[r, k].item(), rel=1e-4, abs=1e-4)


def test_workspace_is_checked_and_guarded(G):
    """A workspace of exactly the size asked for, canaries behind it."""
    import torch
    n, rows, d = 20_000, 3000, 72
    for dtype in ("f32", "bf16"):
        need = G.embedding_backward_workspace(n, rows, d, dtype)
        ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        ids = torch.randint(0, rows, (n,), dtype=torch.int32, device="cuda")
        dout = matrix(n, d, dtype, 2)
        a, b = (torch.zeros((rows, d), dtype=torch_type(dtype), device="cuda") for _ in range(2))
        G.embedding_backward(dout, ids, a, workspace=ws[:need])
        G.embedding_backward(dout, ids, b)
        assert torch.equal(a, b) and (ws[need:] == 0xA5).all()
        with pytest.raises(G.GnnavError):
            G.embedding_backward(dout, ids, a, workspace=ws[:need - 1])


def test_argument_types(G):
    import torch
    t, ids = torch.zeros((4, 8), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (lambda: G.embedding(t, ids.long(), t), lambda: G.embedding(t, ids, t[:2]),
                lambda: G.embedding(t, ids, t.bfloat16()), lambda: G.embedding(t.double(), ids, t.double()),
                lambda: G.embedding(t.t(), ids, t), lambda: G.embedding(t[:, :4], ids, t),
                lambda: G.embedding_backward(t[:3], ids, t), lambda: G.embedding(t, ids[::2], t),
                lambda: G.embedding(t, ids, t, n_ids_dev=torch.zeros(1, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(G.GnnavError):
        G.embedding(torch.zeros((4, 9), device="cuda"), ids, torch.zeros((4, 9), device="cuda"))   # rows off 16 bytes
