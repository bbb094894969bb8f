"""The global gradient norm, clipping and the clipped SGD step, against numpy in 64 bits.

norm: squares and sums in 64 bits, rounded once: half a step of fp32, 2^-24,
and 2^-50 for the sums.  The factor c is a rounding of max_norm / norm, each
element one more product rounded to its type: fp32 2 * 2^-24, bf16 2^-24 + 2^-8.
The step: lr * c two roundings, the product and the difference one each.
"""
import numpy as np
import pytest

from test_gpu_embedding import HALF_STEP, f64, torch_type
from test_gpu_parity import G, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu


def tensors(sizes, dtype, seed, std=1.0, offset=0):
    """Tensors cut from one buffer; offset: elements by which each start leaves a 16-byte boundary."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for k, n in enumerate(sizes):
        shift = (offset * (k + 1)) % 8
        t = torch.empty(n + 16, dtype=torch_type(dtype), device="cuda").normal_(0.0, std, generator=gen)
        out.append(t[shift:shift + n])
    return out


SIZES = [[1], [0], [], [0, 5, 0], [3, 1, 2], [16384], [16383, 16385, 7], [1204 * 256, 512 * 41],
         [100_003, 1, 50_000, 17], [(37 * k) % 501 + 1 for k in range(250)], [4_000_037]]


def reference_norm(ts):
    return float(np.sqrt(sum((f64(t) ** 2).sum() for t in ts)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s, default=0)}")
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_norm_clip_and_step(G, sizes, dtype, offset):
    import torch
    say("clip", len(sizes), sum(sizes), dtype, offset)
    half = HALF_STEP[dtype]
    g = tensors(sizes, dtype, len(sizes) + 1, offset=offset)
    ref = reference_norm(g)
    norm = torch.full((1,), -1.0, device="cuda")
    G.grad_norm(g, norm)
    assert abs(norm.item() - ref) <= (2.0 ** -24 + 2.0 ** -50) * ref + 2.0 ** -149
    for max_norm in (0.4 * ref, 2.0 * ref + 1.0, 0.0, float("inf")):
        m32 = float(np.float32(max_norm))
        c = 1.0 if ref <= m32 else m32 / ref
        # out of place, other offsets than the gradients'
        out = tensors(sizes, dtype, 5, offset=offset + 1)
        keep = [t.clone() for t in g]
        norm.fill_(-1.0)
        G.clip_grads(g, max_norm, norm, out=out)
        assert abs(norm.item() - ref) <= (2.0 ** -24 + 2.0 ** -50) * ref + 2.0 ** -149
        for t, o, k in zip(g, out, keep):
            assert torch.equal(t, k)
            want = c * f64(t)
            assert (np.abs(f64(o) - want) <= (half + 2.0 ** -23) * np.abs(want) + 2.0 ** -149).all()
        # the step, in place on weights
        w = tensors(sizes, dtype, 6, offset=offset)
        before = [f64(t) for t in w]
        G.sgd_clip_step(w, g, 0.3, max_norm, norm)
        lr = float(np.float32(0.3))
        for t, b, x in zip(w, before, g):
            step = lr * c * f64(x)
            want = b - step
            assert (np.abs(f64(t) - want) <= (half + 2.0 ** -24) * np.abs(want) + 2.0 ** -22 * np.abs(step) + 2.0 ** -149).all()
        # in place
        same = [t.clone() for t in g]
        G.clip_grads(same, max_norm, norm)
        for a, o in zip(same, out):
            assert torch.equal(a, o)


def test_squares_beyond_fp32(G):
    """Values whose squares leave fp32's range on either side."""
    import torch
    norm = torch.zeros(1, device="cuda")
    big = [torch.full((1000,), 1e30, device="cuda"), torch.full((10,), -3e33, device="cuda")]
    ref = reference_norm(big)
    G.clip_grads(big, 1.0, norm)
    assert norm.item() == pytest.approx(ref, rel=2.0 ** -23)
    assert reference_norm(big) == pytest.approx(1.0, rel=1e-6)
    tiny = [torch.full((1000,), 1e-30, device="cuda")]
    G.grad_norm(tiny, norm)
    assert norm.item() == pytest.approx(reference_norm(tiny), rel=2.0 ** -23)


def test_infinite_and_nan_norms(G):
    import torch
    norm = torch.zeros(1, device="cuda")
    g = [torch.ones(5, device="cuda"), torch.ones(70_000, device="cuda")]
    g[1][69_999] = float("inf")
    G.clip_grads(g, 1.0, norm)
    assert norm.item() == float("inf")
    assert (g[0] == 0).all() and (g[1][:69_999] == 0).all() and torch.isnan(g[1][69_999])
    g = [torch.ones(5, device="cuda"), torch.ones(7, device="cuda")]
    g[0][2] = float("nan")
    w = [torch.ones(5, device="cuda"), torch.ones(7, device="cuda")]
    G.sgd_clip_step(w, g, 0.1, 1.0, norm)
    assert torch.isnan(norm).all() and all(torch.isnan(t).all() for t in w)


def test_many_tensors_beyond_one_table(G):
    """Tensors of several launches: 1,000 of them, one far larger than the rest."""
    import torch
    sizes = [(k * 53) % 300 for k in range(999)] + [700_000]
    g = tensors(sizes, "f32", 9)
    ref = reference_norm(g)
    norms = [torch.zeros(1, device="cuda") for _ in range(2)]
    lst = G.TensorList(g)
    out = G.TensorList([torch.zeros_like(t) for t in g])
    for norm in norms:
        G.clip_grads(lst, 1.0, norm, out=out)
    assert norms[0].item() == norms[1].item() == pytest.approx(ref, rel=2.0 ** -23)
    assert reference_norm(out.tensors) == pytest.approx(1.0, rel=1e-5)


def test_lists_must_match(G):
    import torch
    norm = torch.zeros(1, device="cuda")
    a, b = torch.zeros(5, device="cuda"), torch.zeros(6, device="cuda")
    for bad in (lambda: G.clip_grads([a], 1.0, norm, out=[b]), lambda: G.sgd_clip_step([a, a], [a], 0.1, 1.0, norm),
                lambda: G.clip_grads([a], 1.0, norm, out=[a.bfloat16()]), lambda: G.TensorList([a, b.bfloat16()]),
                lambda: G.TensorList([a.double()]), lambda: G.TensorList([torch.zeros(4, 4, device="cuda").t()[:2]]),
                lambda: G.grad_norm([a], norm.double())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(G.GnnavError):
        G.clip_grads([a], -1.0, norm)
