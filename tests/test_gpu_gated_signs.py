"""ReLU's side of zero in fp32 blocks that keep what the backward pass needs: that of a's sum in 64 bits, whatever cancels.

Wd is the identity, so that y is h = relu(a) b itself (each part of h times 1): y is zero where a in 64 bits is not positive and nowhere
else.  The reference sums in 64 bits too; entries within 2^-44 of their terms' magnitudes of zero, which it cannot tell, are left out.
"""
import numpy as np
import pytest

from test_gpu_embedding import f64, matrix
from test_gpu_parity import G, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu


def offset(x, w):
    """Features far from zero, columns of weights that sum to nothing: every a cancels to some 2^-10 of its terms."""
    x.add_(1000.0)
    w.sub_(w.double().mean(dim=0, keepdim=True).float())


def ordered(x, w):
    """... the positive weights first, so that the sum is at its largest halfway."""
    offset(x, w)
    w.copy_(w.sort(dim=0, descending=True).values)


def mixed_scales(x, w):
    """Rows, and columns, of sizes from 2^-30 to 2^30."""
    import torch
    m, f = x.shape[0], w.shape[1]
    x.mul_(torch.pow(2.0, (torch.arange(m, device="cuda") * 7 % 61 - 30).float())[:, None])
    w.mul_(torch.pow(2.0, (torch.arange(f, device="cuda") * 11 % 61 - 30).float())[None])


def large_columns(x, w):
    """Columns whose a cancels in every row, beside others that do not, in rows of different sizes."""
    import torch
    d = x.shape[1]
    x[:, d // 2:d // 2 * 2].copy_(x[:, :d // 2] * (1 + 2.0 ** -12 * torch.randn((x.shape[0], d // 2), generator=torch.Generator("cuda").manual_seed(1), device="cuda")))
    w[d // 2:d // 2 * 2, ::3].copy_(-w[:d // 2, ::3])
    x[::5].mul_(2.0 ** -9)


def plain(x, w):
    """Nothing cancels but by chance."""


@pytest.mark.parametrize("make", [plain, offset, ordered, mixed_scales, large_columns], ids=lambda f: f.__name__)
@pytest.mark.parametrize("m,d,f", [(300, 512, 256), (70, 40, 136), (5, 602, 41), (33, 4096, 64), (2100, 257, 520)])
def test_sides(G, m, d, f, make):
    import torch
    say("gated sides", m, d, f, make.__name__)
    x, wg, wu = matrix(m, d, "f32", 1, 1), matrix(d, f, "f32", 2, 1), matrix(d, f, "f32", 3)
    wg.mul_(d ** -0.5)
    wu.mul_(d ** -0.5)
    make(x, wg)
    wd, y = matrix(f, f, "f32", 4), torch.zeros((m, (f + 3) // 4 * 4), device="cuda")[:, :f]
    wd.copy_(torch.eye(f))
    saved = torch.zeros(G.gated_ffn_saved(m, f, "f32"), dtype=torch.uint8, device="cuda")
    G.gated_ffn(x, wg, wu, wd, y, act="relu", saved=saved)
    G.sync()
    a, terms = f64(x) @ f64(wg), np.abs(f64(x)) @ np.abs(f64(wg))
    told = np.abs(a) > 2.0 ** -44 * terms
    wrong = told & ((f64(y) != 0) != (a > 0))
    assert told.mean() > 0.999 and not wrong.any(), (int(wrong.sum()), wrong.size)
