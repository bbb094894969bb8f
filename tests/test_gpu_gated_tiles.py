"""Blocks of every tile of the gated feed-forward kernels, both passes, entry by entry and by norm; tests/test_gated_tiles.py holds the
planner to the tiles that they stand for, gated_tiles.py derives the tolerances."""
import math

import pytest

from gated_tiles import TILES, expected
from test_gpu_embedding import torch_type, unit_end
from test_gpu_gated import saved_for
from test_gpu_parity import G, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu


def rows(m, d, dtype, gen=None, std=1.0):
    """[m, d] in a wider buffer, NaN beside it; -7 in it without a generator, with a row more."""
    import torch
    t = torch.full((m + (gen is None), unit_end(d, dtype) + unit_end(1, dtype)), -7.0 if gen is None else math.nan, dtype=torch_type(dtype), device="cuda")
    if gen is not None:
        t[:, :d] = torch.randn((m, d), generator=gen, device="cuda") * std
    return t[:, :d]


@pytest.mark.parametrize("dtype,m,d,f,o,act,plan", [(*t[:5], act, t[6]) for t in TILES for act in t[5]])
def test_both_passes(G, dtype, m, d, f, o, act, plan):
    import torch
    say("gated tiles", dtype, m, d, f, o, act, plan)
    gen = torch.Generator(device="cuda").manual_seed(m + d)
    x, dy = rows(m, d, dtype, gen), rows(m, o, dtype, gen)
    wg, wu, wd = rows(d, f, dtype, gen, d ** -0.5), rows(d, f, dtype, gen, d ** -0.5), rows(f, o, dtype, gen, f ** -0.5)
    saved = saved_for(G, m, f, dtype)
    got = dict(y=rows(m, o, dtype), dx=rows(m, d, dtype), dwg=rows(d, f, dtype), dwu=rows(d, f, dtype), dwd=rows(f, o, dtype))
    alone = rows(m, o, dtype)
    G.gated_ffn(x, wg, wu, wd, got["y"], act=act, saved=saved)
    G.gated_ffn_backward(x, wg, wu, wd, dy, saved, act=act, dx=got["dx"], dwg=got["dwg"], dwu=got["dwu"], dwd=got["dwd"])
    G.gated_ffn(x, wg, wu, wd, alone, act=act)
    G.sync()
    want = expected(x, wg, wu, wd, dy, act, dtype, (plan[2], *plan[5:]), sides=dtype == "f32")
    got["alone"], want["alone"] = alone, want["y"]
    for n, v in got.items():
        w = want[n]
        r, c = w.value.shape
        off = (v[:r].double() - w.value).abs()
        worst, by_norm = (off / w.off).max().item(), (off.norm() / w.square.sum().sqrt()).item()
        print(f"  {n}: {worst:.3f} of the entry's, {by_norm:.3f} of the norm's", flush=True)
        assert worst <= 1.0 and by_norm <= 1.0, (n, worst, by_norm)
        whole = v.as_strided((v.shape[0], v.stride(0)), (v.stride(0), 1)).float()
        end = unit_end(c, dtype)
        assert (whole[:r, c:end] == 0).all() and (whole[:, end:] == -7).all() and (whole[r:] == -7).all(), n
