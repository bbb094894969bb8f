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


@pytest.mark.parametrize("dtype,m,d,f,o,act", [("bf16", 50_001, 256, 1_024, 256, "silu"), ("bf16", 8_193, 602, 1_024, 41, "relu"),
                                               ("f32", 30_001, 200, 700, 100, "relu"), ("f32", 2_459, 21, 5_499, 105, "gelu")])
def test_captured_and_on_a_share_of_the_units(G, dtype, m, d, f, o, act):
    """Workgroups that take tiles in turn: on a quarter of the units, captured and replayed between eager calls on other rows, the same bits."""
    import torch
    say("gated turns", dtype, m, d, f, o, act)
    gen = torch.Generator(device="cuda").manual_seed(7)
    x, dy, wg, wu, wd = (rows(*s, dtype, gen, c) for s, c in (((m, d), 1.0), ((m, o), 1.0), ((d, f), d ** -0.5), ((d, f), d ** -0.5), ((f, o), f ** -0.5)))
    others = rows(m, d, dtype, gen)
    need = max(G.gated_ffn_workspace(m, d, f, o, dtype), G.gated_ffn_backward_workspace(m, d, f, o, dtype))

    def state():
        out = dict(y=rows(m, o, dtype), dx=rows(m, d, dtype), dwg=rows(d, f, dtype), dwu=rows(d, f, dtype), dwd=rows(f, o, dtype))
        return out, saved_for(G, m, f, dtype), torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")

    def step(s, xx, stream=None):
        out, saved, ws = s
        G.gated_ffn(xx, wg, wu, wd, out["y"], act=act, saved=saved, workspace=ws, stream=stream)
        G.gated_ffn_backward(xx, wg, wu, wd, dy, saved, act=act, workspace=ws, stream=stream, **{n: v for n, v in out.items() if n != "y"})
    eager, other, quarter, captured = (state() for _ in range(4))
    step(eager, x)
    share = G.stream_create(1, 4)
    torch.cuda.synchronize()
    step(quarter, x, share)
    torch.cuda.synchronize()
    G.stream_destroy(share)
    graph, inner = torch.cuda.CUDAGraph(), x.clone()
    xin = rows(m, d, dtype, gen)
    xin.copy_(inner)
    with torch.cuda.graph(graph):
        step(captured, xin)
    for it in range(3):
        for v in captured[0].values():
            v.fill_(3.0)
        graph.replay()
        step(other, others)
        torch.cuda.synchronize()
        for n, v in eager[0].items():
            r = v.shape[0] - 1
            assert torch.equal(v[:r], captured[0][n][:r]), (it, n)
    for n, v in eager[0].items():
        assert torch.equal(v, quarter[0][n]), n
