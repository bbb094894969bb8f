"""The gated feed-forward kernels' planner: every tile of every launch is taken by a block that tests/test_gpu_gated_tiles.py runs,
and what those results are allowed to be off by tells a lost part of an operand.  No GPU: the planner is plain C++."""
import os
import shutil
import subprocess

import pytest

from conftest import ROOT
from gated_tiles import TILES, expected

LARGE, WIDE, MEDIUM, SMALL = range(4)
H = {"bf16": {LARGE: (128, 256, 1), MEDIUM: (64, 128, 3), SMALL: (32, 64, 0)}, "f32": {WIDE: (64, 128, 2), SMALL: (32, 64, 0)}}   # columns, rows, places a unit
DH = {"bf16": (LARGE, MEDIUM, SMALL), "f32": (WIDE, SMALL)}
OUT = {"bf16": (LARGE, WIDE, MEDIUM, SMALL), "f32": (WIDE, MEDIUM, SMALL)}


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path_factory.mktemp("plan") / "plan")
    r = subprocess.run([cxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2404_09544_amd", "csrc"),
                        os.path.join(ROOT, "tests", "gated_plan", "plan.cpp"), "-o", exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    calls = "".join(f"{int(dtype == 'bf16')} {m} {d} {f} {o}\n" for dtype, m, d, f, o, _, _ in TILES)
    r = subprocess.run([exe], input=calls, capture_output=True, text=True, timeout=60)
    return [tuple(int(v) for v in line.split()) for line in r.stdout.splitlines()]


def test_blocks_take_the_tiles_that_they_stand_for(plans):
    import paper_2404_09544_amd as G
    assert len(plans) == len(TILES)
    for (dtype, m, d, f, o, _, want), got in zip(TILES, plans):
        assert got[:8] == want, (dtype, m, d, f, o, got)
        # (the planner in the library is this one)
        assert got[8:] == (G.gated_ffn_workspace(m, d, f, o, dtype), G.gated_ffn_backward_workspace(m, d, f, o, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_tile_is_taken(dtype):
    """Each with sums that are cut and whole; h's larger ones, and fp32's of da and db, by workgroups that take several in turn too;
    their activations all of them."""
    mine = [(t[1], t[3], t[5], t[6]) for t in TILES if t[0] == dtype]
    for tile, (columns, rows, each) in H[dtype].items():
        took = [(m, f, acts) for m, f, acts, p in mine if p[0] == tile]
        assert {a for _, _, acts in took for a in acts} == {"silu", "gelu", "relu"}, tile
        if each:
            assert any(-(-m // rows) * -(-f // columns) > 256 * each for m, f, _ in took), tile
    for tile in DH[dtype]:
        assert {a for _, _, acts, p in mine if p[3] == tile for a in acts} == {"silu", "gelu", "relu"}, tile
    if dtype == "f32":
        assert any(p[3] == WIDE and -(-m // 128) * -(-f // 128) > 512 for m, f, _, p in mine)
    for tile in OUT[dtype]:
        assert {p[2] > 1 for _, _, _, p in mine if p[1] == tile} == {False, True}, tile
        for at in (5, 6, 7):
            assert {p[at] > 1 for _, _, _, p in mine if p[4] == tile} == {False, True}, (tile, at)


def parts(v, n):
    """A matrix as the sum of its first n bf16 parts."""
    import torch
    out, rest = torch.zeros_like(v), v.clone()
    for _ in range(n):
        p = rest.float().bfloat16().double()
        out, rest = out + p, rest - p
    return out


@pytest.mark.parametrize("m,d,f,o", [(400, 602, 512, 41), (700, 100, 256, 256)])
def test_a_lost_part_shows(m, d, f, o):
    """Two parts of any one fp32 operand of a product instead of three: some result is off by more than the norms allow."""
    import torch
    gen = torch.Generator().manual_seed(5)
    x, dy, wg, wu, wd = (torch.randn(s, generator=gen) * c for s, c in (((m, d), 1), ((m, o), 1), ((d, f), d ** -0.5), ((d, f), d ** -0.5), ((f, o), f ** -0.5)))
    want = expected(x, wg, wu, wd, dy, "silu", "f32")
    x, wg, wu, wd, dy = (v.double() for v in (x, wg, wu, wd, dy))

    def run(lost=""):
        two = lambda name, v: parts(v, 2) if name == lost else v   # noqa: E731
        a, b = two("x", x) @ two("wg", wg), two("x", x) @ two("wu", wu)
        g = torch.sigmoid(a)
        h = a * g * b
        dh = two("dy", dy) @ two("wd back", wd).t()
        da, db = dh * b * (g + a * g * (1 - g)), dh * a * g
        return dict(y=two("h", h) @ two("wd", wd), dx=two("da", da) @ two("wg back", wg).t() + two("db", db) @ two("wu back", wu).t(),
                    dwg=two("x back", x).t() @ two("da back", da), dwu=two("x back", x).t() @ two("db back", db),
                    dwd=two("h back", h).t() @ two("dy back", dy))

    def worst(got):
        return max(((got[n] - w.value).norm() / w.square.sum().sqrt()).item() for n, w in want.items())
    assert worst(run()) < 1e-3
    for lost in ("x", "wg", "wu", "dy", "wd", "h", "da", "db", "wd back", "wg back", "wu back", "x back", "da back", "db back", "h back", "dy back"):
        assert worst(run(lost)) > 1.0, lost
