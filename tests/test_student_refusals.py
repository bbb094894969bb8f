"""Refused calls of the gated block, top-logit and distillation entry points.

Every argument is checked before any device work, so these run without a GPU:
the device pointers are made-up addresses that no call may follow.
"""
import pytest

import paper_2404_09544_amd as G

OK, INVALID, CAPACITY = 0, 1, 4
A = 1 << 20          # a 256-byte aligned address
lib = G._lib
BIG = (1 << 31) + 5
HUGE = 1 << 50


def refused(status, want, text):
    assert status == want, (status, lib.gnnav_last_error())
    assert text in lib.gnnav_last_error(), lib.gnnav_last_error()


FFN = dict(x=A, ld_x=8, m=4, d=8, wg=A, ld_wg=16, wu=A, ld_wu=16, f=16, wd=A, ld_wd=8, o=8, dt=G.F32, act=0, y=A, ld_y=8, saved=A,
           saved_bytes=HUGE, ws=A, ws_bytes=HUGE)
COMMON = [
    (dict(dt=2), INVALID, b"dtype"), (dict(act=3), INVALID, b"act"), (dict(act=-1), INVALID, b"act"), (dict(m=-1), INVALID, b"m < 0"),
    (dict(d=0), INVALID, b"d, f or d_out"), (dict(f=0), INVALID, b"d, f or d_out"), (dict(o=-2), INVALID, b"d, f or d_out"),
    (dict(m=(1 << 28) + 1), CAPACITY, b"2^28"), (dict(f=(1 << 20) + 1), CAPACITY, b"2^20"), (dict(d=BIG), CAPACITY, b"2^20"),
    (dict(x=None), INVALID, b"NULL x"), (dict(wg=None), INVALID, b"NULL wg"), (dict(wu=None), INVALID, b"NULL wu"), (dict(wd=None), INVALID, b"NULL wd"),
    (dict(ld_x=4), INVALID, b"x rows"), (dict(ld_x=9), INVALID, b"x rows"), (dict(x=A + 4), INVALID, b"x rows"), (dict(ld_wg=12), INVALID, b"wg rows"),
    (dict(ld_wu=17), INVALID, b"wu rows"), (dict(wd=A + 8), INVALID, b"wd rows"), (dict(ld_wd=7), INVALID, b"wd rows"),
    (dict(dt=G.BF16, ld_x=12), INVALID, b"x rows"), (dict(saved_bytes=10), INVALID, b"saved of"), (dict(saved=A + 8), INVALID, b"saved must"),
    (dict(ws_bytes=10), INVALID, b"needed"), (dict(ws=A + 128), INVALID, b"256-byte"), (dict(ws=None), INVALID, b"256-byte"),
]


@pytest.mark.parametrize("change,want,text", COMMON + [(dict(y=None), INVALID, b"NULL y"), (dict(ld_y=6), INVALID, b"y rows"),
                                                       (dict(y=A + 12), INVALID, b"y rows")])
def test_gated_refusals(change, want, text):
    a = dict(FFN, **change)
    refused(lib.gnnav_gated_ffn(a["x"], a["ld_x"], a["m"], a["d"], a["wg"], a["ld_wg"], a["wu"], a["ld_wu"], a["f"], a["wd"], a["ld_wd"], a["o"], a["dt"],
                                a["act"], a["y"], a["ld_y"], a["saved"], a["saved_bytes"], a["ws"], a["ws_bytes"], None), want, text)


@pytest.mark.parametrize("change,want,text", COMMON + [
    (dict(y=None), INVALID, b"NULL dy"), (dict(ld_y=6), INVALID, b"dy rows"), (dict(dx=A + 4), INVALID, b"dx rows"), (dict(dwg=A + 4), INVALID, b"dwg rows"),
    (dict(dwu=A + 4), INVALID, b"dwu rows"), (dict(dwd=A + 4), INVALID, b"dwd rows"), (dict(saved=None), INVALID, b"saved must")])
def test_gated_backward_refusals(change, want, text):
    a = dict(FFN, dx=A, dwg=A, dwu=A, dwd=A, **change) if not any(n in change for n in ("dx", "dwg", "dwu", "dwd")) else dict(
        FFN, **dict(dict(dx=A, dwg=A, dwu=A, dwd=A), **change))
    refused(lib.gnnav_gated_ffn_backward(a["x"], a["ld_x"], a["m"], a["d"], a["wg"], a["ld_wg"], a["wu"], a["ld_wu"], a["f"], a["wd"], a["ld_wd"], a["o"],
                                         a["dt"], a["act"], a["y"], a["ld_y"], a["saved"], a["saved_bytes"], a["dx"], 8, a["dwg"], 16, a["dwu"], 16,
                                         a["dwd"], 8, a["ws"], a["ws_bytes"], None), want, text)


P = {n: A * (i + 1) for i, n in enumerate(("x", "wg", "wu", "wd", "y", "saved", "ws", "dx", "dwg", "dwu", "dwd"))}


@pytest.mark.parametrize("out,other", [("y", "x"), ("y", "wd"), ("y", "wg")])
def test_gated_refuses_an_output_in_the_place_of_an_input(out, other):
    a = dict(FFN, **dict(P, **{out: P[other]}))
    refused(lib.gnnav_gated_ffn(a["x"], 8, 4, 8, a["wg"], 16, a["wu"], 16, 16, a["wd"], 8, 8, G.F32, 0, a["y"], 8, a["saved"], HUGE, a["ws"], HUGE, None),
            INVALID, b"in the place")


@pytest.mark.parametrize("out,other", [("dx", "y"), ("dx", "x"), ("dwg", "wg"), ("dwu", "wu"), ("dwd", "wd"), ("dwu", "dwg"), ("dwd", "dx")])
def test_gated_backward_refuses_an_output_in_the_place_of_another_operand(out, other):
    a = dict(FFN, **dict(P, **{out: P[other]}))
    refused(lib.gnnav_gated_ffn_backward(a["x"], 8, 4, 8, a["wg"], 16, a["wu"], 16, 16, a["wd"], 8, 8, G.F32, 0, a["y"], 8, a["saved"], HUGE, a["dx"], 8,
                                         a["dwg"], 16, a["dwu"], 16, a["dwd"], 8, a["ws"], HUGE, None), INVALID, b"in the place")



@pytest.mark.parametrize("saved", ["x", "wg", "wu", "wd", "y"])
def test_gated_refuses_what_is_saved_in_the_place_of_an_operand(saved):
    a = dict(FFN, **dict(P, saved=P[saved]))
    refused(lib.gnnav_gated_ffn(a["x"], 8, 4, 8, a["wg"], 16, a["wu"], 16, 16, a["wd"], 8, 8, G.F32, 0, a["y"], 8, a["saved"], HUGE, a["ws"], HUGE, None),
            INVALID, b"in the place")


@pytest.mark.parametrize("out", ["dx", "dwg", "dwu", "dwd"])
def test_gated_backward_refuses_an_output_in_the_place_of_what_was_saved(out):
    a = dict(FFN, **dict(P, **{out: P["saved"]}))
    refused(lib.gnnav_gated_ffn_backward(a["x"], 8, 4, 8, a["wg"], 16, a["wu"], 16, 16, a["wd"], 8, 8, G.F32, 0, a["y"], 8, a["saved"], HUGE, a["dx"], 8,
                                         a["dwg"], 16, a["dwu"], 16, a["dwd"], 8, a["ws"], HUGE, None), INVALID, b"in the place")


TOP = dict(z=A, ld=8, m=3, c=8, dt=G.F32, k=2, values=A, ids=A, ws=A, ws_bytes=HUGE)


@pytest.mark.parametrize("change,want,text", [
    (dict(dt=5), INVALID, b"dtype"), (dict(m=-1), INVALID, b"m < 0"), (dict(c=0), INVALID, b"n_classes"), (dict(k=0), INVALID, b"k outside"),
    (dict(k=257), INVALID, b"k outside"), (dict(m=BIG), CAPACITY, b"int32"), (dict(c=BIG), CAPACITY, b"int32"), (dict(z=None), INVALID, b"NULL logits"),
    (dict(ld=7), INVALID, b"logits rows"), (dict(z=A + 4), INVALID, b"logits rows"), (dict(values=None), INVALID, b"NULL values"),
    (dict(ids=None), INVALID, b"NULL values"), (dict(c=100_000, ld=100_000, ws_bytes=8), INVALID, b"needed"),
    (dict(c=100_000, ld=100_000, ws=A + 16), INVALID, b"256-byte"),
])
def test_top_logits_refusals(change, want, text):
    a = dict(TOP, **change)
    refused(lib.gnnav_top_logits(a["z"], a["ld"], a["m"], a["c"], a["dt"], a["k"], a["values"], a["ids"], a["ws"], a["ws_bytes"], None), want, text)


DISTILL = dict(z=A, ld=8, m=3, c=8, dt=G.F32, ids=A, t=A, k=2, temp=1.0, alpha=0.5, labels=A, loss=A, dz=None, ld_d=8, ws=A, ws_bytes=HUGE)


@pytest.mark.parametrize("change,want,text", [
    (dict(dt=5), INVALID, b"dtype"), (dict(m=-1), INVALID, b"m < 0"), (dict(c=0), INVALID, b"n_classes"), (dict(k=0), INVALID, b"k outside"),
    (dict(k=257), INVALID, b"k outside"), (dict(k=300, alpha=0.0), INVALID, b"k outside"), (dict(k=-1, alpha=0.0), INVALID, b"k outside"),
    (dict(m=BIG), CAPACITY, b"int32"), (dict(c=BIG), CAPACITY, b"int32"), (dict(z=None), INVALID, b"NULL logits"), (dict(ld=6), INVALID, b"logits rows"),
    (dict(ids=None), INVALID, b"NULL ids"), (dict(t=None), INVALID, b"NULL ids"), (dict(loss=None), INVALID, b"NULL loss"),
    (dict(temp=0.0), INVALID, b"temperature"), (dict(temp=-1.0), INVALID, b"temperature"), (dict(temp=float("nan")), INVALID, b"temperature"),
    (dict(temp=float("inf")), INVALID, b"temperature"), (dict(temp=1e-40), INVALID, b"temperature"), (dict(alpha=-0.1), INVALID, b"alpha"),
    (dict(alpha=1.5), INVALID, b"alpha"), (dict(alpha=float("nan")), INVALID, b"alpha"), (dict(dz=A + 4), INVALID, b"dlogits rows"),
    (dict(dz=A + 4096, ld_d=4), INVALID, b"dlogits rows"), (dict(dz=A, ld_d=12), INVALID, b"in place"), (dict(ws_bytes=8), INVALID, b"needed"),
    (dict(ws=A + 64), INVALID, b"256-byte"),
])
def test_distill_refusals(change, want, text):
    a = dict(DISTILL, **change)
    refused(lib.gnnav_distill(a["z"], a["ld"], a["m"], a["c"], a["dt"], a["ids"], a["t"], a["k"], a["temp"], a["alpha"], a["labels"], -1, a["loss"], None,
                              a["dz"], a["ld_d"], a["ws"], a["ws_bytes"], None), want, text)


@pytest.mark.parametrize("temp", [3.5e-39, 4.2e-39, 1e-30, 1e-19, 2e19, 3e38])
def test_distill_refuses_temperatures_past_fp32(temp):
    """log2(e) / T or T^2 is infinite, which zeros would meet, or T^2 is none, which infinite logits / T would."""
    a = dict(DISTILL, temp=temp, dz=A + 4096)
    refused(lib.gnnav_distill(a["z"], a["ld"], a["m"], a["c"], a["dt"], a["ids"], a["t"], a["k"], a["temp"], a["alpha"], a["labels"], -1, a["loss"], None,
                              a["dz"], a["ld_d"], a["ws"], a["ws_bytes"], None), INVALID, b"temperature")


def test_workspace_sizes():
    """Host only: -1 for bad arguments, an answer for every size that a call takes."""
    for bad in [(-1, 8, 8, 8, 0), (4, 0, 8, 8, 0), (4, 8, 0, 8, 0), (4, 8, 8, 0, 0), (4, 8, 8, 8, 2), ((1 << 28) + 1, 8, 8, 8, 0), (4, 8, (1 << 20) + 1, 8, 0)]:
        assert lib.gnnav_gated_ffn_workspace(*bad) == -1 and lib.gnnav_gated_ffn_backward_workspace(*bad) == -1
    for bad in [(-1, 8, 0), (4, 0, 0), (4, 8, 3), ((1 << 28) + 1, 8, 0)]:
        assert lib.gnnav_gated_ffn_saved(*bad) == -1
    for bad in [(-1, 8, 2, 0), (4, 0, 2, 0), (4, 8, 0, 0), (4, 8, 257, 0), (4, 8, 2, 4), (BIG, 8, 2, 0), (4, BIG, 2, 0)]:
        assert lib.gnnav_top_logits_workspace(*bad) == -1
    for bad in [(-1, 8, 2, 0), (4, 0, 2, 0), (4, 8, -1, 0), (4, 8, 257, 0), (4, 8, 2, 4), (BIG, 8, 2, 0), (4, BIG, 2, 0)]:
        assert lib.gnnav_distill_workspace(*bad) == -1
    for call in (lambda: G.gated_ffn_workspace(4, 0, 8, 8, "f32"), lambda: G.gated_ffn_backward_workspace(4, 0, 8, 8, "f32"),
                 lambda: G.gated_ffn_saved(-1, 8, "f32"), lambda: G.top_logits_workspace(4, 8, 0, "f32"), lambda: G.distill_workspace(4, 0, 2, "bf16")):
        with pytest.raises(G.GnnavError):
            call()
    top = 2 ** 31 - 1
    for dt in (0, 1):
        for m, d, f, o in [(0, 1, 1, 1), (1 << 28, 8, 8, 8), (1, 1 << 20, 1 << 20, 1 << 20), (1 << 28, 1 << 20, 1 << 20, 1 << 20)]:
            for query in (lib.gnnav_gated_ffn_workspace, lib.gnnav_gated_ffn_backward_workspace):
                assert 0 <= query(m, d, f, o, dt) < 1 << 62
            assert lib.gnnav_gated_ffn_saved(m, f, dt) == m * ((f + 7) // 8 * 8) * (2 if dt else 14)
        for m, c in [(0, 1), (top, 41), (1, top), (top, top), (64, top)]:
            assert lib.gnnav_top_logits_workspace(m, c, 256, dt) >= 0 and lib.gnnav_distill_workspace(m, c, 256, dt) > 0


def test_empty_calls_do_nothing():
    """Calls without rows succeed without touching a device."""
    assert lib.gnnav_gated_ffn(None, 8, 0, 8, A, 16, A, 16, 16, A, 8, 8, G.F32, 0, None, 8, None, 0, None, 0, None) == OK
    assert lib.gnnav_top_logits(None, 8, 0, 8, G.F32, 2, None, None, None, 0, None) == OK


def test_binding_refuses_host_tensors():
    import torch
    t, ids, loss, saved = torch.zeros(8, 8), torch.zeros(8, 2, dtype=torch.int32), torch.zeros(3), torch.zeros(9000, dtype=torch.uint8)
    for call in (lambda: G.gated_ffn(t, t, t, t, t), lambda: G.gated_ffn_backward(t, t, t, t, t, saved), lambda: G.top_logits(t, t[:, :2], ids),
                 lambda: G.distill(t, ids, t[:, :2], loss)):
        with pytest.raises(ValueError):
            call()


def test_binding_refuses_ids_without_logits():
    import torch
    with pytest.raises(ValueError):
        G._kept(torch.zeros(8, 2, dtype=torch.int32), None, "teacher", 0, 8)
