"""Refused calls of the trained-table, large-class and clipping entry points.

Every argument is checked before any device work, so these run without a GPU:
the device pointers are made-up addresses that no call may follow.
"""
import ctypes as C

import pytest

import paper_2404_09544_amd as G

OK, INVALID, CAPACITY = 0, 1, 4
A = 1 << 20          # a 256-byte aligned address
lib = G._lib
BIG = (1 << 31) + 5


def refused(status, want, text):
    assert status == want, (status, lib.gnnav_last_error())
    assert text in lib.gnnav_last_error(), lib.gnnav_last_error()


EMB = dict(table=A, n_rows=10, ld=8, d=8, dt=G.F32, ids=A, n_dev=None, n=4, scale=1.0, out=A, ld_out=8)


@pytest.mark.parametrize("change,want,text", [
    (dict(dt=2), INVALID, b"dtype"), (dict(d=0), INVALID, b"d <= 0"), (dict(n=-1), INVALID, b"negative"),
    (dict(n_rows=-1), INVALID, b"negative"), (dict(n=BIG), CAPACITY, b"int32"), (dict(n_rows=BIG), CAPACITY, b"int32"),
    (dict(ids=None), INVALID, b"NULL ids"), (dict(table=None), INVALID, b"NULL table"),
    (dict(out=None), INVALID, b"NULL out"), (dict(ld=4), INVALID, b"table rows"), (dict(ld=9), INVALID, b"table rows"),
    (dict(table=A + 4), INVALID, b"table rows"), (dict(ld_out=7), INVALID, b"out rows"),
    (dict(out=A + 8), INVALID, b"out rows"), (dict(dt=G.BF16, ld=12), INVALID, b"table rows"),
])
def test_embedding_refusals(change, want, text):
    a = dict(EMB, **change)
    refused(lib.gnnav_embedding(a["table"], a["n_rows"], a["ld"], a["d"], a["dt"], a["ids"], a["n_dev"], a["n"],
                                a["scale"], a["out"], a["ld_out"], None), want, text)


BWD = dict(dout=A, ld=8, ids=A, n=4, d=8, dt=G.F32, acc=0, dtable=A, n_rows=10, ldt=8, ws=None, ws_bytes=0)


@pytest.mark.parametrize("change,want,text", [
    (dict(dt=-1), INVALID, b"dtype"), (dict(d=-3), INVALID, b"d <= 0"), (dict(n=-1), INVALID, b"negative"),
    (dict(n=BIG), CAPACITY, b"int32"), (dict(n_rows=BIG), CAPACITY, b"int32"), (dict(ids=None), INVALID, b"NULL ids"),
    (dict(dout=None), INVALID, b"NULL dout"), (dict(dtable=None), INVALID, b"NULL dtable"),
    (dict(ld=6), INVALID, b"dout rows"), (dict(ldt=10), INVALID, b"dtable rows"), (dict(dtable=A + 2), INVALID, b"dtable rows"),
    (dict(n=5000), INVALID, b"needed"), (dict(n=5000, ws=A, ws_bytes=1000), INVALID, b"needed"),
    (dict(n=5000, ws=A + 16, ws_bytes=1 << 40), INVALID, b"256-byte"),
    (dict(n=5000, ws=None, ws_bytes=1 << 40), INVALID, b"256-byte"),
])
def test_embedding_backward_refusals(change, want, text):
    a = dict(BWD, **change)
    refused(lib.gnnav_embedding_backward(a["dout"], a["ld"], a["ids"], None, a["n"], a["d"], a["dt"], 1.0, a["acc"],
                                         a["dtable"], a["n_rows"], a["ldt"], a["ws"], a["ws_bytes"], None), want, text)


XENT = dict(h=A, ld_h=8, m=3, w=A, ld_w=8, v=5, d=8, dt=G.F32, labels=A, loss=A, dh=None, ld_dh=0, dw=None, ld_dw=0,
            ws=A, ws_bytes=1 << 40)


@pytest.mark.parametrize("change,want,text", [
    (dict(dt=7), INVALID, b"dtype"), (dict(m=-1), INVALID, b"m < 0"), (dict(v=0), INVALID, b"n_classes"),
    (dict(d=0), INVALID, b"d <= 0"), (dict(m=BIG), CAPACITY, b"int32"), (dict(v=BIG), CAPACITY, b"int32"),
    (dict(d=BIG), CAPACITY, b"int32"), (dict(loss=None), INVALID, b"NULL loss"), (dict(h=None), INVALID, b"NULL h"),
    (dict(w=None), INVALID, b"NULL w"), (dict(labels=None), INVALID, b"NULL labels"), (dict(ld_h=4), INVALID, b"h rows"),
    (dict(w=A + 4), INVALID, b"w rows"), (dict(dh=A, ld_dh=4), INVALID, b"dh rows"),
    (dict(dw=A + 8, ld_dw=8), INVALID, b"dw rows"), (dict(ws_bytes=100), INVALID, b"needed"),
    (dict(ws=A + 128), INVALID, b"256-byte"), (dict(ws=None), INVALID, b"256-byte"),
])
def test_linear_xent_refusals(change, want, text):
    a = dict(XENT, **change)
    refused(lib.gnnav_linear_xent(a["h"], a["ld_h"], a["m"], a["w"], a["ld_w"], a["v"], a["d"], a["dt"], a["labels"], -1,
                                  a["loss"], None, a["dh"], a["ld_dh"], a["dw"], a["ld_dw"], a["ws"], a["ws_bytes"],
                                  None), want, text)


def test_workspace_sizes():
    """Host only: -1 for bad arguments; the cross entropy's does not grow with m * n_classes."""
    for bad in [(-1, 5, 8, 0), (5, -1, 8, 0), (5, 5, 0, 0), (5, 5, 8, 3), (BIG, 5, 8, 0)]:
        assert lib.gnnav_embedding_backward_workspace(*bad) == -1
    for bad in [(-1, 5, 8, 0, 1), (5, 0, 8, 0, 1), (5, 5, 0, 0, 1), (5, 5, 8, 3, 1), (5, BIG, 8, 0, 1)]:
        assert lib.gnnav_linear_xent_workspace(*bad) == -1
    assert lib.gnnav_clip_workspace(-1) == -1 and lib.gnnav_clip_workspace(0) > 0
    with pytest.raises(G.GnnavError):
        G.linear_xent_workspace(5, 0, 8, "f32")
    with pytest.raises(G.GnnavError):
        G.embedding_backward_workspace(5, 5, 0, "bf16")
    for dtype, elt in (("f32", 4), ("bf16", 2)):
        m, v, d = 8192, 10_000_000, 256
        logits = m * v * 4
        assert G.linear_xent_workspace(m, v, d, dtype, True) < logits // 100
        for rows in (1, 32, 33, 200, 8192, 300_000):     # a piece is a piece
            for grads in (False, True):
                one, ten = (G.linear_xent_workspace(rows, k * v, d, dtype, grads) for k in (1, 10))
                assert ten < 1.1 * one + (10 * v if rows <= 32 else 0) + (1 << 20), (rows, grads, one, ten)
        # growing only with what it is made of
        sizes = [G.linear_xent_workspace(m, v, d, dtype, g) for m in (1, 33, 1000) for v in (10, 10_000, 1_000_000)
                 for d in (3, 100) for g in (False, True)]
        assert all(s > 0 for s in sizes)
        assert G.embedding_backward_workspace(1_000_000, 1000, 64, dtype) < 1_000_000 * 64 * 4


@pytest.mark.parametrize("call", ["norm", "clip", "step"])
@pytest.mark.parametrize("case", ["dtype", "n", "list", "count", "tensor", "align", "norm", "ws", "max", "nan", "lr"])
def test_clip_refusals(call, case):
    n, dt, norm, ws, ws_bytes, max_norm, lr = 2, G.F32, A, A, 1 << 20, 1.0, 0.1
    ptrs = (C.c_void_p * 2)(A, A + 4096)
    other = (C.c_void_p * 2)(A + 8192, A + 16384)
    counts = (C.c_int64 * 2)(10, 20)
    text = {"dtype": b"dtype", "n": b"n_tensors", "list": b"NULL tensor list", "count": b"negative count",
            "tensor": b"NULL tensor", "align": b"misaligned", "norm": b"NULL norm", "ws": b"needed",
            "max": b"max_norm", "nan": b"max_norm", "lr": b"lr is not finite"}[case]
    if case == "dtype":
        dt = 9
    elif case == "n":
        n = -1
    elif case == "list":
        ptrs = None
    elif case == "count":
        counts[1] = -1
    elif case == "tensor":
        ptrs[1] = None
    elif case == "align":
        ptrs[1] = A + 2
    elif case == "norm":
        norm = None
    elif case == "ws":
        ws_bytes = 8
    elif case == "max":
        max_norm = -1.0
    elif case == "nan":
        max_norm = float("nan")
    elif case == "lr":
        lr = float("inf")
    if (call == "norm" and case in ("max", "nan", "lr")) or (call == "clip" and case == "lr"):
        pytest.skip("the call has no such argument")
    if call == "norm":
        st = lib.gnnav_grad_norm(n, ptrs, counts, dt, norm, ws, ws_bytes, None)
    elif call == "clip":
        st = lib.gnnav_clip_grads(n, ptrs, counts, dt, max_norm, other, norm, ws, ws_bytes, None)
    else:
        st = lib.gnnav_sgd_clip_step(n, other, ptrs, counts, dt, lr, max_norm, norm, ws, ws_bytes, None)
    refused(st, INVALID, text)


def test_empty_calls_do_nothing():
    """Calls without work succeed without touching a device."""
    assert lib.gnnav_embedding(None, 10, 8, 8, G.F32, None, None, 0, 1.0, None, 8, None) == OK
    assert lib.gnnav_embedding_backward(None, 8, None, None, 0, 8, G.F32, 1.0, 1, None, 10, 8, None, 0, None) == OK
    assert lib.gnnav_embedding_backward(A, 8, A, None, 5, 8, G.F32, 1.0, 0, None, 0, 8, None, 0, None) == OK


def test_binding_refuses_host_tensors():
    import torch
    t, ids, one = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.zeros(1)
    for call in (lambda: G.embedding(t, ids, t), lambda: G.embedding_backward(t, ids, t),
                 lambda: G.linear_xent(t, t, ids, one), lambda: G.TensorList([t]), lambda: G.grad_norm([t], one)):
        with pytest.raises(ValueError):
            call()


def test_workspace_of_the_largest_sizes():
    """Up to the limits of the sizes the query answers, or says that it cannot."""
    top = 2 ** 31 - 1
    for m, v, d in [(top, 10, 8), (2 ** 30 + 1, 300, 64), (1, top, 8), (64, top, 1), (top, top, 1), (5, 7, 2 ** 20)]:
        for dt in (0, 1):
            for grads in (0, 1):
                assert lib.gnnav_linear_xent_workspace(m, v, d, dt, grads) > 0, (m, v, d, dt, grads)
