"""A student that learns from a sampled model, as a program uses the operators together: the model's logits
of a batch are kept by their largest, the student's gated block answers the batch's own rows, learns from
them and from the labels, and takes the clipped step; also captured into a graph, on several streams at
once, and with no allocation.

The reference is torch in 64 bits on the CPU.  A gradient is off by its p and q (2^-15 relative, as
tests/test_gpu_distill.py derives for these sizes) and the fp32 sums after it: 2^-13 of the largest entry, and by
norm, bounds both with the sums' cancellation.
"""
import numpy as np
import pytest

import workloads as W
from test_gpu_embedding import torch_type, unit_end
from test_gpu_parity import G, dev, graph_case, host, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu


def rows(m, d, dtype, seed=None, std=1.0):
    """[m, d], rows on 16-byte boundaries; zeros without a seed."""
    import torch
    t = torch.zeros((m, unit_end(d, dtype)), dtype=torch_type(dtype), device="cuda")
    if seed is not None:
        gen = torch.Generator(device="cuda").manual_seed(seed)
        t.copy_(torch.randn(t.shape, generator=gen, device="cuda") * std)
    return t[:, :d]


def reference(x, wg, wu, wd, teacher, k, labels, temp, alpha):
    """torch in 64 bits: the loss, its two means and the gradients of the three weights and of x."""
    import torch
    leaves = [t.detach().double().cpu().clone().requires_grad_() for t in (x, wg, wu, wd)]
    a, b = leaves[0] @ leaves[1], leaves[0] @ leaves[2]
    z = (torch.nn.functional.silu(a) * b) @ leaves[3]
    t, ids = torch.sort(teacher.double().cpu(), dim=1, descending=True, stable=True)
    t, ids = t[:, :k], ids[:, :k]
    log_q, log_p = torch.log_softmax(t / temp, 1), torch.log_softmax(z / temp, 1).gather(1, ids)
    kd = temp ** 2 * (log_q.exp() * (log_q - log_p)).sum(1).mean()
    ce = torch.nn.functional.cross_entropy(z, labels.long().cpu(), ignore_index=-1)
    loss = alpha * kd + (1 - alpha) * ce
    loss.backward()
    return (loss.item(), kd.item(), ce.item()), [t.grad for t in leaves]


@pytest.mark.parametrize("max_norm", [1e9, 0.05])
def test_learning_from_a_sampled_model(G, max_norm):
    import torch
    n, u, v = graph_case("random-3000-30000-7")
    d, hidden, classes, f, batch, k, temp, alpha, lr = 48, 32, 24, 72, 300, 6, 2.0, 0.6, 0.5
    say("student", n, d, f, batch, max_norm)
    g = G.Graph(n, u, v)
    feats = W.features(n, d, "f32", seed=5)
    cache = G.Cache(g, feats, "f32", 0.5)
    teacher_w = [dev(W.glorot(a, b, "f32", seed=3 + i)) for i, (a, b) in enumerate(((d, hidden), (hidden, classes)))]
    blocks = G.Blocks()
    seeds = W.epoch_permutation(n, 3)[:batch]
    ws = [rows(d, f, "f32", 1, 0.2), rows(d, f, "f32", 2, 0.2), rows(f, classes, "f32", 3, 0.2)]
    grads = [torch.zeros_like(w) for w in ws]
    z, dz, teacher = rows(batch, classes, "f32"), rows(batch, classes, "f32"), rows(batch, classes, "f32")
    values, ids = torch.zeros((batch, k), device="cuda"), torch.zeros((batch, k), dtype=torch.int32, device="cuda")
    loss, norm = torch.zeros(3, device="cuda"), torch.zeros(1, device="cuda")
    saved = torch.zeros(G.gated_ffn_saved(batch, f, "f32"), dtype=torch.uint8, device="cuda")
    labels = torch.randint(0, classes, (batch,), generator=torch.Generator().manual_seed(1)).int()
    labels[::7] = -1
    ref = [w.double().cpu() for w in ws]
    for it in range(3):
        # the model answers from sampled neighbourhoods; the batch's own rows are the first of the gathered ones
        G.sample(g, dev(seeds.astype(np.int32)), [5, 4], 100 + it, blocks)
        sizes, nodes = blocks.sizes()
        x = torch.zeros((sizes[2], cache.ld), device="cuda")
        counts = torch.zeros(3, dtype=torch.int64, device="cuda")
        G.gather(cache, nodes, sizes[2], x, counts)
        G.sage_forward(blocks, x, teacher_w, [d, hidden, classes], "f32", teacher)
        G.top_logits(teacher, values, ids)
        own = x[:batch, :d]
        for w, r in zip(ws, ref):
            w.copy_(r.float())
        start = [w.double().cpu() for w in ws]
        G.gated_ffn(own, *ws, z, saved=saved)
        G.distill(z, ids, values, loss, temperature=temp, alpha=alpha, labels=labels.cuda(), dlogits=dz)
        G.gated_ffn_backward(own, *ws, dz, saved, dwg=grads[0], dwu=grads[1], dwd=grads[2])
        G.sgd_clip_step(ws, grads, lr, max_norm, norm)
        G.sync()
        want, by = reference(own, *start, teacher, k, labels, temp, alpha)
        assert loss.tolist() == pytest.approx(want, rel=1e-5)
        total = float(torch.sqrt(sum((t ** 2).sum() for t in by[1:])))
        c = min(1.0, max_norm / total)
        assert norm.item() == pytest.approx(total, rel=2.0 ** -13)
        ref = []
        for got, t, w, old in zip(grads, by[1:], ws, start):
            assert (got.double().cpu() - t).abs().max().item() <= 2.0 ** -13 * t.abs().max().item()
            new = old - lr * c * t
            assert ((w.double().cpu() - new).norm() <= 2.0 ** -12 * lr * c * t.norm() + 2.0 ** -24 * new.norm()).item()
            ref.append(new)


def chain(G, s, stream=None):
    """Top logits, block, loss, gradients, clipped step: no host synchronisation."""
    st = dict(stream=stream)
    G.top_logits(s["teacher"], s["values"], s["ids"], workspace=s.get("ws0"), **st)
    G.gated_ffn(s["x"], s["wg"], s["wu"], s["wd"], s["z"], saved=s["saved"], workspace=s.get("ws1"), **st)
    G.distill(s["z"], s["ids"], s["values"], s["loss"], temperature=2.0, alpha=0.6, labels=s["labels"], row_loss=s["row"], dlogits=s["dz"],
              workspace=s.get("ws2"), **st)
    G.gated_ffn_backward(s["x"], s["wg"], s["wu"], s["wd"], s["dz"], s["saved"], dx=s["dx"], dwg=s["dwg"], dwu=s["dwu"], dwd=s["dwd"],
                         workspace=s.get("ws3"), **st)
    G.sgd_clip_step([s["wg"], s["wu"], s["wd"]], [s["dwg"], s["dwu"], s["dwd"]], 0.5, 0.1, s["norm"], **st)
    G.gated_ffn(s["x"][:3], s["wg"], s["wu"], s["wd"], s["answer"], workspace=s.get("ws4"), **st)


def chain_state(G, dtype, m, d, f, classes, k, seed):
    import torch
    s = dict(x=rows(m, d, dtype, seed), wg=rows(d, f, dtype, seed + 1, 0.2), wu=rows(d, f, dtype, seed + 2, 0.2), wd=rows(f, classes, dtype, seed + 3, 0.2),
             teacher=rows(m, classes, "f32", seed + 4, 2.0), z=rows(m, classes, dtype), dz=rows(m, classes, dtype), dx=rows(m, d, dtype),
             dwg=rows(d, f, dtype), dwu=rows(d, f, dtype), dwd=rows(f, classes, dtype), answer=rows(3, classes, dtype))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s.update(labels=torch.randint(-1, classes, (m,), generator=gen, dtype=torch.int32, device="cuda"), values=torch.zeros((m, k), device="cuda"),
             ids=torch.zeros((m, k), dtype=torch.int32, device="cuda"), loss=torch.zeros(3, device="cuda"), row=torch.zeros(m, device="cuda"),
             norm=torch.zeros(1, device="cuda"), saved=torch.zeros(G.gated_ffn_saved(m, f, dtype), dtype=torch.uint8, device="cuda"))
    return s


OUT = ("wg", "wu", "wd", "z", "dz", "dx", "dwg", "dwu", "dwd", "loss", "row", "norm", "values", "ids", "answer")
CASES = [("f32", 200, 40, 72, 24, 5), ("bf16", 3000, 64, 128, 48, 8), ("bf16", 20, 24, 64, 40_000, 16), ("f32", 5000, 16, 32, 8, 3),
         ("f32", 300, 104, 304, 9_000, 40), ("bf16", 40, 600, 2048, 64, 64)]


@pytest.mark.parametrize("dtype,m,d,f,classes,k", CASES)
def test_captured_and_replayed(G, dtype, m, d, f, classes, k):
    """Two captured chains, replayed between eager chains on other tensors, give the eager chain's bits each time."""
    import torch
    say("student graph", dtype, m, d, f, classes, k)
    s, e, other = (chain_state(G, dtype, m, d, f, classes, k, seed) for seed in (1, 1, 20))
    start = {n: s[n].clone() for n in ("wg", "wu", "wd")}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(G, s)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for n, w in start.items():
        s[n].copy_(w)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g in graphs:
        with torch.cuda.graph(g):
            chain(G, s)
    for it in range(5):
        graphs[it % 2].replay()
        chain(G, e)
        torch.cuda.synchronize()
        for n in OUT:
            assert torch.equal(s[n], e[n]), (it, n)
        chain(G, other)                       # work of the program's own between the replays
        for t in (s, e):
            t["teacher"].copy_(other["teacher"].roll(it + 1, 0))
            t["labels"].copy_(other["labels"].roll(it, 0))


def test_on_several_streams_at_once(G):
    """Chains on streams together, two of them on shares of the units, give the bits of one after another."""
    import torch
    alone = [chain_state(G, *c, seed=30 + i) for i, c in enumerate(CASES)]
    both = [chain_state(G, *c, seed=30 + i) for i, c in enumerate(CASES)]
    for s in alone:
        for _ in range(3):
            chain(G, s)
    torch.cuda.synchronize()
    shares = [G.stream_create(i, 2) for i in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream(), *shares, torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for st, s in zip(streams, both):
            chain(G, s, stream=st)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for n in OUT:
            assert torch.equal(a[n], b[n]), n
    for st in shares:
        G.stream_destroy(st)


def test_streams_by_address(G):
    """A stream given as an address, the null stream's among them; workspaces come from torch either way."""
    import torch
    a, b, c = (chain_state(G, *CASES[4], seed=3) for _ in range(3))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for s, st in ((a, None), (b, 0), (c, side.cuda_stream)):
        chain(G, s, stream=st)
    torch.cuda.synchronize()
    for n in OUT:
        assert torch.equal(a[n], b[n]) and torch.equal(a[n], c[n]), n


@pytest.mark.parametrize("dtype,m,d,f,classes,k", CASES)
def test_nothing_is_allocated(G, dtype, m, d, f, classes, k):
    """With workspaces given, the library allocates nothing (its allocation hook armed); garbage in them changes no bit."""
    import torch
    s, e = (chain_state(G, dtype, m, d, f, classes, k, seed=3) for _ in range(2))
    for i, need in enumerate((G.top_logits_workspace(m, classes, k, "f32"), G.gated_ffn_workspace(m, d, f, classes, dtype),
                              G.distill_workspace(m, classes, k, dtype), G.gated_ffn_backward_workspace(m, d, f, classes, dtype),
                              G.gated_ffn_workspace(3, d, f, classes, dtype))):
        s[f"ws{i}"] = torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device="cuda")
    G.debug_fail_allocations(0)
    try:
        chain(G, s)
    finally:
        G.debug_fail_allocations(-1)
    chain(G, e)
    G.sync()
    for n in OUT:
        assert torch.equal(s[n], e[n]), n
