"""The operators of a trained table as a program uses them together: a frontier's
rows are looked up, aggregated, scored against every row of the same table, and
the table takes the clipped step of both gradients; also captured into a graph,
on several streams at once and under the pipelined training step.

The reference is torch in 64 bits on the CPU.  A gradient is off by its p (2^-15 relative and twice a
logit's error, as tests/test_gpu_linear_xent.py derives) and the fp32 sums after it: 2^-13 of
the largest entry, and by norm, bounds both with the sums' cancellation.
"""
import numpy as np
import pytest

import workloads as W
from test_gpu_embedding import matrix, torch_type
from test_gpu_parity import G, dev, graph_case, host, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu


class TableStep:
    """One step on a table [n, d]: mean over sampled neighbours, softmax over all rows, clipped SGD."""

    def __init__(self, G, n, d, scale, lr, max_norm, batch, frontier):
        import torch
        self.G, self.scale, self.lr, self.max_norm = G, scale, lr, max_norm
        t = dict(dtype=torch.float32, device="cuda")
        self.x, self.h = torch.zeros((frontier, d), **t), torch.zeros((batch, d), **t)
        self.dh, self.dx = torch.zeros((batch, d), **t), torch.zeros((frontier, d), **t)
        self.grad = torch.zeros((n, d), **t)
        self.loss, self.norm = torch.zeros(1, **t), torch.zeros(1, **t)

    def run(self, table, blocks, labels):
        G, d = self.G, table.shape[1]
        sizes, nodes = blocks.sizes()
        v = blocks.hop(1)
        sizes_dev, bounds = blocks.device_sizes(1)
        G.embedding(table, nodes, self.x, self.scale, n_ids=sizes[1], n_ids_dev=sizes_dev + 4)
        G.aggregate_mean(v.indptr, v.indices, sizes[0], self.x, d, "f32", self.h)
        G.linear_xent(self.h[:sizes[0]], table, labels, self.loss, dh=self.dh[:sizes[0]], dw=self.grad)
        G.aggregate_mean_backward(v.indptr, v.indices, sizes[0], sizes[1], self.dh, d, self.dx)
        G.embedding_backward(self.dx, nodes, self.grad, self.scale, accumulate=True, n_ids=sizes[1])
        G.sgd_clip_step([table], [self.grad], self.lr, self.max_norm, self.norm)


@pytest.mark.parametrize("max_norm", [1e9, 0.05])
def test_training_a_table(G, max_norm):
    import torch
    n, u, v = graph_case("random-3000-30000-7")
    d, batch, scale, lr = 48, 300, 3.0, 0.5
    say("table training", n, d, batch, max_norm)
    g = G.Graph(n, u, v)
    seeds = W.epoch_permutation(n, 3)[:batch]
    blocks = G.Blocks()
    table = matrix(n, d, "f32", 4)
    table.mul_(0.3)
    step = TableStep(G, n, d, scale, lr, max_norm, batch, n)
    ref = table.double().cpu()
    labels = torch.randint(0, n, (batch,), generator=torch.Generator().manual_seed(1))
    labels[::11] = -1
    for it in range(3):
        G.sample(g, dev(seeds.astype(np.int32)), [6], 100 + it, blocks)
        nodes, sizes, ip, _, ix = blocks.to_host()
        table.copy_(ref.float())               # the same start for both
        ref = table.double().cpu()
        step.run(table, blocks, labels.int().cuda())
        G.sync()
        t = ref.clone().requires_grad_()
        x = t[torch.from_numpy(nodes[:sizes[1]]).long()] * scale
        rows = torch.repeat_interleave(torch.arange(sizes[0]), torch.from_numpy(np.diff(ip[0])).long())
        cnt = torch.from_numpy(np.diff(ip[0])).clamp(min=1).double()
        h = torch.zeros((sizes[0], d), dtype=torch.float64).index_add(0, rows, x[torch.from_numpy(ix[0]).long()]) / cnt[:, None]
        loss = torch.nn.functional.cross_entropy(h @ t.t(), labels[:sizes[0]], ignore_index=-1)
        loss.backward()
        grad, norm = t.grad, t.grad.norm().item()
        assert step.loss.item() == pytest.approx(loss.item(), rel=1e-5)
        got = step.grad.double().cpu()
        assert (got - grad).abs().max().item() <= 2.0 ** -13 * grad.abs().max().item()
        assert (got - grad).norm().item() <= 2.0 ** -13 * norm
        assert step.norm.item() == pytest.approx(norm, rel=2.0 ** -13)
        c = min(1.0, max_norm / norm)
        new = ref - lr * c * grad
        assert ((table.double().cpu() - new).norm() <= 2.0 ** -12 * (lr * c * norm) + 2.0 ** -24 * new.norm()).item()
        ref = new


def chain(G, s, stream=None):
    """Lookup, loss with gradients, the lookup's gradient on top, clipped step: no host synchronisation."""
    st = dict(stream=stream)
    G.embedding(s["table"], s["ids"], s["h"], 2.0, **st)
    G.linear_xent(s["h"], s["table"], s["labels"], s["loss"], row_loss=s["row"], dh=s["dh"], dw=s["grad"], workspace=s.get("ws"), **st)
    G.embedding_backward(s["dh"], s["ids"], s["grad"], 2.0, accumulate=True, workspace=s.get("ws2"), **st)
    G.sgd_clip_step([s["table"]], [s["grad"]], 0.5, 0.1, s["norm"], **st)


def chain_state(dtype, n, rows, d, seed):
    import torch
    t = dict(dtype=torch_type(dtype), device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(table=torch.randn((rows, d), generator=gen, device="cuda").to(t["dtype"]),
             ids=torch.randint(-1, rows, (n,), generator=gen, dtype=torch.int32, device="cuda"),
             labels=torch.randint(-1, rows, (n,), generator=gen, dtype=torch.int32, device="cuda"),
             h=torch.zeros((n, d), **t), dh=torch.zeros((n, d), **t), grad=torch.zeros((rows, d), **t))
    s.update(loss=torch.zeros(1, device="cuda"), row=torch.zeros(n, device="cuda"), norm=torch.zeros(1, device="cuda"))
    return s


OUT = ("table", "h", "dh", "grad", "loss", "row", "norm")


@pytest.mark.parametrize("dtype,n,rows,d", [("f32", 200, 1500, 40), ("bf16", 5000, 3000, 64), ("bf16", 20, 700, 24),
                                            ("f32", 5000, 900, 16), ("bf16", 300, 2000, 304)])
def test_captured_and_replayed(G, dtype, n, rows, d):
    """A captured chain, replayed between eager chains on other tensors, gives the eager chain's bits each time."""
    import torch
    say("table graph", dtype, n, rows, d)
    s, e, other = (chain_state(dtype, n, rows, d, k) for k in (1, 1, 2))
    start = s["table"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(G, s)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    s["table"].copy_(start)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g in graphs:        # two graphs of the same calls
        with torch.cuda.graph(g):
            chain(G, s)
    for it in range(5):
        graphs[it % 2].replay()
        chain(G, e)
        torch.cuda.synchronize()
        for k in OUT:
            assert torch.equal(s[k], e[k]), (it, k)
        chain(G, other)                       # work of the program's own between the replays
        s["ids"].copy_(s["ids"].roll(it + 1))
        e["ids"].copy_(s["ids"])
        s["labels"].copy_(s["labels"].flip(0))
        e["labels"].copy_(s["labels"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_on_several_streams_at_once(G, dtype):
    """Chains on four streams together, two of them on shares of the units, give the bits of one after another."""
    import torch
    say("table streams", dtype)
    shapes = [(900, 4000, 64), (6000, 2500, 32), (64, 9000, 104), (300, 3000, 304)]
    alone = [chain_state(dtype, *s, seed=k) for k, s in enumerate(shapes)]
    both = [chain_state(dtype, *s, seed=k) for k, s in enumerate(shapes)]
    for s in alone:
        for _ in range(3):
            chain(G, s)
    torch.cuda.synchronize()
    shares = [G.stream_create(k, 2) for k in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream(), *shares]
    for _ in range(3):
        for st, s in zip(streams, both):
            chain(G, s, stream=st)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for k in OUT:
            assert torch.equal(a[k], b[k]), k
    for st in shares:
        G.stream_destroy(st)


def test_streams_by_address(G):
    """A stream given as an address, the null stream's among them; workspaces come from torch either way."""
    import torch
    a, b, c = (chain_state("f32", 5000, 900, 16, 3) for _ in range(3))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for s, st in ((a, None), (b, 0), (c, side.cuda_stream)):
        chain(G, s, stream=st)
    torch.cuda.synchronize()
    for k in OUT:
        assert torch.equal(a[k], b[k]) and torch.equal(a[k], c[k]), k


def test_nothing_is_allocated(G):
    """With workspaces given, the library allocates nothing (its allocation hook armed)."""
    import torch
    s = chain_state("f32", 5000, 900, 16, 3)
    s["ws"] = torch.empty(G.linear_xent_workspace(5000, 900, 16, "f32"), dtype=torch.uint8, device="cuda")
    s["ws2"] = torch.empty(G.embedding_backward_workspace(5000, 900, 16, "f32"), dtype=torch.uint8, device="cuda")
    G.debug_fail_allocations(0)
    try:
        chain(G, s)
    finally:
        G.debug_fail_allocations(-1)
    G.sync()


@pytest.mark.parametrize("async_mode", [False, True])
@pytest.mark.parametrize("clip_norm", [1e9, 0.01])
def test_clipped_training_step(G, async_mode, clip_norm):
    """MiniBatchStep.train(clip_norm): the plain step's gradients, the clipped update of them, also pipelined."""
    import torch
    from paper_2404_09544_amd.step import MiniBatchStep, Pipeline, to_device_weights
    wl = W.Workload("chunglu-10k-d64")
    s, d = wl.edges()
    g = G.Graph(wl.n, s, d)
    c = G.Cache(g, wl.features(), "f32", 0.3)
    ws = [W.glorot(wl.dims[l], wl.dims[l + 1], "f32", seed=3 + l) for l in range(wl.L)]
    lab, seeds, lr = dev(W.labels(wl.n, wl.dims[-1])), [dev(wl.seeds(b)) for b in range(4)], 0.3
    w_seq = to_device_weights(ws, "f32")
    step = MiniBatchStep(g, c, w_seq, wl.dims, wl.fanouts, "f32")
    w_ref = to_device_weights(ws, "f32")
    ref = MiniBatchStep(g, c, w_ref, wl.dims, wl.fanouts, "f32")
    grads = [torch.zeros_like(w) for w in w_ref]
    for b in range(4):
        say("clipped step", async_mode, clip_norm, b)
        step.train(seeds[b], wl.rng_seed(b), lab, lr, async_mode=async_mode, clip_norm=clip_norm)
        before = [host(w).astype(np.float64) for w in w_ref]
        ref.train(seeds[b], wl.rng_seed(b), lab, 0.0, grads=grads)
        torch.cuda.synchronize()
        norm = float(np.sqrt(sum((host(t).astype(np.float64) ** 2).sum() for t in grads)))
        assert step.grad_norm.item() == pytest.approx(norm, rel=2.0 ** -22)
        assert step.loss.item() == ref.loss.item()
        k = lr * min(1.0, clip_norm / norm)
        for w, r, old, t in zip(w_seq, w_ref, before, grads):
            want = old - k * host(t).astype(np.float64)
            assert np.allclose(host(w), want, rtol=2.0 ** -22, atol=2.0 ** -22 * float(np.abs(want).max()))
            r.copy_(w)
    w_pipe = to_device_weights(ws, "f32")
    pipe = Pipeline(g, c, w_pipe, wl.dims, wl.fanouts, "f32", depth=2)
    for b in range(4):
        pipe.enqueue_train(seeds[b], wl.rng_seed(b), lab, lr, clip_norm=clip_norm)
    pipe.synchronize()
    for a, b in zip(w_seq, w_pipe):
        assert np.array_equal(host(a), host(b))
