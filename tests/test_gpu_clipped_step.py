"""The clipped training step's own buffers: taken without waiting for the device, on the step's stream."""
import numpy as np
import pytest

import workloads as W
from test_gpu_parity import G, dev, host, say  # noqa: F401  (G is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how", ["stream", "address", "current"])
def test_first_clipped_step_does_not_wait(G, monkeypatch, how):
    """After unclipped steps (whose buffers grow, and wait for that) the first clipped one only enqueues; and it gives the
    same weights as a step that was clipped from the start."""
    import torch
    from paper_2404_09544_amd.step import MiniBatchStep, to_device_weights
    say("first clipped step", how)
    wl = W.Workload("chunglu-10k-d64")
    s, d = wl.edges()
    g = G.Graph(wl.n, s, d)
    c = G.Cache(g, wl.features(), "f32", 0.3)
    ws = [W.glorot(wl.dims[l], wl.dims[l + 1], "f32", seed=3 + l) for l in range(wl.L)]
    lab, seeds, lr, clip = dev(W.labels(wl.n, wl.dims[-1])), [dev(wl.seeds(b)) for b in range(3)], 0.3, 0.05
    plain, clipped = to_device_weights(ws, "f32"), to_device_weights(ws, "f32")
    one, two = (MiniBatchStep(g, c, w, wl.dims, wl.fanouts, "f32") for w in (plain, clipped))
    two.train(seeds[0], wl.rng_seed(0), lab, 0.0, clip_norm=clip)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    st = {"stream": stream, "address": stream.cuda_stream, "current": None}[how]
    one.train(seeds[0], wl.rng_seed(0), lab, 0.0, stream=st)
    torch.cuda.synchronize()

    def refuse(self):
        raise AssertionError("waited for a stream")
    for b in (1, 2):
        with monkeypatch.context() as mp:
            mp.setattr(torch.cuda.Stream, "synchronize", refuse)
            one.train(seeds[b], wl.rng_seed(b), lab, lr, stream=st, clip_norm=clip)
        two.train(seeds[b], wl.rng_seed(b), lab, lr, clip_norm=clip)
        torch.cuda.synchronize()
        assert one.grad_norm.item() == two.grad_norm.item() and one.loss.item() == two.loss.item()
        for x, y in zip(plain, clipped):
            assert np.array_equal(host(x), host(y))
