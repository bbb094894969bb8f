"""Python binding of libgnnav.so (the C ABI declared in include/gnnav.h).

Argument marshalling only: every step of the sampled mini-batch path runs in
the HIP kernels of the library.  torch supplies device memory (tensors) and
the stream (``torch.cuda.current_stream()``); nothing else is used from it.
If the library is not built this module raises on import: there is no CPU
fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgnnav.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run `python paper_2404_09544_amd/build.py`")

# torch first: its wheel carries its own HIP runtime, which it loads by a
# file name that differs from the runtime's soname.  Loaded after torch, the
# library's libamdhip64.so.7 dependency resolves to that same copy; loaded
# before, the process would end up with two runtimes (two sets of device
# state), and allocations made through one fail in the other.
import torch  # noqa: E402,F401

_lib = C.CDLL(LIB_PATH)

F32, BF16 = 0, 1
SYMMETRIZE, OFFSETS_I64 = 0x1, 0x2
STORE_ON_DEVICE = 0x1
STATUS = {0: "OK", 1: "E_INVALID", 2: "E_RANGE", 3: "E_NOMEM", 4: "E_CAPACITY", 5: "E_DEVICE"}
EXPORTS = [
    "gnnav_last_error", "gnnav_abi_version", "gnnav_build_csr", "gnnav_graph_info",
    "gnnav_graph_csr_host", "gnnav_graph_free", "gnnav_build_cache", "gnnav_cache_info",
    "gnnav_cache_slot_map_host", "gnnav_cache_contents_host", "gnnav_cache_set_policy",
    "gnnav_cache_set_link_workgroups", "gnnav_cache_free", "gnnav_blocks_create", "gnnav_blocks_free",
    "gnnav_sample", "gnnav_sample_async", "gnnav_sample_biased", "gnnav_blocks_sync", "gnnav_blocks_device_sizes",
    "gnnav_blocks_hop", "gnnav_blocks_nodes", "gnnav_gather", "gnnav_gather_n", "gnnav_gather_n_after",
    "gnnav_aggregate_mean", "gnnav_combine", "gnnav_combine_kernel", "gnnav_sage_forward", "gnnav_sage_train_step",
    "gnnav_softmax_xent", "gnnav_aggregate_mean_backward", "gnnav_weight_grad", "gnnav_profile_start",
    "gnnav_profile_stop", "gnnav_profile_count", "gnnav_profile_get", "gnnav_profile_samples",
    "gnnav_sync", "gnnav_debug_set_spin_limit", "gnnav_debug_fail_allocations", "gnnav_gather_noalloc",
    "gnnav_stream_create", "gnnav_stream_destroy",
    "gnnav_embedding", "gnnav_embedding_backward", "gnnav_embedding_backward_workspace",
    "gnnav_linear_xent", "gnnav_linear_xent_workspace",
    "gnnav_grad_norm", "gnnav_clip_grads", "gnnav_sgd_clip_step", "gnnav_clip_workspace",
]


class GnnavError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class BlockView(C.Structure):
    _fields_ = [("n_dst", C.c_int64), ("n_src", C.c_int64), ("nnz", C.c_int64),
                ("indptr", C.c_void_p), ("indices", C.c_void_p), ("neighbors", C.c_void_p),
                ("src_ids", C.c_void_p)]


P, i64, i32, u32, u64, f64 = C.c_void_p, C.c_int64, C.c_int32, C.c_uint32, C.c_uint64, C.c_double
_sig = {
    "gnnav_last_error": ([], C.c_char_p),
    "gnnav_abi_version": ([], i32),
    "gnnav_build_csr": ([i64, i64, P, P, u32, P], i32),
    "gnnav_graph_info": ([P, P, P, P, P], i32),
    "gnnav_graph_csr_host": ([P, P, P], i32),
    "gnnav_graph_free": ([P], None),
    "gnnav_build_cache": ([P, P, i64, i32, f64, u32, P], i32),
    "gnnav_cache_info": ([P, P, P, P, P, P], i32),
    "gnnav_cache_slot_map_host": ([P, P], i32),
    "gnnav_cache_contents_host": ([P, P, P], i32),
    "gnnav_cache_set_policy": ([P, i32, i64], i32),
    "gnnav_cache_set_link_workgroups": ([P, i32], i32),
    "gnnav_cache_free": ([P], None),
    "gnnav_blocks_create": ([P], i32),
    "gnnav_blocks_free": ([P], None),
    "gnnav_sample": ([P, P, i64, P, i32, u64, P, P], i32),
    "gnnav_sample_async": ([P, P, i64, P, i32, u64, P, P], i32),
    "gnnav_sample_biased": ([P, P, u32, P, i64, P, i32, u64, P, i32, P], i32),
    "gnnav_blocks_sync": ([P, P], i32),
    "gnnav_blocks_device_sizes": ([P, P, P], i32),
    "gnnav_gather_n": ([P, P, P, i64, P, i64, P, P], i32),
    "gnnav_gather_n_after": ([P, P, P, i64, P, i64, P, P, P], i32),
    "gnnav_blocks_hop": ([P, i32, C.POINTER(BlockView)], i32),
    "gnnav_blocks_nodes": ([P, P, P, P], i32),
    "gnnav_gather": ([P, P, i64, P, i64, P, P], i32),
    "gnnav_aggregate_mean": ([P, P, i64, P, i64, i64, i32, P, i64, P], i32),
    "gnnav_combine": ([P, i64, P, i64, i64, i64, P, i64, i32, i32, i32, P, i64, P], i32),
    "gnnav_combine_kernel": ([i64, i64, i32], i32),
    "gnnav_sage_forward": ([P, P, i64, P, P, i32, i32, P, i64, P], i32),
    "gnnav_sage_train_step": ([P, P, i64, P, P, i32, P, C.c_float, P, i64, P, P, P], i32),
    "gnnav_softmax_xent": ([P, i64, i64, i64, P, P, i64, P, P], i32),
    "gnnav_aggregate_mean_backward": ([P, P, i64, i64, P, i64, P, i64, P, i64, i64, P, i64, P], i32),
    "gnnav_weight_grad": ([P, i64, P, i64, i64, i64, P, i64, i64, P, P], i32),
    "gnnav_profile_start": ([], i32),
    "gnnav_profile_stop": ([], i32),
    "gnnav_profile_count": ([], i32),
    "gnnav_profile_get": ([i32, P, i32, P, P], i32),
    "gnnav_profile_samples": ([i32, P, i64, P], i32),
    "gnnav_sync": ([P], i32),
    "gnnav_debug_set_spin_limit": ([u32], i32),
    "gnnav_debug_fail_allocations": ([i64], i32),
    "gnnav_gather_noalloc": ([P, P, i64, P, i64, P, P], i32),
    "gnnav_stream_create": ([i32, i32, P], i32),
    "gnnav_stream_destroy": ([P], i32),
    "gnnav_embedding": ([P, i64, i64, i64, i32, P, P, i64, C.c_float, P, i64, P], i32),
    "gnnav_embedding_backward": ([P, i64, P, P, i64, i64, i32, C.c_float, i32, P, i64, i64, P, i64, P], i32),
    "gnnav_embedding_backward_workspace": ([i64, i64, i64, i32], i64),
    "gnnav_linear_xent": ([P, i64, i64, P, i64, i64, i64, i32, P, i32, P, P, P, i64, P, i64, P, i64, P], i32),
    "gnnav_linear_xent_workspace": ([i64, i64, i64, i32, i32], i64),
    "gnnav_grad_norm": ([i32, P, P, i32, P, P, i64, P], i32),
    "gnnav_clip_grads": ([i32, P, P, i32, C.c_float, P, P, P, i64, P], i32),
    "gnnav_sgd_clip_step": ([i32, P, P, P, i32, C.c_float, C.c_float, P, P, i64, P], i32),
    "gnnav_clip_workspace": ([i32], i64),
}
for _name, (_args, _res) in _sig.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = _res


def _check(st: int):
    if st != 0:
        raise GnnavError(st, _lib.gnnav_last_error().decode())


def abi_version() -> int:
    return int(_lib.gnnav_abi_version())


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def sync(stream=None):
    """gnnav_sync: wait for `stream`; raises E_DEVICE if device-side work has
    reported a failure (a scan whose look-back wait gave up) since the last
    report."""
    _check(_lib.gnnav_sync(_stream(stream)))


def stream_create(part: int, parts: int):
    """gnnav_stream_create: a stream on share `part` of `parts` of the
    compute units, as a torch.cuda.ExternalStream.  The library's stream
    outlives the wrapper; release it with stream_destroy."""
    import torch
    h = C.c_void_p()
    _check(_lib.gnnav_stream_create(int(part), int(parts), C.byref(h)))
    return torch.cuda.ExternalStream(h.value)


def stream_destroy(stream):
    """gnnav_stream_destroy: waits for the stream, then releases it."""
    _check(_lib.gnnav_stream_destroy(_stream(stream)))


def debug_set_spin_limit(polls: int):
    """Testing hook: look-back polls before a scan's wait gives up (0: at once)."""
    _check(_lib.gnnav_debug_set_spin_limit(int(polls)))


def debug_fail_allocations(after: int):
    """Testing hook: allocations after the next `after` fail (negative: off)."""
    _check(_lib.gnnav_debug_fail_allocations(int(after)))


def _dev_ptr(t):
    return None if t is None else t.data_ptr()


def _np_ptr(a: np.ndarray):
    return a.ctypes.data


def dtype_code(dtype: str) -> int:
    return {"f32": F32, "bf16": BF16}[dtype]


def padded_ld(d: int, dtype: str) -> int:
    elt = 2 if dtype == "bf16" else 4
    return (d * elt + 15) // 16 * 16 // elt


# ------------------------------------------------------------------ graph
class Graph:
    """CSR of G(V, E) in HBM (gnnav_build_csr)."""

    def __init__(self, n_nodes: int, src, dst, symmetrize: bool = True, offsets_i64: bool = False):
        src = np.ascontiguousarray(src, dtype=np.int32)
        dst = np.ascontiguousarray(dst, dtype=np.int32)
        if src.shape != dst.shape:
            raise ValueError("src and dst differ in length")
        flags = (SYMMETRIZE if symmetrize else 0) | (OFFSETS_I64 if offsets_i64 else 0)
        h = P()
        _check(_lib.gnnav_build_csr(n_nodes, src.size, _np_ptr(src), _np_ptr(dst), flags, C.byref(h)))
        self._h = h
        n, nnz, md, o64 = i64(), i64(), i64(), i32()
        _check(_lib.gnnav_graph_info(h, C.byref(n), C.byref(nnz), C.byref(md), C.byref(o64)))
        self.n, self.nnz, self.max_degree, self.offsets_i64 = n.value, nnz.value, md.value, bool(o64.value)

    def csr_host(self, with_col: bool = True):
        rp = np.empty(self.n + 1, np.int64)
        col = np.empty(max(self.nnz, 1), np.int32) if with_col else None
        _check(_lib.gnnav_graph_csr_host(self._h, _np_ptr(rp), _np_ptr(col) if with_col else None))
        return rp, (col[:self.nnz] if with_col else None)

    def close(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.gnnav_graph_free(self._h)
            self._h = None

    __del__ = close


# ------------------------------------------------------------------ cache
class Cache:
    """Degree-ranked HBM cache + pinned host store (gnnav_build_cache)."""

    def __init__(self, graph: Graph, feats: np.ndarray, dtype: str, cache_fraction: float,
                 store_on_device: bool = False):
        feats = np.ascontiguousarray(feats)
        if feats.ndim != 2 or feats.shape[0] != graph.n:
            raise ValueError("features must be [n_nodes, d]")
        want = np.uint16 if dtype == "bf16" else np.float32
        if feats.dtype != want:
            raise ValueError(f"features must be {want} for dtype {dtype}")
        h = P()
        _check(_lib.gnnav_build_cache(graph._h, _np_ptr(feats), feats.shape[1], dtype_code(dtype),
                                      float(cache_fraction), STORE_ON_DEVICE if store_on_device else 0,
                                      C.byref(h)))
        self._h = h
        self.dtype = dtype
        nc, d, ld, dt, sod = i64(), i64(), i64(), i32(), i32()
        _check(_lib.gnnav_cache_info(h, C.byref(nc), C.byref(d), C.byref(ld), C.byref(dt), C.byref(sod)))
        self.n_cached, self.d, self.ld = nc.value, d.value, ld.value
        self.store_on_device = bool(sod.value)
        self.n = graph.n

    def set_policy(self, policy: str, dynamic_slots: int = 0):
        """'static', or 'fifo' / 'lru' over the last `dynamic_slots` cache slots."""
        code = {"static": 0, "fifo": 1, "lru": 2}[policy]
        _check(_lib.gnnav_cache_set_policy(self._h, code, int(dynamic_slots)))

    def set_link_workgroups(self, workgroups: int):
        """Workgroups of later gathers that copy misses over the host link."""
        _check(_lib.gnnav_cache_set_link_workgroups(self._h, int(workgroups)))

    def contents(self):
        """(owners int32[n_cached], rows [n_cached, ld]) currently in the cache."""
        owners = np.empty(max(self.n_cached, 1), np.int32)
        rows = np.empty((max(self.n_cached, 1), self.ld), np.uint16 if self.dtype == "bf16" else np.float32)
        _check(_lib.gnnav_cache_contents_host(self._h, _np_ptr(owners), _np_ptr(rows)))
        return owners[:self.n_cached], rows[:self.n_cached]

    def slot_map(self) -> np.ndarray:
        out = np.empty(max(self.n, 1), np.int32)
        _check(_lib.gnnav_cache_slot_map_host(self._h, _np_ptr(out)))
        return out[:self.n]

    def close(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.gnnav_cache_free(self._h)
            self._h = None

    __del__ = close


# ----------------------------------------------------------------- blocks
class Blocks:
    """Device workspace holding one batch's frontiers and hops."""

    def __init__(self):
        h = P()
        _check(_lib.gnnav_blocks_create(C.byref(h)))
        self._h = h

    def hop(self, h: int) -> BlockView:
        v = BlockView()
        _check(_lib.gnnav_blocks_hop(self._h, h, C.byref(v)))
        return v

    def sizes(self):
        L = i32()
        _check(_lib.gnnav_blocks_nodes(self._h, None, None, C.byref(L)))
        n = np.zeros(L.value + 1, np.int64)
        ptr = P()
        _check(_lib.gnnav_blocks_nodes(self._h, C.byref(ptr), _np_ptr(n), None))
        return [int(x) for x in n], ptr.value

    def sync(self, stream=None):
        """Publish the last (async) sample's sizes to the host."""
        _check(_lib.gnnav_blocks_sync(self._h, _stream(stream)))

    def device_sizes(self, n_hops: int):
        """(device pointer to the int32 size array, host Eq. 12 bounds [L+1])."""
        ptr = P()
        bounds = np.zeros(n_hops + 1, np.int64)
        _check(_lib.gnnav_blocks_device_sizes(self._h, C.byref(ptr), _np_ptr(bounds)))
        return ptr.value, [int(x) for x in bounds]

    def nodes_ptr(self) -> int:
        ptr = P()
        _check(_lib.gnnav_blocks_nodes(self._h, C.byref(ptr), None, None))
        return ptr.value

    def to_host(self):
        """Host copies: (nodes, sizes, [indptr], [neighbors], [indices])."""
        import torch
        torch.cuda.synchronize()
        sizes, nodes_ptr = self.sizes()
        L = len(sizes) - 1

        def fetch(ptr, count):
            out = np.empty(max(count, 1), np.int32)
            if count > 0:
                _hip_memcpy_d2h(out, ptr, count * 4)
            return out[:count]
        nodes = fetch(nodes_ptr, sizes[-1])
        ip, nb, ix = [], [], []
        for h in range(1, L + 1):
            v = self.hop(h)
            ip.append(fetch(v.indptr, v.n_dst + 1))
            nb.append(fetch(v.neighbors, v.nnz))
            ix.append(fetch(v.indices, v.nnz))
        return nodes, sizes, ip, nb, ix

    def close(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.gnnav_blocks_free(self._h)
            self._h = None

    __del__ = close


_hip = None


def _hip_memcpy_d2h(dst: np.ndarray, src_ptr: int, nbytes: int):
    """Synchronous device-to-host copy through the HIP runtime (test/tooling use)."""
    global _hip
    if _hip is None:
        _hip = C.CDLL("libamdhip64.so")
        _hip.hipMemcpy.argtypes = [P, P, C.c_size_t, C.c_int]
        _hip.hipMemcpy.restype = C.c_int
    rc = _hip.hipMemcpy(dst.ctypes.data, src_ptr, nbytes, 2)  # hipMemcpyDeviceToHost
    if rc != 0:
        raise GnnavError(5, f"hipMemcpy failed ({rc})")


def _copy_device_i32(dst, src_ptr: int, count: int):
    """Enqueue a device-to-device copy of `count` int32 from src_ptr into the
    torch tensor dst on torch's current stream (bookkeeping, not the path)."""
    global _hip
    if _hip is None:
        _hip = C.CDLL("libamdhip64.so")
        _hip.hipMemcpy.argtypes = [P, P, C.c_size_t, C.c_int]
        _hip.hipMemcpy.restype = C.c_int
    fn = _hip.hipMemcpyAsync
    fn.argtypes = [P, P, C.c_size_t, C.c_int, P]
    fn.restype = C.c_int
    import torch
    rc = fn(dst.data_ptr(), src_ptr, count * 4, 3, torch.cuda.current_stream().cuda_stream)
    if rc != 0:
        raise GnnavError(5, f"hipMemcpyAsync failed ({rc})")


# --------------------------------------------------------------- the path
def sample(graph: Graph, seeds, fanouts, rng_seed: int, blocks: Blocks, stream=None):
    """gnnav_sample: seeds is a device int32 tensor."""
    fan = np.ascontiguousarray(fanouts, dtype=np.int32)
    _check(_lib.gnnav_sample(graph._h, _dev_ptr(seeds), seeds.numel(), _np_ptr(fan), fan.size,
                             int(rng_seed) & 0xFFFFFFFFFFFFFFFF, blocks._h, _stream(stream)))
    return blocks


def sample_async(graph: Graph, seeds, fanouts, rng_seed: int, blocks: Blocks, stream=None):
    """gnnav_sample_async: enqueue only; sizes stay on the device."""
    fan = np.ascontiguousarray(fanouts, dtype=np.int32)
    _check(_lib.gnnav_sample_async(graph._h, _dev_ptr(seeds), seeds.numel(), _np_ptr(fan), fan.size,
                                   int(rng_seed) & 0xFFFFFFFFFFFFFFFF, blocks._h, _stream(stream)))
    return blocks


def sample_biased(graph: Graph, cache: Cache, eta: int, seeds, fanouts, rng_seed: int, blocks: Blocks,
                  async_: bool = False, stream=None):
    """gnnav_sample_biased: cached neighbours weigh eta (eta = 1: uniform weights)."""
    fan = np.ascontiguousarray(fanouts, dtype=np.int32)
    _check(_lib.gnnav_sample_biased(graph._h, cache._h, int(eta), _dev_ptr(seeds), seeds.numel(), _np_ptr(fan),
                                    fan.size, int(rng_seed) & 0xFFFFFFFFFFFFFFFF, blocks._h, int(bool(async_)),
                                    _stream(stream)))
    return blocks


def gather_n(cache: Cache, ids_ptr: int, n_ids_dev_ptr: int, n_ids_max: int, out, counts, stream=None,
             copy_after=None):
    """gnnav_gather_n: the request count is read from device memory.
    copy_after: a recorded torch.cuda.Event the row copies wait for."""
    if copy_after is None:
        _check(_lib.gnnav_gather_n(cache._h, ids_ptr, n_ids_dev_ptr, n_ids_max, _dev_ptr(out), out.stride(0),
                                   _dev_ptr(counts), _stream(stream)))
    else:
        _check(_lib.gnnav_gather_n_after(cache._h, ids_ptr, n_ids_dev_ptr, n_ids_max, _dev_ptr(out),
                                         out.stride(0), _dev_ptr(counts), copy_after.cuda_event, _stream(stream)))


def gather(cache: Cache, ids_ptr: int, n_ids: int, out, counts, stream=None):
    """gnnav_gather into a device tensor `out` [>= n_ids, ld] and int64 counts[3]."""
    ld = out.stride(0)
    _check(_lib.gnnav_gather(cache._h, ids_ptr, n_ids, _dev_ptr(out), ld, _dev_ptr(counts),
                             _stream(stream)))


def gather_noalloc(cache: Cache, ids_ptr: int, n_ids: int, out, counts, stream=None):
    """gnnav_gather_noalloc: gnnav_gather with its workspace in static device
    memory (at most 2**20 ids; calls overlapping on one device race)."""
    _check(_lib.gnnav_gather_noalloc(cache._h, ids_ptr, n_ids, _dev_ptr(out), out.stride(0), _dev_ptr(counts),
                                     _stream(stream)))


def aggregate_mean(indptr_ptr: int, indices_ptr: int, n_dst: int, x, d: int, dtype: str, out,
                   stream=None):
    _check(_lib.gnnav_aggregate_mean(indptr_ptr, indices_ptr, n_dst, _dev_ptr(x), x.stride(0), d,
                                     dtype_code(dtype), _dev_ptr(out), out.stride(0), _stream(stream)))


def combine(self_x, agg, m: int, d_in: int, w, d_out: int, dtype: str, relu: bool, out_bf16: bool,
            out, stream=None):
    _check(_lib.gnnav_combine(_dev_ptr(self_x), self_x.stride(0), _dev_ptr(agg), agg.stride(0), m, d_in,
                              _dev_ptr(w), d_out, dtype_code(dtype), int(relu), int(out_bf16),
                              _dev_ptr(out), out.stride(0), _stream(stream)))



COMBINE_KERNELS = {0: "skinny", 1: "ring", 2: "split"}


def combine_kernel(m: int, d_out: int, dtype: str) -> str:
    """gnnav_combine_kernel: which kernel a combine of m rows runs."""
    k = _lib.gnnav_combine_kernel(int(m), int(d_out), dtype_code(dtype))
    if k < 0:
        raise GnnavError(1, "bad combine_kernel arguments")
    return COMBINE_KERNELS[k]

def sage_train_step(blocks: Blocks, x, weights, dims, labels, lr: float, logits, loss, grads=None,
                    stream=None):
    """gnnav_sage_train_step: fp32; `weights` (device tensors) are updated in place."""
    L = len(weights)
    wp = (P * L)(*[w.data_ptr() for w in weights])
    gp = (P * L)(*[g.data_ptr() for g in grads]) if grads is not None else None
    dm = np.ascontiguousarray(dims, dtype=np.int32)
    _check(_lib.gnnav_sage_train_step(blocks._h, _dev_ptr(x), x.stride(0), wp, _np_ptr(dm), L,
                                      _dev_ptr(labels), float(lr), _dev_ptr(logits), logits.stride(0),
                                      _dev_ptr(loss), gp, _stream(stream)))


def softmax_xent(logits, n: int, n_classes: int, labels, dz, loss, stream=None):
    _check(_lib.gnnav_softmax_xent(_dev_ptr(logits), logits.stride(0), n, n_classes, _dev_ptr(labels),
                                   _dev_ptr(dz), dz.stride(0), _dev_ptr(loss), _stream(stream)))


def aggregate_mean_backward(indptr_ptr: int, indices_ptr: int, n_dst: int, n_src: int, dagg, d: int, out,
                            dself=None, mask=None, stream=None):
    _check(_lib.gnnav_aggregate_mean_backward(
        indptr_ptr, indices_ptr, n_dst, n_src, _dev_ptr(dagg), dagg.stride(0),
        _dev_ptr(dself) if dself is not None else None, dself.stride(0) if dself is not None else 0,
        _dev_ptr(mask) if mask is not None else None, mask.stride(0) if mask is not None else 0,
        d, _dev_ptr(out), out.stride(0), _stream(stream)))


def weight_grad(self_x, agg, m: int, d_in: int, dz, d_out: int, dw, stream=None):
    _check(_lib.gnnav_weight_grad(_dev_ptr(self_x), self_x.stride(0), _dev_ptr(agg), agg.stride(0), m, d_in,
                                  _dev_ptr(dz), dz.stride(0), d_out, _dev_ptr(dw), _stream(stream)))


def sage_forward(blocks: Blocks, x, weights, dims, dtype: str, logits, stream=None):
    L = len(weights)
    wp = (P * L)(*[w.data_ptr() for w in weights])
    dm = np.ascontiguousarray(dims, dtype=np.int32)
    _check(_lib.gnnav_sage_forward(blocks._h, _dev_ptr(x), x.stride(0), wp, _np_ptr(dm), L,
                                   dtype_code(dtype), _dev_ptr(logits), logits.stride(0),
                                   _stream(stream)))


# ------------------------------------- trained tables and large class sets
_TORCH_CODE = {torch.float32: F32, torch.bfloat16: BF16}


def _here() -> int:
    """Index of the current device (a host tensor's is -1; before torch's first use of a device there are no others)."""
    return torch._C._cuda_getDevice() if torch.cuda.is_initialized() else 0


def _on(stream, device: int) -> int:
    """The call's stream as an address: the current stream of the device unless one is given."""
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream)


def _rows(t, what: str, device: int, d=None, dtype=None):
    """Checks a device matrix with contiguous columns (rows at any stride); its (rows, columns, stride)."""
    if t.get_device() != device:
        raise ValueError(f"{what} is not on the current device")
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError(f"{what} must be a matrix with contiguous columns")
    if t.dtype is not dtype and (dtype is not None or t.dtype not in _TORCH_CODE):
        raise ValueError(f"{what} must be {dtype or 'float32 or bfloat16'}")
    if d is not None and shape[1] != d:
        raise ValueError(f"{what} must have {d} columns")
    return shape[0], shape[1], stride[0]


def _vector(t, what: str, device: int, dtype, n: int = 0):
    """Checks a contiguous device tensor of at least n elements; its address."""
    if t.get_device() != device:
        raise ValueError(f"{what} is not on the current device")
    if t.dtype is not dtype or not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of at least {n} elements")
    return t.data_ptr()


def _torch_stream(stream):
    """A stream that is given as a torch stream or as an address, as a torch stream."""
    if hasattr(stream, "cuda_stream"):
        return stream
    return torch.cuda.ExternalStream(_stream(stream)) if _stream(stream) else torch.cuda.default_stream()


def _workspace(given, need: int, device: int, stream):
    """(address, bytes, tensor that holds them) of a call's workspace; one that is not given comes
    from torch's allocator, in the pool of the stream that the call runs on."""
    if given is not None:
        return _vector(given, "workspace", device, torch.uint8), given.numel(), given
    if need == 0:
        return None, 0, None
    if stream is None:
        t = torch.empty(need, dtype=torch.uint8, device="cuda")
    else:
        with torch.cuda.stream(_torch_stream(stream)):
            t = torch.empty(need, dtype=torch.uint8, device="cuda")
    return t.data_ptr(), need, t


def _workspace_bytes(n: int) -> int:
    if n < 0:
        raise GnnavError(1, "bad workspace arguments")
    return int(n)


def _ids(ids, n_ids, device: int):
    """(address, count) of an id list: a device int32 tensor, or an address such as Blocks.nodes_ptr() with its count."""
    if isinstance(ids, int):
        if n_ids is None:
            raise ValueError("an address of ids needs n_ids")
        return ids, n_ids
    n = ids.numel() if n_ids is None else n_ids
    return _vector(ids, "ids", device, torch.int32, n), n


def _count(n_ids_dev, device: int):
    if n_ids_dev is None or isinstance(n_ids_dev, int):
        return n_ids_dev
    return _vector(n_ids_dev, "n_ids_dev", device, torch.int32, 1)


def embedding(table, ids, out, scale: float = 1.0, n_ids=None, n_ids_dev=None, stream=None):
    """gnnav_embedding: out[i] = scale * table[ids[i]] in the table's type (fp32 or
    bf16); an id outside the table gives a zero row.  ids: device int32 tensor,
    or the address of n_ids of them (a frontier's Blocks.nodes_ptr());
    n_ids_dev: device int32 (tensor or address) with the count of ids to take.
    Here and in the calls below rows start on 16-byte boundaries (GnnavError
    otherwise), and a row that is written is written up to the next boundary, with
    zeros behind its columns."""
    dev, dt = _here(), table.dtype
    rows, d, ld = _rows(table, "table", dev)
    n_out, _, ld_out = _rows(out, "out", dev, d, dt)
    ids_ptr, n = _ids(ids, n_ids, dev)
    if n_out < n:
        raise ValueError("out has fewer rows than ids")
    _check(_lib.gnnav_embedding(table.data_ptr(), rows, ld, d, _TORCH_CODE[dt], ids_ptr, _count(n_ids_dev, dev), n,
                                scale, out.data_ptr(), ld_out, _on(stream, dev)))


def embedding_backward_workspace(n_ids: int, n_rows: int, d: int, dtype: str) -> int:
    """Bytes of workspace that embedding_backward needs."""
    return _workspace_bytes(_lib.gnnav_embedding_backward_workspace(int(n_ids), int(n_rows), int(d), dtype_code(dtype)))


def embedding_backward(dout, ids, dtable, scale: float = 1.0, accumulate: bool = False, n_ids=None, n_ids_dev=None,
                       workspace=None, stream=None):
    """gnnav_embedding_backward: dtable[v] (+)= scale * the sum of the rows of dout whose id is v.
    ids, n_ids and n_ids_dev as for embedding."""
    dev, dt = _here(), dout.dtype
    n_in, d, ld = _rows(dout, "dout", dev)
    rows, _, ld_table = _rows(dtable, "dtable", dev, d, dt)
    (ids_ptr, n), code = _ids(ids, n_ids, dev), _TORCH_CODE[dt]
    if n_in < n:
        raise ValueError("dout has fewer rows than ids")
    need = 0 if workspace is not None else _workspace_bytes(_lib.gnnav_embedding_backward_workspace(n, rows, d, code))
    ws, ws_bytes, _hold = _workspace(workspace, need, dev, stream)
    _check(_lib.gnnav_embedding_backward(dout.data_ptr(), ld, ids_ptr, _count(n_ids_dev, dev), n, d, code, scale, bool(accumulate),
                                         dtable.data_ptr(), rows, ld_table, ws, ws_bytes, _on(stream, dev)))


def linear_xent_workspace(m: int, n_classes: int, d: int, dtype: str, grads: bool = True) -> int:
    """Bytes of workspace that linear_xent needs (grads: whether dh or dw is asked for)."""
    return _workspace_bytes(_lib.gnnav_linear_xent_workspace(int(m), int(n_classes), int(d), dtype_code(dtype),
                                                             int(bool(grads))))


def linear_xent(h, w, labels, loss, row_loss=None, dh=None, dw=None, ignore_label: int = -1, workspace=None,
                stream=None):
    """gnnav_linear_xent: softmax cross entropy of h [m, d] against the classes' rows w
    [n_classes, d] without the logits.  loss: float32[1], the mean over the rows
    whose label is not ignore_label; row_loss (float32[m]), dh [m, d] and dw
    [n_classes, d] are written where given."""
    dev, dt = _here(), h.dtype
    m, d, ld_h = _rows(h, "h", dev)
    v, _, ld_w = _rows(w, "w", dev, d, dt)
    labels_ptr = _vector(labels, "labels", dev, torch.int32, m)
    loss_ptr = _vector(loss, "loss", dev, torch.float32, 1)
    row_ptr = None if row_loss is None else _vector(row_loss, "row_loss", dev, torch.float32, m)
    dh_ptr = dw_ptr = None
    ld_dh = ld_dw = 0
    if dh is not None:
        n, _, ld_dh = _rows(dh, "dh", dev, d, dt)
        dh_ptr = dh.data_ptr()
        if n < m:
            raise ValueError("dh has fewer rows than h")
    if dw is not None:
        n, _, ld_dw = _rows(dw, "dw", dev, d, dt)
        dw_ptr = dw.data_ptr()
        if n < v:
            raise ValueError("dw has fewer rows than w")
    code = _TORCH_CODE[dt]
    need = 0 if workspace is not None else _workspace_bytes(
        _lib.gnnav_linear_xent_workspace(m, v, d, code, dh is not None or dw is not None))
    ws, ws_bytes, _hold = _workspace(workspace, need, dev, stream)
    _check(_lib.gnnav_linear_xent(h.data_ptr(), ld_h, m, w.data_ptr(), ld_w, v, d, code, labels_ptr, ignore_label,
                                  loss_ptr, row_ptr, dh_ptr, ld_dh, dw_ptr, ld_dw, ws, ws_bytes, _on(stream, dev)))


class TensorList:
    """Contiguous device tensors of one type, with the address and count arrays
    that the calls over many tensors take.  Holds the tensors."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        types = {t.dtype for t in self.tensors} or {torch.float32}
        if len(types) > 1 or next(iter(types)) not in _TORCH_CODE:
            raise ValueError("tensors must be all float32 or all bfloat16")
        self.device = self.tensors[0].get_device() if self.tensors else None
        for t in self.tensors:
            if t.get_device() < 0 or t.get_device() != self.device or not t.is_contiguous():
                raise ValueError("tensors must be contiguous tensors of one device")
        self.code = _TORCH_CODE[next(iter(types))]
        self.n = len(self.tensors)
        self.sizes = [t.numel() for t in self.tensors]
        self.ptrs = (P * max(self.n, 1))(*[t.data_ptr() for t in self.tensors])
        self.counts = (i64 * max(self.n, 1))(*self.sizes)


def _tensor_list(x, device: int) -> TensorList:
    x = x if isinstance(x, TensorList) else TensorList(x)
    if x.device is not None and x.device != device:
        raise ValueError("the tensors are not on the current device")
    return x


def _same(a: TensorList, b: TensorList, what: str):
    if a.sizes != b.sizes or (a.n and a.code != b.code):
        raise ValueError(f"{what} must match the gradients in number, sizes and type")
    return b


def clip_workspace(grads) -> int:
    """Bytes of workspace that grad_norm, clip_grads and sgd_clip_step need for these tensors."""
    return int(_lib.gnnav_clip_workspace(grads.n if isinstance(grads, TensorList) else len(grads)))


def _clip_args(grads, norm, workspace, stream):
    dev = _here()
    g = _tensor_list(grads, dev)
    norm_ptr = _vector(norm, "norm", dev, torch.float32, 1)
    return dev, g, norm_ptr, _workspace(workspace, 0 if workspace is not None else clip_workspace(g), dev, stream)


def grad_norm(grads, norm, workspace=None, stream=None):
    """gnnav_grad_norm: norm[0] = the global 2-norm of the tensors (a list or a TensorList)."""
    dev, g, norm_ptr, (ws, ws_bytes, _hold) = _clip_args(grads, norm, workspace, stream)
    _check(_lib.gnnav_grad_norm(g.n, g.ptrs, g.counts, g.code, norm_ptr, ws, ws_bytes, _on(stream, dev)))


def clip_grads(grads, max_norm: float, norm, out=None, workspace=None, stream=None):
    """gnnav_clip_grads: the tensors times min(1, max_norm / norm), in place or into `out`."""
    dev, g, norm_ptr, (ws, ws_bytes, _hold) = _clip_args(grads, norm, workspace, stream)
    o = g if out is None else _same(g, _tensor_list(out, dev), "out")
    _check(_lib.gnnav_clip_grads(g.n, g.ptrs, g.counts, g.code, max_norm, o.ptrs, norm_ptr, ws, ws_bytes,
                                 _on(stream, dev)))


def sgd_clip_step(weights, grads, lr: float, max_norm: float, norm, workspace=None, stream=None):
    """gnnav_sgd_clip_step: weights -= lr * min(1, max_norm / norm) * grads, in place."""
    dev, g, norm_ptr, (ws, ws_bytes, _hold) = _clip_args(grads, norm, workspace, stream)
    w = _same(g, _tensor_list(weights, dev), "weights")
    _check(_lib.gnnav_sgd_clip_step(g.n, w.ptrs, g.ptrs, g.counts, g.code, lr, max_norm, norm_ptr, ws, ws_bytes,
                                    _on(stream, dev)))


# -------------------------------------------------------------- profiling
def profile_start():
    _check(_lib.gnnav_profile_start())


def profile_samples() -> dict:
    """After profile_stop: {kernel name: float32 array of per-launch ms}."""
    out = {}
    buf = C.create_string_buffer(128)
    for i in range(_lib.gnnav_profile_count()):
        n = i64()
        _check(_lib.gnnav_profile_get(i, buf, 128, None, None))
        _check(_lib.gnnav_profile_samples(i, None, 0, C.byref(n)))
        ms = np.empty(max(n.value, 1), np.float32)
        _check(_lib.gnnav_profile_samples(i, _np_ptr(ms), n.value, None))
        out[buf.value.decode()] = ms[:n.value]
    return out


def profile_stop() -> dict:
    """Stop recording; {kernel name: (launches, total ms)}."""
    _check(_lib.gnnav_profile_stop())
    out = {}
    buf = C.create_string_buffer(128)
    for i in range(_lib.gnnav_profile_count()):
        n, ms = i64(), f64()
        _check(_lib.gnnav_profile_get(i, buf, 128, C.byref(n), C.byref(ms)))
        out[buf.value.decode()] = (n.value, ms.value)
    return out
