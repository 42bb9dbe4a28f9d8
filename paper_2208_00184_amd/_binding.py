"""Thin ctypes binding over libcel.so (the C ABI in include/cel.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  Arrays are torch tensors on a ROCm device; outputs are allocated
with torch on the same device and work is enqueued on the current torch
stream.  There is no CPU fallback: a missing library or a failed call raises.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from contextlib import nullcontext
from dataclasses import dataclass

import numpy as np
import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libcel.so")

OK, E_ARG, E_CYCLE, E_OVERFLOW, E_HIP, E_NOMEM, E_ORDER = 0, -1, -2, -3, -4, -5, -6
COMM_OFF = 1
CLUSTER_DP, CLUSTER_GREEDY = 0, 1

EXPORTS = ("cel_topo_levels", "cel_blevel", "cel_cpd_order", "cel_dfs_order", "cel_cluster", "cel_place", "cel_place_ext", "cel_makespan", "cel_makespan_noalloc",
           "cel_makespan_info", "cel_makespan_blocks_info", "cel_makespan_relax", "cel_blevel_info", "cel_policy_iteration",
           "cel_topo_levels_info", "cel_cluster_info",
           "cel_order_place", "cel_comm_sums", "cel_makespan_model", "cel_colocate",
           "cel_attention", "cel_attention_grad", "cel_attention_grad_scratch", "cel_embed", "cel_embed_grad", "cel_embed_grad_scratch", "cel_step_latency", "cel_timing", "cel_kernel_stats", "cel_last_error", "cel_version")


class CelError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libcel error {code}: {msg}")
        self.code = code


class _Graph(C.Structure):
    _fields_ = [("n", C.c_int32), ("m", C.c_int32),
                ("out_ptr", C.c_void_p), ("out_idx", C.c_void_p),
                ("in_ptr", C.c_void_p), ("in_idx", C.c_void_p),
                ("w", C.c_void_p), ("mem", C.c_void_p), ("ob", C.c_void_p)]


class _Hetero(C.Structure):
    _fields_ = [("tmul", C.POINTER(C.c_int64)), ("bw", C.POINTER(C.c_int64)),
                ("lat", C.POINTER(C.c_int64))]


class _Devices(C.Structure):
    _fields_ = [("D", C.c_int32), ("cap", C.POINTER(C.c_int64)),
                ("bw", C.c_int64), ("lat", C.c_int64)]


class _Rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("row", C.c_int64), ("head", C.c_int64)]


class _Attn(C.Structure):
    _fields_ = [("type", C.c_int32), ("tokens", C.c_int32), ("n_seq", C.c_int32),
                ("heads", C.c_int32), ("kv_heads", C.c_int32), ("dim", C.c_int32),
                ("scale", C.c_float), ("seq_ptr", C.c_void_p),
                ("q", _Rows), ("k", _Rows), ("v", _Rows)]


class _Embed(C.Structure):
    _fields_ = [("type", C.c_int32), ("id_bytes", C.c_int32),
                ("tokens", C.c_int64), ("vocab", C.c_int64), ("hidden", C.c_int64), ("stride", C.c_int64),
                ("ids", C.c_void_p), ("scale", C.c_float)]


_lib = None


def lib() -> C.CDLL:
    """Load libcel.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run __graft_entry__.build() "
                               "(or python -m paper_2208_00184_amd.build) first")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        G, Dv = C.POINTER(_Graph), C.POINTER(_Devices)
        L.cel_topo_levels.argtypes = [G, vp, vp, vp, C.POINTER(i32), vp]
        L.cel_blevel.argtypes = [G, Dv, vp, vp, vp, i32, i32, vp, vp, vp, C.POINTER(i64), vp]
        L.cel_cluster.argtypes = [G, Dv, vp, i32, i64, i32, vp, C.POINTER(i32), C.POINTER(i64), vp]
        L.cel_place.argtypes = [G, Dv, vp, i32, vp, vp, vp, C.POINTER(i64), C.POINTER(i32), vp]
        L.cel_place_ext.argtypes = [G, Dv, C.POINTER(_Hetero), vp, i32, vp, i32, vp, vp, vp,
                                    C.POINTER(i64), C.POINTER(i32), vp]
        L.cel_makespan.argtypes = [G, Dv, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp]
        L.cel_makespan_noalloc.argtypes = [G, Dv, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp]
        L.cel_cpd_order.argtypes = [G, vp, vp, vp, vp]
        L.cel_dfs_order.argtypes = [G, vp, vp]
        L.cel_order_place.argtypes = [G, Dv, vp, i32, vp, vp, C.POINTER(i32), vp]
        L.cel_comm_sums.argtypes = [G, Dv, vp, C.POINTER(i64), C.POINTER(i64), vp]
        L.cel_makespan_model.argtypes = [G, Dv, C.POINTER(_Hetero), vp, i32, vp, i32, vp, vp, vp, vp]
        L.cel_colocate.argtypes = [G, vp, vp, i32, i32, vp, vp]
        At, Ro = C.POINTER(_Attn), C.POINTER(_Rows)
        L.cel_attention.argtypes = [At, Ro, vp, vp]
        L.cel_attention_grad_scratch.argtypes = [At]
        L.cel_attention_grad_scratch.restype = i64
        L.cel_attention_grad.argtypes = [At, Ro, vp, Ro, vp, Ro, Ro, Ro, vp]
        Em = C.POINTER(_Embed)
        L.cel_embed.argtypes = [Em, vp, vp, vp]
        L.cel_embed_grad.argtypes = [Em, vp, vp, i32, vp, vp]
        L.cel_embed_grad_scratch.argtypes = [i64, i64, i64]
        L.cel_embed_grad_scratch.restype = i64
        for f in ("cel_topo_levels", "cel_blevel", "cel_cluster", "cel_place", "cel_place_ext",
                  "cel_makespan",
                  "cel_makespan_noalloc",
                  "cel_cpd_order", "cel_dfs_order", "cel_order_place", "cel_comm_sums", "cel_makespan_model",
                  "cel_colocate", "cel_attention", "cel_attention_grad", "cel_embed", "cel_embed_grad", "cel_version"):
            getattr(L, f).restype = C.c_int
        L.cel_last_error.argtypes = []
        L.cel_last_error.restype = C.c_char_p
        L.cel_step_latency.argtypes = [i32, i32, C.POINTER(C.c_double), vp]
        L.cel_step_latency.restype = C.c_int
        L.cel_timing.argtypes = [C.c_int]
        L.cel_timing.restype = C.c_int
        L.cel_kernel_stats.argtypes = [C.c_char_p, C.c_int, C.c_int]
        L.cel_kernel_stats.restype = C.c_int
        L.cel_makespan_info.argtypes = [C.POINTER(i32), C.POINTER(i32)]
        L.cel_makespan_info.restype = C.c_int
        L.cel_makespan_blocks_info.argtypes = [C.POINTER(i32)]
        L.cel_makespan_blocks_info.restype = C.c_int
        L.cel_makespan_relax.argtypes = [C.c_int]
        L.cel_makespan_relax.restype = C.c_int
        L.cel_blevel_info.argtypes = [C.POINTER(i32)]
        L.cel_blevel_info.restype = C.c_int
        L.cel_policy_iteration.argtypes = [C.c_int]
        L.cel_policy_iteration.restype = C.c_int
        L.cel_topo_levels_info.argtypes = [C.POINTER(i32)]
        L.cel_topo_levels_info.restype = C.c_int
        L.cel_cluster_info.argtypes = [C.POINTER(i32)]
        L.cel_cluster_info.restype = C.c_int
        _lib = L
    return _lib


def version() -> int:
    return lib().cel_version()


def step_latency(variant: int = 0, steps: int = 200000) -> float:
    """ns per dependent gather -> wave scan -> write step (variant 0: one wave
    over LDS; 1: 1024 threads with a barrier; 2: one wave gathering from L2)."""
    ns = C.c_double(0.0)
    _check(lib().cel_step_latency(int(variant), int(steps), C.byref(ns), _stream()))
    return ns.value


MS_PATH_RELAX, MS_PATH_SWEEP, MS_PATH_BATCH = 0, 1, 2


def makespan_info() -> tuple:
    """(path, rounds) of the calling thread's last makespan call: path 0 =
    relaxation over cross-device edges (exact after `rounds` rounds), 1 = the
    level sweep (after `rounds` relaxation rounds that did not converge), 2 =
    a batch (K > 1)."""
    path, rounds = C.c_int32(0), C.c_int32(0)
    _check(lib().cel_makespan_info(C.byref(path), C.byref(rounds)))
    return path.value, rounds.value


def makespan_blocks_info() -> tuple:
    """(path, iterations, blocks) of the calling thread's last makespan or
    makespan_model call: path 0 = blocks of tasks gave the result, 1 = another
    method did (iterations and blocks of a try that was given up, or 0); of the
    placement that took most of each."""
    info = (C.c_int32 * 3)()
    _check(lib().cel_makespan_blocks_info(info))
    return info[0], info[1], info[2]


def makespan_relax(mode: int) -> int:
    """K = 1 makespan path of the calling thread: 0 = the level sweep, 1 = the
    relaxation first (default), m >= 2 = the relaxation on at most m
    workgroups; returns the previous mode."""
    r = lib().cel_makespan_relax(int(mode))
    if r < 0:
        _check(r)
    return r


LP_POLICY, LP_SWEEP, LP_NONE = 0, 1, 2


def blevel_info() -> tuple:
    """((path, iterations) of the b-level, (path, iterations) of the t-level)
    of the calling thread's last blevel call: path 0 = policy iteration, 1 =
    the level sweep, 2 = not requested."""
    info = (C.c_int32 * 4)()
    _check(lib().cel_blevel_info(info))
    return (info[0], info[1]), (info[2], info[3])


def topo_levels_info() -> tuple:
    """(path, iterations) of the calling thread's last topo_levels call: path
    0 = policy iteration, 1 = Kahn's level-synchronous kernel."""
    info = (C.c_int32 * 2)()
    _check(lib().cel_topo_levels_info(info))
    return info[0], info[1]


def cluster_info() -> tuple:
    """(path, iterations) of the calling thread's last cluster call (DP mode):
    path 0 = policy iteration, 1 = the blocked DP."""
    info = (C.c_int32 * 2)()
    _check(lib().cel_cluster_info(info))
    return info[0], info[1]


def policy_iteration(mode: int) -> int:
    """Levels, b-level, t-level and clustering-DP path of the calling thread:
    0 = Kahn's kernel, the level sweeps and the blocked DP, 1 = policy
    iteration first (default; packed entries and asynchronous pointer jumping
    where the values fit), 2 = policy iteration first with 16-byte entries and
    synchronous rounds, 3 = as 1, but the clustering DP's iteration gives up at
    its first barrier (for tests); returns the previous mode."""
    r = lib().cel_policy_iteration(int(mode))
    if r < 0:
        _check(r)
    return r


def timing(enable: bool) -> bool:
    """Turn per-kernel event timing on/off; returns the previous setting."""
    return bool(lib().cel_timing(1 if enable else 0))


def kernel_stats(reset: bool = False) -> dict:
    """{kernel name: (launches, total_ms)} accumulated since the last reset."""
    buf = C.create_string_buffer(1 << 16)
    lib().cel_kernel_stats(buf, len(buf), 1 if reset else 0)
    out = {}
    for line in buf.value.decode().splitlines():
        name, cnt, ms = line.split()
        out[name] = (int(cnt), float(ms))
    return out


def _check(rc: int):
    if rc != OK:
        raise CelError(rc, lib().cel_last_error().decode(errors="replace"))


def _p(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


@dataclass
class Graph:
    """Device-resident operator DAG (int32 CSR/CSC, int64 w/mem/ob)."""
    n: int
    m: int
    out_ptr: torch.Tensor
    out_idx: torch.Tensor
    in_ptr: torch.Tensor
    in_idx: torch.Tensor
    w: torch.Tensor
    mem: torch.Tensor
    ob: torch.Tensor

    @staticmethod
    def from_arrays(wl, device="cuda") -> "Graph":
        """From any object with numpy fields n, m, out_ptr, ... (e.g. a Workload)."""
        def t(a, dt):
            return torch.from_numpy(np.ascontiguousarray(a, dtype=dt)).to(device)
        return Graph(int(wl.n), int(wl.m), t(wl.out_ptr, np.int32), t(wl.out_idx, np.int32),
                     t(wl.in_ptr, np.int32), t(wl.in_idx, np.int32), t(wl.w, np.int64),
                     t(wl.mem, np.int64), t(wl.ob, np.int64))

    @property
    def device(self):
        return self.out_ptr.device

    def _c(self) -> _Graph:
        return _Graph(self.n, self.m, self.out_ptr.data_ptr(), self.out_idx.data_ptr(),
                      self.in_ptr.data_ptr(), self.in_idx.data_ptr(), self.w.data_ptr(),
                      self.mem.data_ptr(), self.ob.data_ptr())


@dataclass
class Devices:
    """Modelled target devices: count, host memory caps, link bw (B/ns) and latency (ns)."""
    D: int
    cap: np.ndarray
    bw: int
    lat: int

    @staticmethod
    def from_arrays(wl) -> "Devices":
        return Devices(int(wl.D), np.ascontiguousarray(wl.cap, np.int64), int(wl.bw), int(wl.lat))

    def _c(self) -> _Devices:
        self._cap = np.ascontiguousarray(self.cap, np.int64)  # keep alive during the call
        return _Devices(int(self.D), self._cap.ctypes.data_as(C.POINTER(C.c_int64)),
                        int(self.bw), int(self.lat))


def _empty(n, dtype, device):
    return torch.empty(max(int(n), 1), dtype=dtype, device=device)


def topo_levels(g: Graph):
    """-> (level int32[n], order_id int32[n], level_ptr int32[L+1], L)"""
    n = g.n
    level = _empty(n, torch.int32, g.device)
    order = _empty(n, torch.int32, g.device)
    lptr = torch.empty(n + 1, dtype=torch.int32, device=g.device)
    L = C.c_int32(0)
    gc = g._c()
    _check(lib().cel_topo_levels(C.byref(gc), _p(level), _p(order), _p(lptr), C.byref(L),
                                 _stream()))
    return level[:n], order[:n], lptr[:L.value + 1], L.value


def blevel(g: Graph, d: Devices, level, level_ptr, order_id, n_levels, comm_off=False,
           want_tlevel=False, want_prio=True):
    """-> (blevel int64[n], tlevel int64[n] | None, prio_order int32[n] | None, cp)"""
    n = g.n
    bl = _empty(n, torch.int64, g.device)
    tl = _empty(n, torch.int64, g.device) if want_tlevel else None
    pr = _empty(n, torch.int32, g.device) if want_prio else None
    cp = C.c_int64(0)
    gc, dc = g._c(), d._c()
    _check(lib().cel_blevel(C.byref(gc), C.byref(dc), _p(level), _p(level_ptr), _p(order_id),
                            int(n_levels), COMM_OFF if comm_off else 0, _p(bl), _p(tl), _p(pr),
                            C.byref(cp), _stream()))
    return bl[:n], (tl[:n] if tl is not None else None), (pr[:n] if pr is not None else None), \
        cp.value


def cpd_order(g: Graph, blevel_, tlevel_):
    """CPD-TOPO order (Algorithm 1) from b-/t-levels -> int32[n] node ids."""
    n = g.n
    out = _empty(n, torch.int32, g.device)
    gc = g._c()
    _check(lib().cel_cpd_order(C.byref(gc), _p(blevel_), _p(tlevel_), _p(out), _stream()))
    return out[:n]


def dfs_order(g: Graph):
    """DFS-TOPO order (Section 4.2.2) -> int32[n] node ids."""
    n = g.n
    out = _empty(n, torch.int32, g.device)
    gc = g._c()
    _check(lib().cel_dfs_order(C.byref(gc), _p(out), _stream()))
    return out[:n]


def cluster(g: Graph, d: Devices, order, R=200, M=-1, mode=CLUSTER_DP):
    """-> (cluster_id int32[n], n_clusters, cut_cost)"""
    n = g.n
    cid = _empty(n, torch.int32, g.device)
    nc = C.c_int32(0)
    cut = C.c_int64(0)
    gc, dc = g._c(), d._c()
    _check(lib().cel_cluster(C.byref(gc), C.byref(dc), _p(order), int(R), int(M), int(mode),
                             _p(cid), C.byref(nc), C.byref(cut), _stream()))
    return cid[:n], nc.value, cut.value


def place(g: Graph, d: Devices, cluster_id, n_clusters, want_fin=False):
    """-> (cluster_dev uint8[C], node_dev uint8[n], coarse_makespan, best_effort_count)
    plus cluster_fin int64[C] when ``want_fin``."""
    n = g.n
    cdev = _empty(n_clusters, torch.uint8, g.device)
    ndev = _empty(n, torch.uint8, g.device)
    fin = _empty(n_clusters, torch.int64, g.device) if want_fin else None
    span = C.c_int64(0)
    be = C.c_int32(0)
    gc, dc = g._c(), d._c()
    _check(lib().cel_place(C.byref(gc), C.byref(dc), _p(cluster_id), int(n_clusters), _p(cdev),
                           _p(ndev), _p(fin), C.byref(span), C.byref(be), _stream()))
    out = (cdev[:n_clusters], ndev[:n], span.value, be.value)
    return out + (fin[:n_clusters],) if want_fin else out


def order_place(g: Graph, d: Devices, cluster_id, n_clusters):
    """Order-Place -> (cluster_dev uint8[C], node_dev uint8[n], best_effort_count)"""
    n = g.n
    cdev = _empty(n_clusters, torch.uint8, g.device)
    ndev = _empty(n, torch.uint8, g.device)
    be = C.c_int32(0)
    gc, dc = g._c(), d._c()
    _check(lib().cel_order_place(C.byref(gc), C.byref(dc), _p(cluster_id), int(n_clusters), _p(cdev),
                                 _p(ndev), C.byref(be), _stream()))
    return cdev[:n_clusters], ndev[:n], be.value


MODEL_INSERT, MODEL_COMM_TASKS, MODEL_COMM_BLOCK = 1, 2, 4


def _hetero(tmul, bw, lat, keep):
    """cel_hetero over host copies (kept alive in `keep`), or None."""
    if tmul is None and bw is None and lat is None:
        return None
    ptrs = []
    for a in (tmul, bw, lat):
        if a is None:
            ptrs.append(None)
            continue
        arr = (C.c_int64 * int(np.asarray(a).size))(*[int(x) for x in np.asarray(a).reshape(-1)])
        keep.append(arr)
        ptrs.append(C.cast(arr, C.POINTER(C.c_int64)))
    return _Hetero(*ptrs)


def place_ext(g: Graph, d: Devices, cluster_id, n_clusters, tmul=None, bw=None, lat=None,
              group=None, n_groups=0):
    """Adjusting Placement with heterogeneous devices/links (host tmul [D], bw / lat
    [D, D]) and co-location groups (device int32 [n] in [-1, n_groups)) inside the
    algorithm -> (cluster_dev, node_dev, coarse_makespan, best_effort_count, cluster_fin)."""
    keep = []
    het = _hetero(tmul, bw, lat, keep)
    n = g.n
    cdev = _empty(n_clusters, torch.uint8, g.device)
    ndev = _empty(n, torch.uint8, g.device)
    fin = _empty(n_clusters, torch.int64, g.device)
    span = C.c_int64(0)
    be = C.c_int32(0)
    gc, dc = g._c(), d._c()
    _check(lib().cel_place_ext(C.byref(gc), C.byref(dc), None if het is None else C.byref(het),
                               _p(group), int(n_groups), _p(cluster_id), int(n_clusters), _p(cdev),
                               _p(ndev), _p(fin), C.byref(span), C.byref(be), _stream()))
    return cdev[:n_clusters], ndev[:n], span.value, be.value, fin[:n_clusters]


def makespan_model(g: Graph, d: Devices, order, node_dev, model, want_times=False, tmul=None,
                   bw=None, lat=None):
    """Makespan under the device models (MODEL_* bits; 0 = FIFO devices, contention-free
    comm). node_dev uint8 [n] or [K, n] -> (makespan int64[K], start, finish) ([K, n] or None).
    tmul [D], bw / lat [D, D]: heterogeneous devices (host values, time x tmul / 1024)."""
    keep = []
    het = _hetero(tmul, bw, lat, keep)
    n = g.n
    nd = node_dev.contiguous()
    K = 1 if nd.dim() == 1 else nd.shape[0]
    ms = torch.empty(K, dtype=torch.int64, device=g.device)
    st = torch.empty((K, max(n, 1)), dtype=torch.int64, device=g.device) if want_times else None
    fi = torch.empty((K, max(n, 1)), dtype=torch.int64, device=g.device) if want_times else None
    gc, dc = g._c(), d._c()
    _check(lib().cel_makespan_model(C.byref(gc), C.byref(dc), None if het is None else C.byref(het),
                                    _p(order), int(K), _p(nd), int(model), _p(st), _p(fi), _p(ms),
                                    _stream()))
    if want_times:
        st, fi = st[:, :n], fi[:, :n]
    return ms, st, fi


def colocate(g: Graph, order, group, n_groups, node_dev):
    """Co-location groups: node_dev (uint8 [n] or [K, n], device) rewritten in place so that
    every group follows its first node in `order`; returns node_dev."""
    nd = node_dev
    assert nd.is_contiguous()
    K = 1 if nd.dim() == 1 else nd.shape[0]
    gc = g._c()
    _check(lib().cel_colocate(C.byref(gc), _p(order), _p(group), int(n_groups), int(K), _p(nd),
                              _stream()))
    return nd


def comm_sums(g: Graph, d: Devices, cluster_id=None):
    """CCR parts (eq. 1) -> (edge comm, total w); with cluster_id only edges between clusters."""
    ec = C.c_int64(0)
    ws = C.c_int64(0)
    gc, dc = g._c(), d._c()
    _check(lib().cel_comm_sums(C.byref(gc), C.byref(dc), _p(cluster_id), C.byref(ec), C.byref(ws),
                               _stream()))
    return ec.value, ws.value


def makespan(g: Graph, d: Devices, order, level, level_ptr, n_levels, node_dev, want_times=False,
             noalloc=False):
    """node_dev uint8 [n] or [K, n] -> (makespan int64[K], start, finish) ([K, n] or None).
    noalloc=True calls cel_makespan_noalloc (the library allocates nothing;
    the outputs are still allocated here by torch)."""
    n = g.n
    nd = node_dev.contiguous()
    K = 1 if nd.dim() == 1 else nd.shape[0]
    ms = torch.empty(K, dtype=torch.int64, device=g.device)
    st = torch.empty((K, max(n, 1)), dtype=torch.int64, device=g.device) if want_times else None
    fi = torch.empty((K, max(n, 1)), dtype=torch.int64, device=g.device) if want_times else None
    gc, dc = g._c(), d._c()
    f = lib().cel_makespan_noalloc if noalloc else lib().cel_makespan
    _check(f(C.byref(gc), C.byref(dc), _p(order), _p(level), _p(level_ptr), int(n_levels), int(K),
             _p(nd), _p(st), _p(fi), _p(ms), _stream()))
    if want_times:
        st, fi = st[:, :n], fi[:, :n]
    return ms, st, fi


# ---------------------------------------------- operations of a training step
# They enqueue their work on the current stream of the tensors' device and
# return; outputs and scratch come from torch's allocator on that stream.  An
# input that another stream fills or frees is the caller's to order, as with
# any torch operation.  They record nothing for torch's automatic gradients, and
# refuse tensors that ask for one, unless those are switched off
# (torch.no_grad(), or inside a torch.autograd.Function).

_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


def _refuse(what):
    raise CelError(E_ARG, what)


def _on(index):
    """The device as the current one for the launches of a call."""
    return nullcontext() if index == torch.cuda.current_device() else torch.cuda.device(index)


def _raw_stream(index):
    """The handle of the device's current stream."""
    return torch._C._cuda_getCurrentRawStream(index)


def _device_of(fn, **tensors):
    """The index of the ROCm device that all of them are on.  None may ask for a gradient: results
    would be cut off from it without a sign."""
    index, graph = -1, torch.is_grad_enabled()
    for name, t in tensors.items():
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            _refuse(f"{fn}: {name} is not a tensor on a ROCm device")
        at = t.get_device()
        if index >= 0 and at != index:
            _refuse(f"{fn}: {name} is on device {at}, not on {index}")
        if graph and t.requires_grad:
            _refuse(f"{fn}: {name} requires a gradient, which is not recorded: call under torch.no_grad()")
        index = at
    return index


def _view(t):
    """t [tokens, heads, dim] as the kernels read and write it, or None where its values are not
    contiguous or its address or strides are off 16 bytes.  A single token's and a single head's stride
    is never taken, whatever it says."""
    row, head, one = t.stride()
    T, H, d = t.shape
    p = t.data_ptr()
    if T == 1:
        row = d
    if H == 1:
        head = 0
    if one != 1 or row & 7 or head & 7 or p & 15 or not d <= row <= 1 << 23:
        return None
    return _Rows(p, row, head)


def _views(*tensors):
    """Views to read, of copies where need be -> (views, tensors to keep alive)."""
    views, keep = [], []
    for t in tensors:
        x = _view(t)
        if x is None:
            t = t.clone(memory_format=torch.contiguous_format)
            x = _Rows(t.data_ptr(), t.shape[1] * t.shape[2], t.shape[2])
        views.append(x)
        keep.append(t)
    return views, keep


def _block(x, T, H, d):
    """A view's (first element, element behind its last, row stride, head stride, heads)."""
    at, row, head = (x.p or 0) // 2, x.row, x.head
    return at, at + (T - 1) * row + (H - 1) * head + d, row, head, H


def _folded(x, T, d):
    """Whether elements of a block share memory."""
    if x[2] >= (x[4] - 1) * x[3] + d and (x[3] >= d or x[4] == 1):
        return False  # heads side by side, rows one behind the other
    (lo, n), (hi, m) = sorted([(s, k) for s, k in ((x[3], x[4]), (x[2], T)) if k > 1] + [(1 << 62, 1)] * 2)[:2]
    if n == 1:
        return False
    if lo < d or m == 1:
        return lo < d
    for a in range(1, min(m, ((n - 1) * lo + d - 1) // hi + 1)):  # a large steps against the nearest small ones
        b, off = divmod(a * hi, lo)
        if (off < d and b < n) or (lo - off < d and b + 1 < n):
            return True
    return False


def _meet(x, y, T, d):
    """Whether two blocks share memory.  Of blocks that interleave with different row strides only
    those with the same first element are known to."""
    if x[1] <= y[0] or y[1] <= x[0]:
        return False
    g = math.gcd(x[2], x[3], y[2], y[3])  # all steps are multiples of it
    if d <= (x[0] - y[0]) % g <= g - d:
        return False
    row = x[2]
    if y[2] != row:
        return x[0] == y[0]
    parts = []
    for at, _, _, head, heads in (x, y):  # the heads of a row as one piece, where they fit in it
        width = (heads - 1) * head + d
        parts.append([(at, width)] if width <= row else [(at + h * head, d) for h in range(heads)])
    for whole in (True, False):
        if not any(-w < a - b - s * row < v and -T < s < T
                   for a, w in parts[0] for b, v in parts[1] for s in ((a - b) // row, (a - b) // row + 1)):
            return False
        if whole:
            parts = [[(at + h * head, d) for h in range(heads)] for at, _, _, head, heads in (x, y)]
    return True


def _attn(fn, q, k, v, seq_ptr, scale):
    """-> (descriptor, tensors to keep alive)"""
    if q.dim() != 3 or k.dim() != 3 or v.dim() != 3 or q.dtype not in (torch.bfloat16, torch.float16) or \
            k.dtype != q.dtype or v.dtype != q.dtype:
        _refuse(f"{fn}: q, k and v are not [tokens, heads, dim] in bfloat16 or in float16")
    T, H, d = q.shape
    shape = k.shape
    if v.shape != shape or shape[0] != T or shape[2] != d:
        _refuse(f"{fn}: shapes q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}")
    if seq_ptr.dim() != 1 or seq_ptr.dtype != torch.int32 or seq_ptr.numel() < 1:
        _refuse(f"{fn}: seq_ptr is not int32 [sequences + 1]")
    if T >= 1 << 31:
        _refuse(f"{fn}: {T} tokens")
    (qv, kv, vv), keep = _views(q, k, v)
    seq_ptr = seq_ptr.contiguous()
    keep.append(seq_ptr)
    return _Attn(_TYPES[q.dtype], T, seq_ptr.numel() - 1, H, shape[1], d,
                 (d or 1) ** -0.5 if scale is None else scale, seq_ptr.data_ptr(), qv, kv, vv), keep


def attention(q, k, v, seq_ptr, scale=None):
    """Causal attention over a packed batch: sequence s is the tokens seq_ptr[s] ..
    seq_ptr[s + 1] - 1 (int32, on the device), a token sees itself and the earlier tokens of its
    sequence.  q [T, heads, dim], k and v [T, kv_heads, dim] in bfloat16 or float16, any strides
    (views of a fused projection are read in place; where a head's values are not contiguous, or an
    address or stride is no multiple of 16 bytes, the call copies the tensor); heads a multiple of
    kv_heads, dim a multiple of 8 up to 128; scale: of the scores, 1 / sqrt(dim) by default.
    -> (out [T, heads, dim], lse float32 [heads, T]); tokens of no sequence have 0 and -inf."""
    index = _device_of("attention", q=q, k=k, v=v, seq_ptr=seq_ptr)
    with _on(index):
        a, keep = _attn("attention", q, k, v, seq_ptr, scale)
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty((a.heads, a.tokens), dtype=torch.float32, device=q.device)
        rows = _Rows(out.data_ptr(), a.heads * a.dim, a.dim)
        _check(lib().cel_attention(C.byref(a), C.byref(rows), lse.data_ptr(), _raw_stream(index)))
    return out, lse


def attention_grad(dout, q, k, v, out, lse, seq_ptr, scale=None, grads=None):
    """The gradient of attention() at dout [T, heads, dim], with its out and lse.
    -> (dq, dk, dv) as q, k, v are shaped.  grads: three tensors to write them to (for instance views
    of one fused gradient; values contiguous, addresses and strides multiples of 16 bytes; no memory
    shared with an input, with each other or within one).  The same inputs give the same bits."""
    fn = "attention_grad"
    index = _device_of(fn, q=q, k=k, v=v, seq_ptr=seq_ptr, dout=dout, out=out, lse=lse)
    with _on(index):
        a, keep = _attn(fn, q, k, v, seq_ptr, scale)
        for name, t in (("dout", dout), ("out", out)):
            if t.shape != q.shape or t.dtype != q.dtype:
                _refuse(f"{fn}: {name} is {tuple(t.shape)} {t.dtype}, not as q")
        if lse.shape != (a.heads, a.tokens) or lse.dtype != torch.float32:
            _refuse(f"{fn}: lse is not float32 [heads, tokens]")
        (gv, ov), keep2 = _views(dout, out)
        lse = lse.contiguous()
        given = grads is not None
        if not given:
            grads = tuple(torch.empty(t.shape, dtype=q.dtype, device=q.device) for t in (q, k, v))
        elif len(grads) != 3:
            _refuse(f"{fn}: grads are not three tensors")
        else:
            _device_of(fn, q=q, dq=grads[0], dk=grads[1], dv=grads[2])
        views = []
        for name, t, x in zip(("dq", "dk", "dv"), grads, (q, k, v)):
            view = _view(t) if t.shape == x.shape and t.dtype == q.dtype else None
            if view is None and t.numel():
                _refuse(f"{fn}: {name} cannot be written in place: {tuple(t.shape)} {t.dtype}, strides {t.stride()}")
            views.append(view or _Rows())
        if given and a.tokens:
            T, d, heads = a.tokens, a.dim, (a.heads, a.kv_heads, a.kv_heads)
            blocks = [_block(x, T, n, d) for x, n in zip(views, heads)]
            others = [(name, _block(x, T, n, d)) for name, x, n in zip(
                ("q", "k", "v", "out", "dout"), (a.q, a.k, a.v, ov, gv), heads + (heads[0], heads[0]))]
            first, last = min(x[0] for x in blocks), max(x[1] for x in blocks)
            others = [y for y in others if y[1][0] < last and first < y[1][1]]
            for name, x in zip(("dq", "dk", "dv"), blocks):
                if _folded(x, T, d):
                    _refuse(f"{fn}: values of {name} share memory")
                for other, y in others:
                    if _meet(x, y, T, d):
                        _refuse(f"{fn}: {name} shares memory with {other}")
                others.append((name, x))
        size = lib().cel_attention_grad_scratch(C.byref(a))
        if size < 0:
            _check(size)
        scratch = torch.empty(size, dtype=torch.uint8, device=q.device)
        _check(lib().cel_attention_grad(C.byref(a), C.byref(ov), lse.data_ptr(), C.byref(gv), scratch.data_ptr(), *map(C.byref, views),
                                        _raw_stream(index)))
    return tuple(grads)


def _embed(fn, what, rows, ids, vocab, scale):
    """-> (descriptor, rows with contiguous values, ids): checks that embed and embed_grad share."""
    if rows.dim() != 2 or rows.dtype not in _TYPES:
        _refuse(f"{fn}: {what} is not [rows, hidden] in bfloat16, float16 or float32")
    if ids.dim() != 1 or ids.dtype not in (torch.int32, torch.int64):
        _refuse(f"{fn}: ids are not int32 or int64 [tokens]")
    h = rows.shape[1]
    stride, one = rows.stride()
    if rows.shape[0] <= 1:
        stride = h
    if (h > 1 and one != 1) or stride < h:
        rows, stride = rows.clone(memory_format=torch.contiguous_format), h
    ids = ids.contiguous()
    return _Embed(_TYPES[rows.dtype], ids.element_size(), ids.numel(), vocab, h, stride, ids.data_ptr(),
                  float(scale)), rows, ids


def embed(table, ids, scale=1.0):
    """scale * table[ids]: rows of table [vocab, hidden] (bfloat16, float16 or float32, rows any
    stride apart) by token id (int32 or int64 [tokens]); an id outside [0, vocab) is padding, a row
    of zeros. -> [tokens, hidden] in the table's type.  A table whose rows' values are not contiguous
    (a transposed one) or overlap (an expanded one) is copied whole by every call."""
    index = _device_of("embed", table=table, ids=ids)
    with _on(index):
        a, table, ids = _embed("embed", "table", table, ids, table.shape[0] if table.dim() else 0, scale)
        out = torch.empty((a.tokens, a.hidden), dtype=table.dtype, device=table.device)
        _check(lib().cel_embed(C.byref(a), table.data_ptr(), out.data_ptr(), _raw_stream(index)))
    return out


def embed_grad(dx, ids, vocab, scale=1.0, dtype=None):
    """The gradient of embed()'s table at dx [tokens, hidden], the gradient of its rows: a dense
    [vocab, hidden] in `dtype` (dx's by default, or float32), zeros for words that do not occur.
    The tokens are sorted by id and added in 32 bits in a fixed order: the same inputs give the
    same bits.  A dx whose rows' values are not contiguous or overlap is copied by the call."""
    fn = "embed_grad"
    index = _device_of(fn, dx=dx, ids=ids)
    with _on(index):
        a, dx, ids = _embed(fn, "dx", dx, ids, int(vocab), scale)
        if a.tokens != dx.shape[0]:
            _refuse(f"{fn}: {a.tokens} ids of {dx.shape[0]} rows")
        dtype = dx.dtype if dtype is None else dtype
        if dtype not in (dx.dtype, torch.float32):
            _refuse(f"{fn}: a gradient in {dtype} of rows in {dx.dtype}")
        size = lib().cel_embed_grad_scratch(a.tokens, int(vocab), a.hidden)
        if size < 0:
            _check(size)
        work = torch.empty(size, dtype=torch.uint8, device=dx.device)
        grad = torch.empty((int(vocab), a.hidden), dtype=dtype, device=dx.device)
        _check(lib().cel_embed_grad(C.byref(a), dx.data_ptr(), work.data_ptr(), _TYPES[dtype], grad.data_ptr(),
                                    _raw_stream(index)))
    return grad
