"""ctypes binding of liba2a_topo.so: same names as include/a2a_topo.h, marshalling only.

Device buffers are torch tensors (PyTorch is used for device memory and streams, nothing
else); their ``data_ptr()`` and the current stream's handle cross the C ABI as plain pointers.
"""
from __future__ import annotations

import ctypes
import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
_CSRC = os.path.join(_HERE, "csrc")
_LIB = os.path.join(_HERE, "liba2a_topo.so")
_lib = None

OK = 0
ERR_INVALID_ARG = -1
ERR_SELF_LOOP = -2
ERR_WORKSPACE_TOO_SMALL = -3
ERR_HIP = -4
ERR_NOT_IMPLEMENTED = -5
ERR_DISCONNECTED = -6
ERR_NO_MEMORY = -7
ERR_LEVEL_OVERFLOW = -8

WS_DISTANCES = 0x0
WS_SIGMA = 0x1
WS_LOADS = 0x2
WS_SSSP = 0x4
WS_COSTS = 0x8
WS_MINIMAL = 0x100
FLAG_SIGMA_INEXACT = 0x1
FLAG_UNREACHABLE = 0x2

EXPORTED_SYMBOLS = (
    "a2a_topo_create", "a2a_topo_destroy", "a2a_topo_info", "a2a_workspace_bytes",
    "a2a_distances", "a2a_link_loads", "a2a_link_loads_demand", "a2a_schedule_bound", "a2a_status_string",
    "a2a_profile_enable", "a2a_profile_read", "a2a_tree_lower_bound", "a2a_schedule_bound_cap",
    "a2a_link_loads_static", "a2a_sssp_loads", "a2a_path_costs", "a2a_dispatch_counts", "a2a_dispatch_demand",
    "a2a_balance_workspace_bytes", "a2a_balance_loss", "a2a_balance_loss_grad",
)
MOST_EXPERTS = 4096
STATIC_WORKSPACE_BYTES = 32 << 20

PROF_KERNELS = ("init", "bfs", "offsets", "fwd_rows", "fwd_few", "fwd_spread", "bwd_rows", "bwd_few", "bwd_spread",
                "reduce", "extract", "search", "sources", "tokens")
PROF_MAX_LEVELS = 64

HIPCC_FLAGS = [
    "-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


class A2AError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class Bound(ctypes.Structure):
    """Mirror of ``a2a_bound``."""
    _fields_ = [
        ("max_load", ctypes.c_double), ("argmax_arc", ctypes.c_int64), ("min_load", ctypes.c_double),
        ("sum_dist", ctypes.c_int64), ("n_links", ctypes.c_int64), ("n_nodes", ctypes.c_int32),
        ("dmax", ctypes.c_int32), ("t_sched", ctypes.c_double), ("t_lb_nd", ctypes.c_double),
        ("t_lb_links", ctypes.c_double), ("ratio", ctypes.c_double), ("throughput", ctypes.c_double),
        ("flow_value", ctypes.c_double), ("throughput_upper", ctypes.c_double),
    ]

    def as_dict(self) -> dict:
        return {n: getattr(self, n) for n, _ in self._fields_}


class BoundCap(ctypes.Structure):
    """Mirror of ``a2a_bound_cap``."""
    _fields_ = [
        ("max_util", ctypes.c_double), ("argmax_arc", ctypes.c_int64), ("min_util", ctypes.c_double),
        ("sum_dist", ctypes.c_int64), ("n_links", ctypes.c_int64), ("n_nodes", ctypes.c_int32),
        ("reserved", ctypes.c_int32), ("total_capacity", ctypes.c_double),
        ("max_node_capacity", ctypes.c_double), ("t_sched", ctypes.c_double), ("t_lb_nd", ctypes.c_double),
        ("t_lb_links", ctypes.c_double), ("ratio", ctypes.c_double), ("throughput", ctypes.c_double),
        ("flow_value", ctypes.c_double), ("throughput_upper", ctypes.c_double),
    ]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_ if n != "reserved"}


class TreeBound(ctypes.Structure):
    """Mirror of ``a2a_tree_bound``."""
    _fields_ = [("s_min", ctypes.c_int64), ("height", ctypes.c_int32), ("full", ctypes.c_int32),
                ("t_lb", ctypes.c_double), ("throughput_ub", ctypes.c_double)]


class Profile(ctypes.Structure):
    """Mirror of ``a2a_profile``."""
    _fields_ = [("ms", ctypes.c_double * 16), ("launches", ctypes.c_int64 * 16),
                ("ms_level", (ctypes.c_double * PROF_MAX_LEVELS) * 16),
                ("pairs_level", ctypes.c_int64 * PROF_MAX_LEVELS),
                ("dag_level", ctypes.c_int64 * PROF_MAX_LEVELS),
                ("dag_links", ctypes.c_int64), ("calls", ctypes.c_int64),
                ("depth", ctypes.c_int32), ("groups", ctypes.c_int32), ("narrow_levels", ctypes.c_uint64),
                ("fwd_flavours", ctypes.c_uint64), ("bwd_flavours", ctypes.c_uint64)]

    def as_dict(self) -> dict:
        d = {"dag_links": self.dag_links, "calls": self.calls, "depth": self.depth,
             "groups": self.groups, "narrow_levels": self.narrow_levels, "fwd_flavours": self.fwd_flavours,
             "bwd_flavours": self.bwd_flavours, "pairs_level": list(self.pairs_level),
             "dag_level": list(self.dag_level)}
        for i, n in enumerate(PROF_KERNELS):
            d[n] = {"ms": self.ms[i], "launches": self.launches[i], "ms_level": list(self.ms_level[i])}
        return d


class Routing(ctypes.Structure):
    """Mirror of ``a2a_routing``."""
    _fields_ = [("tokens", ctypes.c_int64), ("choices_per_token", ctypes.c_int32), ("experts", ctypes.c_int32),
                ("choices_type", ctypes.c_int32), ("reserved", ctypes.c_int32), ("choices", ctypes.c_void_p),
                ("choices_stride", ctypes.c_int64), ("host_begin", ctypes.c_void_p), ("expert_host", ctypes.c_void_p)]


def library_path() -> str:
    return _LIB


def build_library(verbose: bool = False) -> str:
    """Compile csrc/ for gfx950 with hipcc (works without a GPU): the host side with the level kernels, and the kernels
    for each width of the link tables, side by side."""
    global _lib
    flags = [*HIPCC_FLAGS, "-I" + os.path.join(_ROOT, "include")]
    with tempfile.TemporaryDirectory() as tmp:
        units = [("a2a_topo", [])] + [("a2a_words", [f"-DA2A_WORDS={w}"]) for w in (2, 3, 4, 5, 8)]
        objects = [os.path.join(tmp, f"{i}.o") for i in range(len(units))]

        def compile_unit(i):
            name, extra = units[i]
            return _run(["hipcc", *flags, *extra, "-c", "-o", objects[i], os.path.join(_CSRC, name + ".hip")], verbose)

        with ThreadPoolExecutor(max_workers=min(len(units), os.cpu_count() or 1)) as pool:
            list(pool.map(compile_unit, range(len(units))))
        _run(["hipcc", "--offload-arch=gfx950", "-shared", "-o", _LIB, *objects], verbose)
    _lib = None
    return _LIB


def _run(cmd, verbose: bool) -> None:
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if verbose or res.returncode != 0:
        print(res.stdout)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + res.stdout)


def load_library():
    """Load liba2a_topo.so; raises if it has not been built (there is no fallback path)."""
    global _lib, _torch
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB):
        raise RuntimeError(
            f"{_LIB} is missing: build it with paper_2309_13541_amd.build_library() "
            "(or __graft_entry__.build()); there is no CPU fallback")
    # PyTorch ships its own HIP runtime (same soname as the system one).  It has to be in the
    # process first, so that this library binds to the runtime that owns torch's tensors and
    # streams instead of bringing in a second one.
    import torch
    _torch = torch
    _type_codes.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, torch.int32: 3, torch.int64: 4})
    lib = ctypes.CDLL(_LIB)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.a2a_topo_create.restype = ctypes.c_int
    lib.a2a_topo_create.argtypes = [i32, vp, vp, ctypes.POINTER(vp)]
    lib.a2a_topo_destroy.restype = None
    lib.a2a_topo_destroy.argtypes = [vp]
    lib.a2a_topo_info.restype = ctypes.c_int
    lib.a2a_topo_info.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i64), ctypes.POINTER(i32),
                                  ctypes.POINTER(i32)]
    lib.a2a_workspace_bytes.restype = sz
    lib.a2a_workspace_bytes.argtypes = [vp, i32, ctypes.c_int]
    lib.a2a_distances.restype = ctypes.c_int
    lib.a2a_distances.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.a2a_link_loads.restype = ctypes.c_int
    lib.a2a_link_loads.argtypes = [vp, i32, i32, vp, vp, vp, vp, sz, vp]
    lib.a2a_link_loads_static.restype = ctypes.c_int
    lib.a2a_link_loads_static.argtypes = [vp, i32, i32, vp, vp, vp, vp]
    lib.a2a_sssp_loads.restype = ctypes.c_int
    lib.a2a_sssp_loads.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, sz, vp]
    lib.a2a_link_loads_demand.restype = ctypes.c_int
    lib.a2a_link_loads_demand.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.a2a_path_costs.restype = ctypes.c_int
    lib.a2a_path_costs.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.a2a_dispatch_counts.restype = ctypes.c_int
    lib.a2a_dispatch_counts.argtypes = [vp, i32, ctypes.POINTER(Routing), vp, vp]
    lib.a2a_dispatch_demand.restype = ctypes.c_int
    lib.a2a_dispatch_demand.argtypes = [vp, i32, ctypes.POINTER(Routing), ctypes.c_int, vp, vp]
    lib.a2a_balance_workspace_bytes.restype = sz
    lib.a2a_balance_workspace_bytes.argtypes = [vp, i32, i64, i32]
    lib.a2a_balance_loss.restype = ctypes.c_int
    lib.a2a_balance_loss.argtypes = [vp, i32, ctypes.POINTER(Routing), vp, ctypes.c_int, i64, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.a2a_balance_loss_grad.restype = ctypes.c_int
    lib.a2a_balance_loss_grad.argtypes = [vp, i32, ctypes.POINTER(Routing), vp, ctypes.c_int, i64, vp, vp, vp, vp, vp, i64, vp]
    lib.a2a_schedule_bound_cap.restype = ctypes.c_int
    lib.a2a_schedule_bound_cap.argtypes = [vp, vp, vp, i64, i64, ctypes.c_double, ctypes.c_double, vp, vp]
    lib.a2a_schedule_bound.restype = ctypes.c_int
    lib.a2a_schedule_bound.argtypes = [vp, vp, i64, i64, ctypes.c_double, ctypes.c_double,
                                       ctypes.POINTER(Bound), vp]
    lib.a2a_profile_enable.restype = ctypes.c_int
    lib.a2a_profile_enable.argtypes = [vp, ctypes.c_int]
    lib.a2a_profile_read.restype = ctypes.c_int
    lib.a2a_profile_read.argtypes = [vp, ctypes.POINTER(Profile)]
    lib.a2a_tree_lower_bound.restype = ctypes.c_int
    lib.a2a_tree_lower_bound.argtypes = [i32, i32, ctypes.c_double, ctypes.c_double, ctypes.POINTER(TreeBound)]
    lib.a2a_status_string.restype = ctypes.c_char_p
    lib.a2a_status_string.argtypes = [ctypes.c_int]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().a2a_status_string(int(status)).decode()


def tree_lower_bound(N: int, d: int, m_bytes: float = 1.0, b_bytes_per_s: float = 1.0) -> TreeBound:
    """a2a_tree_lower_bound: Theorem 1's bound for any N-host, degree-d topology (host arithmetic)."""
    out = TreeBound()
    _check(load_library().a2a_tree_lower_bound(int(N), int(d), float(m_bytes), float(b_bytes_per_s),
                                               ctypes.byref(out)), "a2a_tree_lower_bound")
    return out


def _check(status: int, where: str, allow=()):
    if status != OK and status not in allow:
        raise A2AError(status, where)
    return status


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


_torch = None    # the module, once the library is loaded
_type_codes = {}  # a2a_type of a torch type


def _device() -> int:
    """The current device."""
    load_library()
    return _torch._C._cuda_getDevice()


def _refuse(where: str, why: str):
    raise A2AError(ERR_INVALID_ARG, f"{where}: {why}")


def _whole(where: str, device: int, name: str, t, dtype, shape) -> int:
    """Address of a contiguous tensor of that type and shape on the current device."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        _refuse(where, f"{name} has to be a contiguous {dtype} tensor of shape {tuple(shape)} on the current device")
    return t.data_ptr()


def _workspace(where: str, device: int, t):
    """Address and bytes of a workspace on the current device."""
    if t is None:
        return None, 0
    if t.get_device() != device or not t.is_contiguous():
        _refuse(where, "workspace has to be a contiguous tensor on the current device")
    return t.data_ptr(), t.nbytes


def _rows(where: str, device: int, name: str, t, codes):
    """Type and distance of the rows of a device matrix whose numbers lie next to each other in a row."""
    code = _type_codes.get(t.dtype)
    if code not in codes or t.get_device() != device or t.dim() != 2:
        _refuse(where, f"{name} has to be a matrix on the current device, of one of the types in the header")
    stride, step = t.stride()
    if step != 1 and t.shape[1] > 1 and t.numel() > 0:
        _refuse(where, f"{name} has to have the numbers of a row next to each other")
    return code, stride if t.shape[0] > 1 else t.shape[1]


def _routing(where: str, device: int, src_count: int, host_begin, experts: int, expert_host, *, choices=None, tokens=0, choices_per_token=0):
    kind = at = stride = 0
    if choices is not None:
        kind, stride = _rows(where, device, "choices", choices, (3, 4))
        tokens, choices_per_token = choices.shape
        at = choices.data_ptr()
    return Routing(tokens, choices_per_token, experts, kind, 0, at, stride,
                   _whole(where, device, "host_begin", host_begin, _torch.int64, (src_count + 1,)),
                   None if expert_host is None else _whole(where, device, "expert_host", expert_host, _torch.int32, (experts,)))


def _written(status: int, where: str, *outputs) -> int:
    """After a call that writes these tensors by their addresses: torch counts them as changed, so that an autograd graph
    that has saved one refuses to go on with what is there now."""
    _check(status, where)
    _torch._C._increment_version(outputs)
    return status


def _stream(stream) -> Optional[int]:
    if stream is None:  # (an object for it is most of a microsecond)
        return _torch._C._cuda_getCurrentRawStream(_torch._C._cuda_getDevice()) or None
    return stream.cuda_stream or None


class Topology:
    """Owns an ``a2a_topo`` handle.  Methods are the C entry points with the same names."""

    def __init__(self, row_ptr, col_idx):
        lib = load_library()
        rp = np.ascontiguousarray(row_ptr, dtype=np.int32)
        ci = np.ascontiguousarray(col_idx, dtype=np.int32)
        h = ctypes.c_void_p()
        _check(lib.a2a_topo_create(len(rp) - 1, rp.ctypes.data, ci.ctypes.data if len(ci) else None,
                                   ctypes.byref(h)), "a2a_topo_create")
        self._h = h
        n, e, d, lb = ctypes.c_int32(), ctypes.c_int64(), ctypes.c_int32(), ctypes.c_int32()
        _check(lib.a2a_topo_info(h, ctypes.byref(n), ctypes.byref(e), ctypes.byref(d), ctypes.byref(lb)),
               "a2a_topo_info")
        self.N, self.E, self.dmax, self.level_bound = n.value, e.value, d.value, lb.value

    def close(self):
        if getattr(self, "_h", None):
            load_library().a2a_topo_destroy(self._h)
            self._h = None

    __del__ = close

    def workspace_bytes(self, src_count: int, flags: int) -> int:
        return int(load_library().a2a_workspace_bytes(self._h, src_count, flags))

    def alloc_workspace(self, src_count: int, flags: int, max_bytes: Optional[int] = None):
        """A torch uint8 device tensor of the recommended size, capped at max_bytes."""
        import torch
        want = self.workspace_bytes(src_count, flags)
        least = self.workspace_bytes(src_count, flags | WS_MINIMAL)
        if max_bytes is not None:
            want = max(least, min(want, int(max_bytes)))
        return torch.empty(want, dtype=torch.uint8, device="cuda")

    def distances(self, src_begin: int, src_count: int, *, dist=None, sigma=None, dist_sum=None,
                  unreachable=None, flags=None, workspace, stream=None) -> int:
        return _check(load_library().a2a_distances(
            self._h, src_begin, src_count, _ptr(dist), _ptr(sigma), _ptr(dist_sum), _ptr(unreachable),
            _ptr(flags), _ptr(workspace), workspace.numel() if workspace is not None else 0,
            _stream(stream)), "a2a_distances")

    def link_loads(self, src_begin: int, src_count: int, *, load, dist_sum_total=None, flags=None,
                   workspace, stream=None) -> int:
        return _check(load_library().a2a_link_loads(
            self._h, src_begin, src_count, _ptr(load), _ptr(dist_sum_total), _ptr(flags),
            _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream(stream)),
            "a2a_link_loads")

    def link_loads_static(self, src_begin: int, src_count: int, *, load, dist_sum_total=None, flags=None,
                          stream=None) -> int:
        """a2a_link_loads on the library's fixed workspace array (no device allocation in the call)."""
        return _check(load_library().a2a_link_loads_static(
            self._h, src_begin, src_count, _ptr(load), _ptr(dist_sum_total), _ptr(flags), _stream(stream)),
            "a2a_link_loads_static")

    def sssp_loads(self, src_begin: int, src_count: int, iter_sources: int = 64, *, load, dist_sum_total=None,
                   flags=None, workspace, stream=None) -> int:
        """a2a_sssp_loads: single-path SSSP baseline, one iteration per ``iter_sources`` sources."""
        return _check(load_library().a2a_sssp_loads(
            self._h, src_begin, src_count, iter_sources, _ptr(load), _ptr(dist_sum_total), _ptr(flags),
            _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream(stream)),
            "a2a_sssp_loads")

    def link_loads_demand(self, src_begin: int, src_count: int, *, demand, load, weighted_dist=None,
                          dist_sum_total=None, flags=None, workspace, stream=None) -> int:
        """``demand``: device float64 [N][src_count], ``demand[t][s - src_begin]`` = what s sends to t."""
        return _check(load_library().a2a_link_loads_demand(
            self._h, src_begin, src_count, _ptr(demand), _ptr(load), _ptr(weighted_dist), _ptr(dist_sum_total),
            _ptr(flags), _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream(stream)),
            "a2a_link_loads_demand")

    def path_costs(self, src_begin: int, src_count: int, *, dist, sigma, link_cost=None, cost, workspace, stream=None) -> int:
        """a2a_path_costs: ``dist`` and ``sigma`` as :meth:`distances` leaves them, ``link_cost`` float64 [E] (None: 1 each),
        ``cost`` float64 [src_count][N]: mean cost of the shortest paths, the gradient of ``(link_cost * load).sum()`` by
        the demands of :meth:`link_loads_demand` (there by target, here by source)."""
        where, device, shape = "a2a_path_costs", _device(), (src_count, self.N)
        return _written(load_library().a2a_path_costs(
            self._h, src_begin, src_count, _whole(where, device, "dist", dist, _torch.int32, shape),
            _whole(where, device, "sigma", sigma, _torch.float64, shape),
            None if link_cost is None else _whole(where, device, "link_cost", link_cost, _torch.float64, (self.E,)),
            _whole(where, device, "cost", cost, _torch.float64, shape), *_workspace(where, device, workspace), _stream(stream)), where, cost)

    def dispatch_counts(self, src_count: int, *, choices, host_begin, experts: int, counts, stream=None) -> int:
        """a2a_dispatch_counts: how many of the ``choices`` (int32 or int64 [tokens][k]) of each source's tokens fall on
        each expert.  Source s has the tokens ``host_begin[s]`` to ``host_begin[s + 1] - 1`` (int64 [src_count + 1]).
        ``counts``: int32 [src_count][experts]."""
        where, device = "a2a_dispatch_counts", _device()
        r = _routing(where, device, src_count, host_begin, experts, None, choices=choices)
        return _written(load_library().a2a_dispatch_counts(
            self._h, src_count, r, _whole(where, device, "counts", counts, _torch.int32, (src_count, experts)), _stream(stream)),
            where, counts)

    def dispatch_demand(self, src_count: int, *, choices, host_begin, experts: int, expert_host=None, once: bool = False,
                        demand, stream=None) -> int:
        """a2a_dispatch_demand: what each source sends to each host, ``demand`` of :meth:`link_loads_demand` (float64
        [N][src_count]), in tokens.  Expert e lies on host ``expert_host[e]`` (int32; None: on host e); ``once``: a token goes
        to a host once, however many of its choices are there."""
        where, device = "a2a_dispatch_demand", _device()
        r = _routing(where, device, src_count, host_begin, experts, expert_host, choices=choices)
        return _written(load_library().a2a_dispatch_demand(
            self._h, src_count, r, int(once), _whole(where, device, "demand", demand, _torch.float64, (self.N, src_count)),
            _stream(stream)), where, demand)

    def balance_workspace_bytes(self, src_count: int, *, tokens: int, experts: int) -> int:
        return int(load_library().a2a_balance_workspace_bytes(self._h, src_count, tokens, experts))

    def alloc_balance_workspace(self, src_count: int, *, tokens: int, experts: int):
        """A torch uint8 device tensor for :meth:`balance_loss`."""
        import torch
        return torch.empty(self.balance_workspace_bytes(src_count, tokens=tokens, experts=experts), dtype=torch.uint8,
                           device="cuda")

    def balance_loss(self, src_count: int, *, logits, choices, host_begin, cost=None, expert_host=None, loss, counts,
                     prob_sums, rows, workspace, stream=None) -> int:
        """a2a_balance_loss: ``loss`` (float32 [1]) of a router with ``logits`` (float32, bfloat16 or float16
        [tokens][experts]) that made ``choices``, weighted by ``cost`` (float64 [src_count][N]; None: 1 each); and, for the
        gradient, ``counts`` (int32 [src_count][experts]), ``prob_sums`` (float32, the same) and ``rows`` (int32 [src_count]).  Autograd does not
        record the call, also where the logits require a gradient: that is :meth:`balance_loss_grad`'s, for the program to hand on."""
        where, device = "a2a_balance_loss", _device()
        kind, stride = _rows(where, device, "logits", logits, (0, 1, 2))
        tokens, experts = logits.shape
        r = _routing(where, device, src_count, host_begin, experts, expert_host, choices=choices)
        if r.tokens != tokens:
            _refuse(where, "logits and choices have to have as many rows")
        shape = (src_count, experts)
        return _written(load_library().a2a_balance_loss(
            self._h, src_count, r, logits.data_ptr(), kind, stride,
            None if cost is None else _whole(where, device, "cost", cost, _torch.float64, (src_count, self.N)),
            _whole(where, device, "loss", loss, _torch.float32, (1,)), _whole(where, device, "counts", counts, _torch.int32, shape),
            _whole(where, device, "prob_sums", prob_sums, _torch.float32, shape),
            _whole(where, device, "rows", rows, _torch.int32, (src_count,)), *_workspace(where, device, workspace), _stream(stream)),
            where, loss, counts, prob_sums, rows)

    def balance_loss_grad(self, src_count: int, *, logits, choices_per_token: int, host_begin, cost=None, expert_host=None,
                          counts, rows, upstream=None, grad, stream=None) -> int:
        """a2a_balance_loss_grad: gradient of :meth:`balance_loss` by the logits, ``grad`` (like ``logits``), times
        ``upstream`` (float32 [1]; None: 1).  ``grad`` may be ``logits`` themselves; an autograd graph that has saved them then
        refuses its backward pass, as after any change in place."""
        where, device = "a2a_balance_loss_grad", _device()
        kind, stride = _rows(where, device, "logits", logits, (0, 1, 2))
        grad_stride = _rows(where, device, "grad", grad, (kind,))[1]
        tokens, experts = logits.shape
        if grad.shape != logits.shape:
            _refuse(where, "grad has to have the shape of logits")
        r = _routing(where, device, src_count, host_begin, experts, expert_host, tokens=tokens, choices_per_token=choices_per_token)
        return _written(load_library().a2a_balance_loss_grad(
            self._h, src_count, r, logits.data_ptr(), kind, stride,
            None if cost is None else _whole(where, device, "cost", cost, _torch.float64, (src_count, self.N)),
            _whole(where, device, "counts", counts, _torch.int32, (src_count, experts)),
            _whole(where, device, "rows", rows, _torch.int32, (src_count,)),
            None if upstream is None else _whole(where, device, "upstream", upstream, _torch.float32, (1,)),
            grad.data_ptr(), grad_stride, _stream(stream)), where, grad)

    def profile_enable(self, mode: int = 1) -> None:
        """0 off, 1 events around the launches, 2 the same of the level kernels, which then serve every topology, and
        a count of shortest-path (source, link) pairs."""
        _check(load_library().a2a_profile_enable(self._h, int(mode)), "a2a_profile_enable")

    def profile_read(self) -> dict:
        out = Profile()
        _check(load_library().a2a_profile_read(self._h, ctypes.byref(out)), "a2a_profile_read")
        return out.as_dict()

    def schedule_bound(self, load, sum_dist: int, flags: int = 0, m_bytes: float = 1.0,
                       b_bytes_per_s: float = 1.0, stream=None, allow_disconnected: bool = False):
        out = Bound()
        st = load_library().a2a_schedule_bound(self._h, _ptr(load), int(sum_dist), int(flags),
                                               float(m_bytes), float(b_bytes_per_s), ctypes.byref(out),
                                               _stream(stream))
        _check(st, "a2a_schedule_bound", allow=(ERR_DISCONNECTED,) if allow_disconnected else ())
        return out, st

    def schedule_bound_cap(self, load, cap, sum_dist: int, flags: int = 0, m_bytes: float = 1.0,
                           b_bytes_per_s: float = 1.0, stream=None, allow_disconnected: bool = False):
        out = BoundCap()
        st = load_library().a2a_schedule_bound_cap(self._h, _ptr(load), _ptr(cap), int(sum_dist), int(flags),
                                                   float(m_bytes), float(b_bytes_per_s), ctypes.byref(out),
                                                   _stream(stream))
        _check(st, "a2a_schedule_bound_cap", allow=(ERR_DISCONNECTED,) if allow_disconnected else ())
        return out, st
