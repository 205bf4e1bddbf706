"""ctypes binding of libaspis (include/aspis.h).

Argument marshalling only: torch supplies device memory and the current HIP
stream; every step of the path runs in the library (host C++ for the
assignment and clique steps, gfx950 kernels for everything that touches the
gradients).  If the library is not built this module raises on import of
the library -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import operator
import os
from dataclasses import dataclass

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libaspis.so")

OK, ERR_INVALID_ARG, ERR_OVERFLOW, ERR_BUFFER_SMALL, ERR_DEVICE, ERR_NO_FILES = range(6)
REDUCE = {"median": 0, "mean": 1, "paper": 2}
ATTACK = {"weak": 0, "optimal": 1}
FLAG_TWO_PASS = 1
FLAG_TIMING = 2
FLAG_FULL_KEYS = 4
FLAG_HALF_KEYS = 8
FLAG_PROBE_PREFIX = 16
CLIP_HAVE_SUMSQ = 1
CLIP_SKIP_NONFINITE = 2
CLIP_NO_WAIT = 4
EMBED_ACCUMULATE = 1

EXPORTED = (
    "aspis_num_files", "aspis_assign", "aspis_detect", "aspis_clique",
    "aspis_aggregate_workspace", "aspis_aggregate", "aspis_detect_aggregate",
    "aspis_detect_aggregate_wm", "aspis_detect_aggregate_noalloc", "aspis_worker_rows",
    "aspis_plan",
    "aspis_read_probe_sink_words", "aspis_read_probe", "aspis_simulate", "aspis_detox",
    "aspis_last_error",
    "aspis_tensor_chunks", "aspis_tensor_entries", "aspis_tensor_table", "aspis_norm_workspace",
    "aspis_grad_norm", "aspis_clip_grads", "aspis_row_workspace", "aspis_row_norms",
    "aspis_clip_rows", "aspis_clipped_sgd", "aspis_clipped_adamw",
    "aspis_embed", "aspis_embed_workspace", "aspis_embed_grad", "aspis_dropout",
    "aspis_policy_workspace", "aspis_token_logps", "aspis_policy_loss",
)


class AspisError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"aspis status {status}: {message}")
        self.status = status


class DetectOut(ctypes.Structure):
    _fields_ = [("pair_diff", ctypes.c_void_p), ("vote", ctypes.c_void_p),
                ("has_majority", ctypes.c_void_p), ("disagree", ctypes.c_void_p)]


class CliqueResult(ctypes.Structure):
    _fields_ = [("success", ctypes.c_int32), ("omega", ctypes.c_int32),
                ("n_maximum", ctypes.c_int32), ("n_words", ctypes.c_int32),
                ("n_maximal", ctypes.c_int64), ("honest", ctypes.c_uint64 * 2),
                ("detected", ctypes.c_uint64 * 2), ("first", ctypes.c_uint64 * 2)]

    def as_dict(self, K: int) -> dict:
        def members(words):
            return frozenset(u for u in range(K) if (words[u // 64] >> (u % 64)) & 1)
        return {"success": bool(self.success), "omega": self.omega,
                "n_maximum": self.n_maximum, "n_maximal": self.n_maximal,
                "honest": members(self.honest) if self.success else frozenset(),
                "detected": members(self.detected) if self.success else frozenset(),
                "first": members(self.first)}


class SimResult(ctypes.Structure):
    _fields_ = [("files", ctypes.c_int64), ("distorted", ctypes.c_int64),
                ("dropped", ctypes.c_int64), ("success", ctypes.c_int32),
                ("omega", ctypes.c_int32), ("n_maximum", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("n_maximal", ctypes.c_int64),
                ("epsilon", ctypes.c_double), ("epsilon_baseline", ctypes.c_double),
                ("ms_files", ctypes.c_double), ("ms_clique", ctypes.c_double)]

    def as_dict(self) -> dict:
        d = {k: getattr(self, k) for k, _ in self._fields_ if k != "reserved"}
        d["success"] = bool(d["success"])
        return d


class RunStats(ctypes.Structure):
    _fields_ = [("fused", ctypes.c_int32), ("speculation_hit", ctypes.c_int32),
                ("probe_coords", ctypes.c_int64), ("ms_probe", ctypes.c_float),
                ("ms_main", ctypes.c_float), ("ms_fallback", ctypes.c_float),
                ("ms_total", ctypes.c_float), ("tile_cols", ctypes.c_int32),
                ("half_keys", ctypes.c_int32), ("tie_rows", ctypes.c_int32),
                ("probe_blocks", ctypes.c_int32), ("repair_groups", ctypes.c_int32)]

    def as_dict(self) -> dict:
        return {k: getattr(self, k) for k, _ in self._fields_}


KERNEL = {0: "none", 1: "fused_ws", 2: "fused", 3: "median_ws", 4: "median_tile",
          5: "median_radix"}


class KernelPlan(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("tile_cols", ctypes.c_int32),
                ("sweeps", ctypes.c_int32), ("half_keys", ctypes.c_int32),
                ("stream_threads", ctypes.c_int32), ("row_table", ctypes.c_int32),
                ("block", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("lds_bytes", ctypes.c_int64)]

    def as_dict(self) -> dict:
        d = {k: getattr(self, k) for k, _ in self._fields_ if k != "reserved"}
        d["kernel"] = KERNEL.get(self.kernel, str(self.kernel))
        return d


class Chunk(ctypes.Structure):
    _fields_ = [("addr", ctypes.c_uint64), ("n", ctypes.c_int32), ("info", ctypes.c_int32)]


class SgdOptions(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("momentum", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("max_norm", ctypes.c_double),
                ("nesterov", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class AdamwOptions(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta_one", ctypes.c_double),
                ("beta_two", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("max_norm", ctypes.c_double),
                ("step", ctypes.c_int64), ("flags", ctypes.c_uint32),
                ("reserved", ctypes.c_uint32)]


class PolicyOptions(ctypes.Structure):
    _fields_ = [("clip_low", ctypes.c_double), ("clip_high", ctypes.c_double),
                ("kl", ctypes.c_double), ("temperature", ctypes.c_double),
                ("grad_scale", ctypes.c_double)]


_lib = None


def lib():
    """Load libaspis.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; "
                          f"g.build()'` (or python paper_2108_02416_amd/build.py) first")
    # torch bundles a HIP runtime whose soname equals the system one; it must
    # be mapped first so that torch and this library share one runtime.
    import torch  # noqa: F401
    L = ctypes.CDLL(LIB_PATH)
    P, i32, i64, u32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32
    L.aspis_num_files.argtypes = [i32, i32]
    L.aspis_num_files.restype = i64
    L.aspis_assign.argtypes = [i32, i32, P, i64]
    L.aspis_assign.restype = ctypes.c_int
    L.aspis_detect.argtypes = [P, i32, i32, i64, P, ctypes.POINTER(DetectOut), P]
    L.aspis_detect.restype = ctypes.c_int
    L.aspis_clique.argtypes = [P, i32, i32, ctypes.POINTER(CliqueResult)]
    L.aspis_clique.restype = ctypes.c_int
    L.aspis_aggregate_workspace.argtypes = [i32, i32, i64]
    L.aspis_aggregate_workspace.restype = ctypes.c_size_t
    L.aspis_aggregate.argtypes = [P, i32, i32, i64, P, ctypes.POINTER(DetectOut),
                                  ctypes.POINTER(CliqueResult), ctypes.c_int, P, P,
                                  ctypes.POINTER(i64), P, ctypes.c_size_t, P]
    L.aspis_aggregate.restype = ctypes.c_int
    L.aspis_detect_aggregate.argtypes = [P, i32, i32, i32, i64, P, ctypes.POINTER(DetectOut),
                                         ctypes.c_int, P, P, ctypes.POINTER(CliqueResult),
                                         ctypes.POINTER(i64), P, ctypes.c_size_t, u32,
                                         ctypes.POINTER(RunStats), P]
    L.aspis_detect_aggregate.restype = ctypes.c_int
    L.aspis_detect_aggregate_wm.argtypes = L.aspis_detect_aggregate.argtypes
    L.aspis_detect_aggregate_wm.restype = ctypes.c_int
    L.aspis_detect_aggregate_noalloc.argtypes = [P, i32, i32, i32, i64, P,
                                                 ctypes.POINTER(DetectOut), ctypes.c_int, P, P,
                                                 ctypes.POINTER(CliqueResult),
                                                 ctypes.POINTER(i64), u32,
                                                 ctypes.POINTER(RunStats), P]
    L.aspis_detect_aggregate_noalloc.restype = ctypes.c_int
    L.aspis_worker_rows.argtypes = [i32, i32, P, i64]
    L.aspis_worker_rows.restype = ctypes.c_int
    L.aspis_plan.argtypes = [i32, i32, i64, i32, u32, ctypes.POINTER(KernelPlan),
                             ctypes.POINTER(KernelPlan)]
    L.aspis_plan.restype = ctypes.c_int
    L.aspis_read_probe_sink_words.argtypes = []
    L.aspis_read_probe_sink_words.restype = ctypes.c_size_t
    L.aspis_read_probe.argtypes = [P, ctypes.c_size_t, P, P]
    L.aspis_read_probe.restype = ctypes.c_int
    L.aspis_simulate.argtypes = [i32, i32, i32, ctypes.c_int, P, P, ctypes.POINTER(SimResult), P]
    L.aspis_simulate.restype = ctypes.c_int
    L.aspis_detox.argtypes = [i32, i32, i32, ctypes.c_int, ctypes.POINTER(i64),
                              ctypes.POINTER(ctypes.c_double)]
    L.aspis_detox.restype = ctypes.c_int
    f64, size = ctypes.c_double, ctypes.c_size_t
    L.aspis_tensor_chunks.argtypes = [P, i32]
    L.aspis_tensor_chunks.restype = i64
    L.aspis_tensor_entries.argtypes = [P, i32]
    L.aspis_tensor_entries.restype = i64
    L.aspis_tensor_table.argtypes = [P, P, P, i32, P, i64]
    L.aspis_tensor_table.restype = ctypes.c_int
    L.aspis_norm_workspace.argtypes = [i64]
    L.aspis_norm_workspace.restype = size
    L.aspis_grad_norm.argtypes = [P, i64, i32, P, P, P, P, size, P]
    L.aspis_grad_norm.restype = ctypes.c_int
    L.aspis_clip_grads.argtypes = [P, P, i64, f64, P, P, u32, P, size, P]
    L.aspis_clip_grads.restype = ctypes.c_int
    L.aspis_row_workspace.argtypes = [i64, i64, ctypes.c_int]
    L.aspis_row_workspace.restype = size
    L.aspis_row_norms.argtypes = [P, i64, i64, i64, ctypes.c_int, P, P, size, P]
    L.aspis_row_norms.restype = ctypes.c_int
    L.aspis_clip_rows.argtypes = [P, i64, i64, i64, ctypes.c_int, f64, P, i64, P, u32, P, size, P]
    L.aspis_clip_rows.restype = ctypes.c_int
    L.aspis_clipped_sgd.argtypes = [P, P, P, P, i64, ctypes.POINTER(SgdOptions), P, P, P, size, P]
    L.aspis_clipped_sgd.restype = ctypes.c_int
    L.aspis_clipped_adamw.argtypes = [P, P, P, P, P, i64, ctypes.POINTER(AdamwOptions), P, P, P,
                                      size, P]
    L.aspis_clipped_adamw.restype = ctypes.c_int
    kind, u64 = ctypes.c_int, ctypes.c_uint64
    L.aspis_embed.argtypes = [P, i64, i64, i64, kind, P, i64, kind, f64, P, i64, kind, P]
    L.aspis_embed.restype = ctypes.c_int
    L.aspis_embed_workspace.argtypes = [i64, i64]
    L.aspis_embed_workspace.restype = size
    L.aspis_embed_grad.argtypes = [P, i64, i64, i64, kind, P, kind, f64, P, i64, i64, kind, u32, P,
                                   size, P]
    L.aspis_embed_grad.restype = ctypes.c_int
    L.aspis_dropout.argtypes = [P, i64, i64, i64, kind, f64, u64, P, u64, P, i64, P, i64, P]
    L.aspis_dropout.restype = ctypes.c_int
    L.aspis_policy_workspace.argtypes = [i64, i64, kind]
    L.aspis_policy_workspace.restype = size
    L.aspis_token_logps.argtypes = [P, i64, i64, i64, kind, P, kind, f64, P, P, size, P]
    L.aspis_token_logps.restype = ctypes.c_int
    L.aspis_policy_loss.argtypes = [P, i64, i64, i64, kind, P, kind, P, P, P, P,
                                    ctypes.POINTER(PolicyOptions), P, P, P, i64, P, size, P]
    L.aspis_policy_loss.restype = ctypes.c_int
    L.aspis_last_error.argtypes = []
    L.aspis_last_error.restype = ctypes.c_char_p
    _lib = L
    return L


def _check(status: int):
    if status != OK:
        raise AspisError(status, lib().aspis_last_error().decode())


# ---------------------------------------------------------------- host steps

def num_files(K: int, r: int) -> int:
    return int(lib().aspis_num_files(K, r))


def assign(K: int, r: int) -> np.ndarray:
    f = num_files(K, r)
    if f <= 0:
        raise AspisError(ERR_INVALID_ARG, f"invalid (K={K}, r={r})")
    out = np.zeros((f, r), dtype=np.int32)
    _check(lib().aspis_assign(K, r, out.ctypes.data, f))
    return out


def worker_rows(K: int, r: int) -> np.ndarray:
    """Row of replica (i, s) in the worker-major upload [K][l][d]:
    int32 [f, r] (aspis_worker_rows)."""
    f = num_files(K, r)
    if f <= 0:
        raise AspisError(ERR_INVALID_ARG, f"invalid (K={K}, r={r})")
    out = np.zeros((f, r), dtype=np.int32)
    _check(lib().aspis_worker_rows(K, r, out.ctypes.data, f * r))
    return out


def plan(K: int, r: int, d: int, layout: str = "file", flags: int = 0) -> tuple[dict, dict]:
    """The kernels the device entry points take for this shape (aspis_plan):
    (single pass, median), each a dict of the kernel's tile parameters;
    flags may hold FLAG_FULL_KEYS."""
    sp, med = KernelPlan(), KernelPlan()
    _check(lib().aspis_plan(K, r, d, 1 if layout == "worker" else 0, flags, ctypes.byref(sp),
                            ctypes.byref(med)))
    return sp.as_dict(), med.as_dict()


def clique(disagree_rows: np.ndarray, K: int, q: int) -> CliqueResult:
    rows = np.ascontiguousarray(disagree_rows, dtype=np.uint64).reshape(K, -1)
    res = CliqueResult()
    _check(lib().aspis_clique(rows.ctypes.data, K, q, ctypes.byref(res)))
    return res


def simulate(K: int, r: int, q: int, attack: str = "optimal", adversaries=None,
             disagree_set=None, want_rows: bool = False) -> dict:
    """Distortion-fraction simulation of one attack on symbolic replicas
    (aspis_simulate); returns the result fields, plus the disagreement rows
    when want_rows."""
    def ids(x):
        if x is None:
            return None, None
        a = np.ascontiguousarray(np.asarray(x, dtype=np.int32).reshape(-1))
        if a.size != q:
            raise AspisError(ERR_INVALID_ARG, f"need {q} worker ids, got {a.size}")
        return a, a.ctypes.data
    a_arr, a_ptr = ids(adversaries)
    d_arr, d_ptr = ids(disagree_set)
    res = SimResult()
    rows = np.zeros((K, (K + 63) // 64), dtype=np.uint64) if want_rows else None
    _check(lib().aspis_simulate(K, r, q, ATTACK[attack], a_ptr, d_ptr, ctypes.byref(res),
                                rows.ctypes.data if rows is not None else None))
    out = res.as_dict()
    if want_rows:
        out["disagree_rows"] = rows
    return out


def detox(K: int, r: int, q: int, attack: str = "optimal") -> tuple[int, float]:
    """DETOX group-majority distortion (aspis_detox): (groups, epsilon)."""
    groups = ctypes.c_int64(0)
    eps = ctypes.c_double(0.0)
    _check(lib().aspis_detox(K, r, q, ATTACK[attack], ctypes.byref(groups), ctypes.byref(eps)))
    return int(groups.value), float(eps.value)


# -------------------------------------------------------------- device steps

def _torch():
    import torch
    return torch


def _stream_ptr():
    torch = _torch()
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check_grads(grads, K: int, r: int):
    torch = _torch()
    f = num_files(K, r)
    if not (grads.is_cuda and grads.dtype == torch.float32 and grads.dim() == 3
            and grads.is_contiguous() and grads.shape[0] == f and grads.shape[1] == r):
        raise AspisError(ERR_INVALID_ARG,
                         f"grads must be a contiguous cuda float32 [{f}, {r}, d] tensor")
    return f, grads.shape[2]


def _check_buffer(name: str, t, dtype, n: int, device):
    """A caller-supplied buffer must be a contiguous tensor of `dtype` with at
    least n elements on the replicas' device: the kernels write n elements."""
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise AspisError(ERR_INVALID_ARG, f"{name} must be a torch tensor")
    if t.dtype != dtype or not t.is_contiguous() or t.device != device or t.numel() < n:
        raise AspisError(ERR_INVALID_ARG,
                         f"{name} must be a contiguous {dtype} tensor on {device} with at "
                         f"least {n} elements (got {t.dtype}, {tuple(t.shape)}, {t.device}, "
                         f"contiguous={t.is_contiguous()})")


def _check_outputs(device, f: int, K: int, d: int, bufs=None, out=None, sel_out=None, ws=None):
    torch = _torch()
    if bufs is not None:
        _check_buffer("bufs.pair_diff", bufs.pair_diff, torch.int32, f, device)
        _check_buffer("bufs.vote", bufs.vote, torch.int8, f, device)
        _check_buffer("bufs.has_majority", bufs.has_majority, torch.uint8, f, device)
        _check_buffer("bufs.disagree", bufs.disagree, torch.int64, K, device)
    if out is not None:
        _check_buffer("out", out, torch.float32, d, device)
    if sel_out is not None:
        _check_buffer("sel_out", sel_out, torch.int32, f, device)
    if ws is not None:
        _check_buffer("ws", ws, torch.uint8, 1, device)


@dataclass
class DetectBuffers:
    pair_diff: object
    vote: object
    has_majority: object
    disagree: object

    @classmethod
    def empty(cls, f: int, K: int, device):
        torch = _torch()
        return cls(torch.empty(f, dtype=torch.int32, device=device),
                   torch.empty(f, dtype=torch.int8, device=device),
                   torch.empty(f, dtype=torch.uint8, device=device),
                   torch.empty(K, dtype=torch.int64, device=device))

    def c(self) -> DetectOut:
        return DetectOut(self.pair_diff.data_ptr(), self.vote.data_ptr(),
                         self.has_majority.data_ptr(), self.disagree.data_ptr())


_subsets_cache: dict = {}


def subsets_device(K: int, r: int, device):
    key = (K, r, str(device))
    if key not in _subsets_cache:
        torch = _torch()
        _subsets_cache[key] = torch.from_numpy(assign(K, r)).to(device)
    return _subsets_cache[key]


def workspace(K: int, r: int, d: int, device):
    torch = _torch()
    n = int(lib().aspis_aggregate_workspace(K, r, d))
    if n == 0:
        raise AspisError(ERR_INVALID_ARG, "invalid shape for workspace")
    return torch.empty(n + 256, dtype=torch.uint8, device=device)


def _aligned_ptr(ws) -> tuple[int, int]:
    p = ws.data_ptr()
    off = (-p) % 256
    return p + off, ws.numel() - off


def detect(grads, K: int, r: int, bufs: DetectBuffers | None = None) -> DetectBuffers:
    f, d = _check_grads(grads, K, r)
    bufs = bufs or DetectBuffers.empty(f, K, grads.device)
    _check_outputs(grads.device, f, K, d, bufs=bufs)
    sub = subsets_device(K, r, grads.device)
    out = bufs.c()
    _check(lib().aspis_detect(grads.data_ptr(), K, r, d, sub.data_ptr(), ctypes.byref(out),
                              _stream_ptr()))
    return bufs


def aggregate(grads, K: int, r: int, bufs: DetectBuffers, res: CliqueResult,
              mode: str = "median", out=None, sel_out=None, ws=None):
    torch = _torch()
    f, d = _check_grads(grads, K, r)
    out = out if out is not None else torch.empty(d, dtype=torch.float32, device=grads.device)
    ws = ws if ws is not None else workspace(K, r, d, grads.device)
    _check_outputs(grads.device, f, K, d, bufs=bufs, out=out, sel_out=sel_out, ws=ws)
    wp, wn = _aligned_ptr(ws)
    n_sel = ctypes.c_int64(0)
    det = bufs.c()
    st = lib().aspis_aggregate(grads.data_ptr(), K, r, d,
                               subsets_device(K, r, grads.device).data_ptr(), ctypes.byref(det),
                               ctypes.byref(res), REDUCE[mode], out.data_ptr(),
                               sel_out.data_ptr() if sel_out is not None else None,
                               ctypes.byref(n_sel), wp, wn, _stream_ptr())
    _check(st)
    return out, int(n_sel.value)


def _check_grads_wm(grads, K: int, r: int):
    torch = _torch()
    f = num_files(K, r)
    l_files = f * r // K
    if not (grads.is_cuda and grads.dtype == torch.float32 and grads.dim() == 3
            and grads.is_contiguous() and grads.shape[0] == K and grads.shape[1] == l_files):
        raise AspisError(ERR_INVALID_ARG,
                         f"grads must be a contiguous cuda float32 [{K}, {l_files}, d] tensor")
    return f, grads.shape[2]


def detect_aggregate(grads, K: int, r: int, q: int, mode: str = "median", flags: int = 0,
                     bufs: DetectBuffers | None = None, out=None, sel_out=None, ws=None,
                     want_sel: bool = True, layout: str = "file") -> dict:
    """The whole step (Algorithm 3 then Algorithm 1) in one library call.
    layout "file": grads is [f][r][d]; "worker": grads is the workers'
    upload [K][l][d] (aspis_detect_aggregate_wm)."""
    torch = _torch()
    if layout not in ("file", "worker"):
        raise AspisError(ERR_INVALID_ARG, f"unknown layout {layout!r}")
    f, d = (_check_grads if layout == "file" else _check_grads_wm)(grads, K, r)
    bufs = bufs or DetectBuffers.empty(f, K, grads.device)
    out = out if out is not None else torch.empty(d, dtype=torch.float32, device=grads.device)
    if sel_out is None and want_sel:
        sel_out = torch.empty(f, dtype=torch.int32, device=grads.device)
    ws = ws if ws is not None else workspace(K, r, d, grads.device)
    _check_outputs(grads.device, f, K, d, bufs=bufs, out=out, sel_out=sel_out, ws=ws)
    wp, wn = _aligned_ptr(ws)
    res = CliqueResult()
    stats = RunStats()
    n_sel = ctypes.c_int64(0)
    det = bufs.c()
    entry = lib().aspis_detect_aggregate if layout == "file" else lib().aspis_detect_aggregate_wm
    st = entry(
        grads.data_ptr(), K, r, q, d, subsets_device(K, r, grads.device).data_ptr(),
        ctypes.byref(det), REDUCE[mode], out.data_ptr(),
        sel_out.data_ptr() if sel_out is not None else None, ctypes.byref(res),
        ctypes.byref(n_sel), wp, wn, flags, ctypes.byref(stats), _stream_ptr())
    _check(st)
    return {"out": out, "sel": sel_out, "bufs": bufs, "clique": res,
            "n_selected": int(n_sel.value), "stats": stats.as_dict()}


def detect_aggregate_noalloc(grads, K: int, r: int, q: int, bufs: DetectBuffers, out,
                             sel_out=None, mode: str = "median", flags: int = 0) -> dict:
    """aspis_detect_aggregate_noalloc: the whole step with the library's
    static device scratch instead of a workspace; the caller passes every
    output buffer (nothing is allocated here either)."""
    f, d = _check_grads(grads, K, r)
    _check_outputs(grads.device, f, K, d, bufs=bufs, out=out, sel_out=sel_out)
    res = CliqueResult()
    stats = RunStats()
    n_sel = ctypes.c_int64(0)
    det = bufs.c()
    st = lib().aspis_detect_aggregate_noalloc(
        grads.data_ptr(), K, r, q, d, subsets_device(K, r, grads.device).data_ptr(),
        ctypes.byref(det), REDUCE[mode], out.data_ptr(),
        sel_out.data_ptr() if sel_out is not None else None, ctypes.byref(res),
        ctypes.byref(n_sel), flags, ctypes.byref(stats), _stream_ptr())
    _check(st)
    return {"out": out, "sel": sel_out, "bufs": bufs, "clique": res,
            "n_selected": int(n_sel.value), "stats": stats.as_dict()}


def read_probe(buf, sink=None) -> float:
    """Stream buf once; returns nothing useful on the host (see bench.py)."""
    torch = _torch()
    words = int(lib().aspis_read_probe_sink_words())
    if sink is None:
        sink = torch.empty(words, dtype=torch.int32, device=buf.device)
    nbytes = buf.numel() * buf.element_size()
    nbytes -= nbytes % 16
    _check(lib().aspis_read_probe(buf.data_ptr(), nbytes, sink.data_ptr(), _stream_ptr()))
    return sink


# ------------------------------------- norms, clipping and the model update

_dtype_codes: dict = {}


def _dtype_code(dtype) -> int:
    if not _dtype_codes:
        torch = _torch()
        _dtype_codes.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    code = _dtype_codes.get(dtype)
    if code is None:
        raise AspisError(ERR_INVALID_ARG, f"unsupported type {dtype}: float32, bfloat16 or float16")
    return code


def _layout(t):
    """Shape and strides of a tensor whose elements fill one span of memory
    without gaps or overlaps, None otherwise (strides of dimensions of one
    element say nothing and read 0)."""
    shape = tuple(t.shape)
    strides = tuple(0 if n == 1 else st for n, st in zip(shape, t.stride()))
    want = 1
    if t.numel() > 0:
        for st, n in sorted((st, n) for st, n in zip(strides, shape) if n > 1):
            if st != want:
                return None
            want *= n
    return shape, strides


def _raw_stream(device) -> int:
    """The current stream of a device with an index, as the library takes it
    (an order of magnitude quicker than asking for the stream object)."""
    return _torch()._C._cuda_getCurrentRawStream(device.index)


def _launch(device, call, *args):
    """Calls a library function that enqueues work on `device`, and checks
    its status."""
    torch = _torch()
    if device.index == torch._C._cuda_getDevice():
        _check(call(*args))
    else:
        with torch.cuda.device(device):
            _check(call(*args))


def _capturing(device) -> bool:
    """Whether the device's current stream is being captured into a graph."""
    torch = _torch()
    if device.type != "cuda":
        return False
    with torch.cuda.device(device):
        return torch.cuda.is_current_stream_capturing()


_native = None


def _tensors():
    """The module that looks torch tensors over (csrc/aspis_tensors.cpp)."""
    global _native
    if _native is None:
        import torch  # noqa: F401  (its libraries come first)
        try:
            from . import _tensors as module
        except ImportError as e:
            raise ImportError(f"{os.path.join(HERE, '_tensors.so')} is missing or does not load "
                              f"({e}): run python -c 'import __graft_entry__ as g; g.build()'") from e
        _native = module
    return _native


def _tensor_state(tensors) -> bytes:
    """Where the tensors of a list are and how they are laid out."""
    return _tensors().state(tensors)


def _buffer(name: str, t, dtype, n: int, device) -> int:
    """The address of a caller's buffer, checked as _check_buffer does."""
    at = _tensors().buffer(t, dtype, n, device.index)
    if at is None:
        _check_buffer(name, t, dtype, n, device)
        if t.is_neg():
            raise AspisError(ERR_INVALID_ARG, f"{name} is a negated view (resolve_neg())")
        at = t.data_ptr()
    return at


class TensorList:
    """A list of CUDA tensors as the norm, clipping and update calls take it
    (aspis_tensor_table): made once for tensors that stay, or by the call
    itself from any sequence of tensors.

    Tensors are float32, bfloat16 or float16 (types may mix), on one device,
    of any shape, also empty; each must fill one span of memory (any order of
    its dimensions, no gaps).  The list holds the tensors and looks at every
    call whether they still are where they were, of the types and in the
    layouts they had, so that a tensor whose storage was replaced
    (`t.data = ...`) is read as it is now.  It does not see other tensors that
    take their place: where gradients are new objects every step (`p.grad`
    after `zero_grad()`, which drops them by default), zero them in place
    (`zero_grad(set_to_none=False)`) or hand each call the new sequence.

    Making a list, or reading one again, uploads its table and waits for the
    current stream, so that the table is there for every stream; it cannot be
    done while a graph is captured.  A list that a call makes itself serves
    the current stream alone and does not wait.

    A graph that captured a call reads the table the list had then: keep the
    list and its tensors where they are for as long as it is replayed."""

    _own_stream_only = False

    def __init__(self, tensors, device=None):
        torch = _torch()
        self.tensors = [tensors] if isinstance(tensors, torch.Tensor) else list(tensors)
        for i, t in enumerate(self.tensors):
            if not isinstance(t, torch.Tensor) or not t.is_cuda or t.layout != torch.strided:
                raise AspisError(ERR_INVALID_ARG, f"tensor {i} of the list must be a strided cuda "
                                                  f"tensor")
        if device is None:
            device = self.tensors[0].device if self.tensors else \
                torch.device("cuda", torch.cuda.current_device())
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._read()

    def __len__(self):
        return len(self.tensors)

    def _read(self):
        """Looks the tensors over and uploads their table.  The list takes
        over what it read only when all of it is there: after a refusal or a
        failed upload the next call reads again."""
        torch = _torch()
        ts = self.tensors
        n = len(ts)
        state = _tensor_state(ts)
        self._where = None
        where, numels = [t.data_ptr() for t in ts], [t.numel() for t in ts]
        dtypes = [t.dtype for t in ts]
        codes = np.array([_dtype_code(d) for d in dtypes], dtype=np.int32)
        contiguous = True
        for i, t in enumerate(ts):
            if t.device != self.device:
                raise AspisError(ERR_INVALID_ARG, f"tensor {i} of the list is on {t.device}, the "
                                                  f"list on {self.device}")
            if t.is_neg():
                raise AspisError(ERR_INVALID_ARG, f"tensor {i} of the list is a negated view: its "
                                                  f"memory holds other values (resolve_neg())")
            if not t.is_contiguous():
                contiguous = False
                if _layout(t) is None:
                    raise AspisError(ERR_INVALID_ARG,
                                     f"tensor {i} of the list has gaps or overlaps in memory: "
                                     f"shape {tuple(t.shape)}, strides {t.stride()}")
        spans = sorted((p, p + k * t.element_size()) for p, k, t in zip(where, numels, ts) if k)
        ends = max((b for _, b in spans), default=0)
        ptrs = np.array(where, dtype=np.uint64)
        sizes = np.array(numels, dtype=np.int64)
        n_chunks = int(lib().aspis_tensor_chunks(sizes.ctypes.data, n))
        entries = int(lib().aspis_tensor_entries(sizes.ctypes.data, n))
        if entries < 0:
            raise AspisError(ERR_OVERFLOW, "too many elements in the list")
        if _capturing(self.device):
            raise AspisError(ERR_INVALID_ARG, "a list's table cannot be uploaded while a graph is "
                                              "captured: make a TensorList before, and keep its "
                                              "tensors where they are")
        host = np.empty((max(entries, 1), 2), dtype=np.int64)
        _check(lib().aspis_tensor_table(ptrs.ctypes.data, sizes.ctypes.data, codes.ctypes.data, n,
                                        host.ctypes.data, entries))
        # from pageable memory the copy returns when it is done; pinned memory
        # is not given out again before the copy from it is done
        table = torch.from_numpy(host)
        if self._own_stream_only:
            table = table.pin_memory()
        table = table.to(self.device, non_blocking=self._own_stream_only)
        self._table, self._address = table, table.data_ptr()
        self._stream = _raw_stream(self.device)
        self.numels, self.dtypes, self.contiguous = numels, dtypes, contiguous
        self.disjoint = all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
        self.spans = np.array([*(x for s in spans for x in s), ends], dtype=np.uint64).tobytes()
        self.n_chunks = n_chunks
        self.all_float32 = all(d == torch.float32 for d in dtypes)
        self.ws_bytes = int(lib().aspis_norm_workspace(n_chunks))
        self._where = state

    def table(self) -> int:
        """Device address of the table, brought up to date."""
        if _tensor_state(self.tensors) != self._where:
            self._read()
        if _raw_stream(self.device) != self._stream:
            self._table.record_stream(_torch().cuda.current_stream(self.device))
        return self._address


class _CallList(TensorList):
    """A list made by a call, for the stream the call is on."""
    _own_stream_only = True


def _list(x) -> TensorList:
    return x if isinstance(x, TensorList) else _CallList(x)


def _check_match(name: str, a: TensorList, ref: TensorList, same_types: bool = False,
                 float32: bool = False):
    """`a` lists tensors of the sizes, order of elements and device of ref's."""
    if a.numels != ref.numels or a.device != ref.device:
        raise AspisError(ERR_INVALID_ARG, f"{name} must list tensors of the gradients' sizes, in "
                                          f"their order, on their device")
    if not (a.contiguous and ref.contiguous):
        for x, y in zip(a.tensors, ref.tensors):
            if not (x.is_contiguous() and y.is_contiguous()) and _layout(x) != _layout(y):
                raise AspisError(ERR_INVALID_ARG, f"{name}: tensors that are not contiguous must "
                                                  f"have the gradients' shapes and strides")
    if same_types and a.dtypes != ref.dtypes:
        raise AspisError(ERR_INVALID_ARG, f"{name} must have the gradients' types")
    if float32 and not a.all_float32:
        raise AspisError(ERR_INVALID_ARG, f"{name} must be float32")


def _check_written(name: str, a: TensorList):
    if not a.disjoint:
        raise AspisError(ERR_INVALID_ARG, f"{name} is written and lists overlapping tensors")


def _check_apart(*lists: TensorList):
    if not _tensors().apart(*[a.spans for a in lists]):
        raise AspisError(ERR_INVALID_ARG, "the lists of a call overlap in memory")


@dataclass
class NormBuffers:
    """What the norm of a list leaves on the device: norm float32 [1], sumsq
    float64 [1] (of a call by a given sum of squares: that one) and, when
    asked for, each float32 [n] (every tensor's own)."""
    norm: object
    sumsq: object
    each: object = None

    @classmethod
    def empty(cls, device, each: int = 0):
        torch = _torch()
        return cls(torch.empty(1, dtype=torch.float32, device=device),
                   torch.empty(1, dtype=torch.float64, device=device),
                   torch.empty(each, dtype=torch.float32, device=device) if each else None)


def norm_workspace(grads):
    """Workspace of grad_norm, clip_grads and the updates for a list."""
    torch = _torch()
    grads = _list(grads)
    grads.table()
    return torch.empty(grads.ws_bytes, dtype=torch.uint8, device=grads.device)


def _scratch(grads: TensorList, bufs, ws, sumsq, each: int = 0):
    """Checked or new buffers of a call: bufs, the addresses of norm, sum of
    squares and each, the workspace and its address, and the flags they ask for."""
    torch = _torch()
    dev, f32, f64 = grads.device, torch.float32, torch.float64
    if bufs is None:
        bufs = NormBuffers.empty(dev, each)
    norm = _buffer("bufs.norm", bufs.norm, f32, 1, dev)
    total = _buffer("bufs.sumsq", bufs.sumsq, f64, 1, dev)
    each_at = _buffer("bufs.each", bufs.each, f32, each, dev) if each else None
    flags = 0
    if sumsq is not None:
        # bufs holds the sum the call went by; given in bufs.sumsq it is there
        if _buffer("sumsq", sumsq, f64, 1, dev) != total:
            bufs.sumsq.view(-1)[:1].copy_(sumsq.view(-1)[:1])
        flags = CLIP_HAVE_SUMSQ
    if ws is None:
        ws = torch.empty(grads.ws_bytes, dtype=torch.uint8, device=dev)
    ws_at = _buffer("ws", ws, torch.uint8, grads.ws_bytes, dev)
    return bufs, norm, total, each_at, ws, ws_at, flags


def grad_norm(grads, each: bool = False, bufs: NormBuffers | None = None, ws=None) -> NormBuffers:
    """The global L2 norm of a list of tensors (aspis_grad_norm), with every
    tensor's own norm when `each`.  Nothing is synchronised, whether `grads`
    is a kept list or any sequence: the results are on the device.  Where ranks hold shards of one model, all-reduce
    bufs.sumsq and hand it to clip_grads or an update as sumsq (with the same
    bufs it is used where it is, otherwise copied)."""
    grads = _list(grads)
    table = grads.table()
    bufs, norm, total, each_at, ws, ws_at, _ = _scratch(grads, bufs, ws, None,
                                                        len(grads) if each else 0)
    if each and bufs.each is None:   # no tensors
        bufs.each = _torch().empty(0, dtype=_torch().float32, device=grads.device)
    _launch(grads.device, lib().aspis_grad_norm, table, grads.n_chunks, len(grads), total,
            norm, each_at, ws_at, ws.numel(), _raw_stream(grads.device))
    return bufs


def clip_grads(grads, max_norm: float, out=None, sumsq=None, bufs: NormBuffers | None = None,
               ws=None) -> NormBuffers:
    """Scales a list of tensors so that its global norm is at most max_norm
    (aspis_clip_grads): in place, or into the tensors of `out`.  Returns the
    norm before clipping.  sumsq: the sum of squares to clip by (of all
    ranks), instead of this list's own.

    Autograd does not see it: results carry no graph, and writing in place
    does not count in the tensors' versions."""
    grads = _list(grads)
    table = grads.table()
    bufs, norm, total, _, ws, ws_at, flags = _scratch(grads, bufs, ws, sumsq)
    if out is None:
        _check_written("grads", grads)
        out_table = None
    else:
        out = _list(out)
        out_table = out.table()
        _check_match("out", out, grads, same_types=True)
        _check_written("out", out)
        if out._where != grads._where:   # each tensor onto itself is in place
            _check_apart(grads, out)
    _launch(grads.device, lib().aspis_clip_grads, table, out_table, grads.n_chunks, max_norm,
            total, norm, flags, ws_at, ws.numel(), _raw_stream(grads.device))
    return bufs


def _rows(name: str, x):
    """rows, d, elements between rows' starts and type of a tensor of rows."""
    plain = _tensors().rows(x)
    if plain is not None:
        return plain
    torch = _torch()
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dim() < 1:
        raise AspisError(ERR_INVALID_ARG, f"{name} must be a cuda tensor of rows [..., d]")
    if x.is_neg():
        raise AspisError(ERR_INVALID_ARG, f"{name} is a negated view: its memory holds other values "
                                          f"(resolve_neg())")
    code = _dtype_code(x.dtype)
    d = x.shape[-1]
    rows = 1
    for n in x.shape[:-1]:
        rows *= n
    if rows * d == 0:
        return rows, d, d, code
    # the leading dimensions have to be one series of rows, equally far apart
    ld, run = None, 1
    for n, st in zip(reversed(x.shape[:-1]), reversed(x.stride()[:-1])):
        if n == 1:
            continue
        if ld is None:
            ld = st
        elif st != ld * run:
            ld = -1
            break
        run *= n
    ld = d if ld is None else ld
    if ld < d or (d > 1 and x.stride(-1) != 1):
        raise AspisError(ERR_INVALID_ARG, f"{name} must hold rows of contiguous elements, equally "
                                          f"far apart: shape {tuple(x.shape)}, strides "
                                          f"{x.stride()}")
    return rows, d, ld, code


def row_workspace(x):
    """Workspace of row_norms and clip_rows for a tensor of rows."""
    torch = _torch()
    rows, d, _, code = _rows("x", x)
    return torch.empty(int(lib().aspis_row_workspace(rows, d, code)), dtype=torch.uint8,
                       device=x.device)


def _row_buffers(x, rows: int, d: int, code: int, norms, ws):
    """Checked or new buffers of a call on rows, and their addresses."""
    torch = _torch()
    if norms is None:
        norms = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    if ws is None:
        ws = torch.empty(int(lib().aspis_row_workspace(rows, d, code)), dtype=torch.uint8,
                         device=x.device)
    # the workspace's size is the library's to check
    return (norms, _buffer("norms", norms, torch.float32, rows, x.device),
            ws, _buffer("ws", ws, torch.uint8, 0, x.device))


def row_norms(x, norms=None, ws=None):
    """The L2 norm of every row of x [..., d] (aspis_row_norms): the replicas
    [f][r][d] or a worker's upload [l][d].  Results carry no autograd graph."""
    rows, d, ld, code = _rows("x", x)
    norms, norms_at, ws, ws_at = _row_buffers(x, rows, d, code, norms, ws)
    _launch(x.device, lib().aspis_row_norms, x.data_ptr(), rows, d, ld, code, norms_at, ws_at,
            ws.numel(), _raw_stream(x.device))
    return norms


def clip_rows(x, max_norm: float, out=None, norms=None, ws=None, flags: int = 0):
    """Scales every row of x [..., d] whose norm is above max_norm down to it
    (aspis_clip_rows): in place, or into `out`.  Returns (out, the norms before
    clipping).  Replicas with equal bits are equal after it, so a server may
    clip them before detection (of float32 replicas) and workers before they
    upload.  flags may hold CLIP_NO_WAIT.  Autograd does not see it, as with
    clip_grads."""
    rows, d, ld, code = _rows("x", x)
    out = x if out is None else out
    ldo = ld
    if out is not x:
        _, _, ldo, out_code = _rows("out", out)
        if out.shape != x.shape or out_code != code or out.device != x.device:
            raise AspisError(ERR_INVALID_ARG, "out must have the shape, type and device of x")
    norms, norms_at, ws, ws_at = _row_buffers(x, rows, d, code, norms, ws)
    _launch(x.device, lib().aspis_clip_rows, x.data_ptr(), rows, d, ld, code, max_norm,
            out.data_ptr(), ldo, norms_at, flags, ws_at, ws.numel(), _raw_stream(x.device))
    return out, norms


def _update_lists(params, grads, states: dict, copies):
    """The lists of an update, checked against the gradients', and their
    tables.  The caller keeps the lists until it has launched: a list made
    for the call owns its table's memory."""
    lists = {"params": _list(params), **{k: _list(v) for k, v in states.items()}}
    if copies is not None:
        lists["copies"] = _list(copies)
    tables = [grads.table()]
    for name, a in lists.items():
        tables.append(a.table())
        _check_match(name, a, grads, float32=name != "copies")
        _check_written(name, a)
    _check_apart(grads, *lists.values())
    return lists, tables


def clipped_sgd(params, grads, mean=None, *, lr: float, momentum: float = 0.0,
                nesterov: bool = False, weight_decay: float = 0.0,
                max_norm: float = float("inf"), copies=None, sumsq=None,
                skip_nonfinite: bool = False, bufs: NormBuffers | None = None,
                ws=None) -> NormBuffers:
    """One SGD update in place, by the gradients clipped to max_norm
    (aspis_clipped_sgd); the gradients stay as they are.  params and mean
    (the momentum, needed unless it is 0) are lists of float32 tensors,
    copies a list that receives the new parameters rounded to its types.
    Returns the norm before clipping.  skip_nonfinite: a norm that is not
    finite as the float32 it is returned in leaves parameters, state and
    copies as they are.

    The update is not seen by autograd's version counters."""
    if momentum and mean is None:
        raise AspisError(ERR_INVALID_ARG, "momentum needs the list `mean`")
    grads = _list(grads)
    lists, tables = _update_lists(params, grads, {} if mean is None else {"mean": mean}, copies)
    bufs, norm, total, _, ws, ws_at, flags = _scratch(grads, bufs, ws, sumsq)
    opt = SgdOptions(lr, momentum, weight_decay, max_norm, int(nesterov),
                     flags | (CLIP_SKIP_NONFINITE if skip_nonfinite else 0))
    _launch(grads.device, lib().aspis_clipped_sgd, tables[1], tables[0],
            tables[2] if mean is not None else None, tables[-1] if copies is not None else None,
            grads.n_chunks, ctypes.byref(opt), total, norm, ws_at, ws.numel(),
            _raw_stream(grads.device))
    del lists   # their tables were needed until here
    return bufs


def clipped_adamw(params, grads, mean, square, *, step: int, lr: float, betas=(0.9, 0.999),
                  eps: float = 1e-8, weight_decay: float = 0.01,
                  max_norm: float = float("inf"), copies=None, sumsq=None,
                  skip_nonfinite: bool = False, bufs: NormBuffers | None = None,
                  ws=None) -> NormBuffers:
    """One AdamW update in place, by the gradients clipped to max_norm
    (aspis_clipped_adamw); as clipped_sgd otherwise.  step counts from 1.

    step, lr and the other numbers are taken when the call is made: a graph
    that captured it replays the update of that step."""
    grads = _list(grads)
    lists, tables = _update_lists(params, grads, {"mean": mean, "square": square}, copies)
    bufs, norm, total, _, ws, ws_at, flags = _scratch(grads, bufs, ws, sumsq)
    opt = AdamwOptions(lr, betas[0], betas[1], eps, weight_decay, max_norm, step,
                       flags | (CLIP_SKIP_NONFINITE if skip_nonfinite else 0), 0)
    _launch(grads.device, lib().aspis_clipped_adamw, tables[1], tables[0], tables[2], tables[3],
            tables[4] if copies is not None else None, grads.n_chunks, ctypes.byref(opt),
            total, norm, ws_at, ws.numel(), _raw_stream(grads.device))
    del lists   # their tables were needed until here
    return bufs


# ------------------------------------------ a worker's step on token data

def _place(name: str, x):
    """Address, rows, d, elements between rows, type code and device index of a
    tensor of rows [..., d]."""
    place = _tensors().place(x)
    if place is not None:
        return place
    rows, d, ld, code = _rows(name, x)
    return x.data_ptr(), rows, d, ld, code, x.device.index


def _token_place(tokens, n: int, index: int):
    """Address and type code of the n tokens of a call on device `index`."""
    place = _tensors().tokens(tokens)
    if place is None or place[1] != n or place[3] != index:
        torch = _torch()
        what = f"{tokens.dtype}, {tuple(tokens.shape)}, {tokens.device}" \
            if isinstance(tokens, torch.Tensor) else type(tokens).__name__
        raise AspisError(ERR_INVALID_ARG, f"tokens must be a contiguous int32 or int64 tensor of {n} "
                                          f"tokens on cuda:{index} (got {what})")
    return place[0], place[2]


def _floats(name: str, t, n: int, index: int, exact: bool = True) -> int:
    """The address of a contiguous float32 tensor of n elements (or at least so
    many)."""
    at = _tensors().buffer(t, _float32(), n, index)
    if at is None:
        at = _buffer(name, t, _float32(), n, _torch().device("cuda", index))
    if exact and t.numel() != n:
        raise AspisError(ERR_INVALID_ARG, f"{name} must hold {n} numbers (got {tuple(t.shape)})")
    return at


def _scratch_at(ws, index: int) -> int:
    """The address of a workspace (its size is the library's to check)."""
    at = _tensors().buffer(ws, _uint8(), 0, index)
    return at if at is not None else \
        _buffer("ws", ws, _uint8(), 0, _torch().device("cuda", index))


_kinds: list = []


def _float32():
    if not _kinds:
        torch = _torch()
        _kinds.extend([torch.float32, torch.uint8])
    return _kinds[0]


def _uint8():
    _float32()
    return _kinds[1]


_cuda: list = []


def _enqueue(index: int, call, *args):
    """Calls a library function with the current stream of a device as its last
    argument, and checks its status."""
    if not _cuda:
        c = _torch()._C
        _cuda.extend([c._cuda_getDevice, c._cuda_getCurrentRawStream])
    if _cuda[0]() == index:
        status = call(*args, _cuda[1](index))
    else:
        with _torch().cuda.device(index):
            status = call(*args, _cuda[1](index))
    if status != OK:
        _check(status)


def embed(table, tokens, scale: float = 1.0, out=None):
    """scale * table[tokens] (aspis_embed): rows of table [vocab, d] for tokens
    (int32 or int64, any shape) into out [*tokens.shape, d], of the table's type
    unless given.  A token outside [0, vocab) gives a row of zeros: padding, or
    one that another rank's part of the table holds (subtract the part's first
    token, add the ranks' results).  Its gradient is embed_grad; autograd does
    not see either."""
    at, vocab, d, ld, code, index = _place("table", table)
    if table.dim() != 2:
        raise AspisError(ERR_INVALID_ARG, f"table must be [vocab, d], not {tuple(table.shape)}")
    if out is None:
        torch = _torch()
        shape = tokens.shape if isinstance(tokens, torch.Tensor) else ()
        out = torch.empty((*shape, d), dtype=table.dtype, device=table.device)
    to, n, width, ldo, out_code, out_index = _place("out", out)
    ids, wide = _token_place(tokens, n, index)
    if width != d or out_index != index:
        raise AspisError(ERR_INVALID_ARG, f"out must hold rows of {d} on {table.device}")
    _enqueue(index, lib().aspis_embed, at, vocab, d, ld, code, ids, n, wide, scale, to, ldo,
             out_code)
    return out


def embed_workspace(grad, tokens, vocab: int):
    """Workspace of embed_grad for a gradient [..., d] of these tokens (of any
    vocabulary)."""
    torch = _torch()
    _, rows, d, _, _, index = _place("grad", grad)
    n = int(lib().aspis_embed_workspace(rows, d))
    if n == ctypes.c_size_t(-1).value:
        raise AspisError(ERR_OVERFLOW, f"{rows} tokens of {d} are too many")
    return torch.empty(n, dtype=torch.uint8, device=grad.device)


def embed_grad(grad, tokens, vocab: int, scale: float = 1.0, out=None, accumulate: bool = False,
               ws=None):
    """The table's gradient of embed (aspis_embed_grad): row v of out [vocab, d]
    (float32 unless given) is scale times the sum of the rows of grad [..., d]
    whose token is v, in the tokens' order, so that equal inputs give equal
    bits.  Rows without a token are zeroed; with accumulate the sums are added
    to what out holds, and those rows are left alone.  (An expanded grad, as a
    mean over positions sends back, holds no rows: hand in grad.contiguous().)"""
    at, n, d, ld, code, index = _place("grad", grad)
    ids, wide = _token_place(tokens, n, index)
    if out is None:
        if accumulate:
            raise AspisError(ERR_INVALID_ARG, "accumulate needs out")
        out = _torch().empty((vocab, d), dtype=_float32(), device=grad.device)
    to, rows, width, ldo, out_code, out_index = _place("out", out)
    if rows != vocab or width != d or out_index != index:
        raise AspisError(ERR_INVALID_ARG, f"out must be [{vocab}, {d}] on {grad.device}, not "
                                          f"{tuple(out.shape)} on {out.device}")
    if ws is None:
        ws = embed_workspace(grad, tokens, vocab)
    _enqueue(index, lib().aspis_embed_grad, at, n, d, ld, code, ids, wide, scale, to, vocab, ldo,
             out_code, EMBED_ACCUMULATE if accumulate else 0, _scratch_at(ws, index), ws.numel())
    return out


def dropout(x, p: float, seed, offset: int = 0, residual=None, out=None):
    """x [..., d] with a share p of its elements dropped and the others scaled
    by 1 / (1 - p), plus residual when given (aspis_dropout), into out (x or
    residual themselves, another tensor, or a new one).

    Which elements are dropped depends on the seed (an int) and an element's
    position, offset + its index, alone, and is never stored: the gradient by
    x is dropout(grad, p, seed, offset), and workers that seed by file, layer
    and step drop the same.  Ranks with shards give the shard's first position
    as offset.  p counts in steps of 2^-16.  A graph that captured a call
    replays its mask; with seed a cuda int64 tensor [1] it draws what that then
    holds.  Autograd does not see it."""
    at, rows, d, ld, code, index = _place("x", x)
    if out is None:
        out = _torch().empty(x.shape, dtype=x.dtype, device=x.device)
    to, ldo, res, ldr = at, ld, None, 0
    if out is not x:
        to, _, _, ldo, out_code, out_index = _place("out", out)
        if out.shape != x.shape or out_code != code or out_index != index:
            raise AspisError(ERR_INVALID_ARG, "out must have the shape, type and device of x")
    if residual is not None:
        res, _, _, ldr, res_code, res_index = _place("residual", residual)
        if residual.shape != x.shape or res_code != code or res_index != index:
            raise AspisError(ERR_INVALID_ARG, "residual must have the shape, type and device of x")
    seed_at = None
    if isinstance(seed, _torch().Tensor):
        seed_at, seed = _buffer("seed", seed, _torch().int64, 1, x.device), 0
    seed, offset = operator.index(seed), operator.index(offset)
    _enqueue(index, lib().aspis_dropout, at, rows, d, ld, code, p, seed & 0xFFFFFFFFFFFFFFFF,
             seed_at, offset & 0xFFFFFFFFFFFFFFFF, res, ldr, to, ldo)
    return out


@dataclass
class PolicyBuffers:
    """What policy_loss leaves on the device: sums float32 [3], the weighted
    sums of the loss, of the KL term and of the positions where the clip acts;
    logps float32 [rows], the tokens' log-probabilities."""
    sums: object
    logps: object

    @classmethod
    def empty(cls, rows: int, device):
        torch = _torch()
        return cls(torch.empty(3, dtype=torch.float32, device=device),
                   torch.empty(rows, dtype=torch.float32, device=device))


def policy_workspace(logits):
    """Workspace of token_logps and policy_loss for logits [..., vocab]."""
    torch = _torch()
    _, rows, vocab, _, code, _ = _place("logits", logits)
    n = int(lib().aspis_policy_workspace(rows, vocab, code))
    if n == ctypes.c_size_t(-1).value:
        raise AspisError(ERR_OVERFLOW, f"{rows} rows of {vocab} logits are too many")
    return torch.empty(n, dtype=torch.uint8, device=logits.device)


def token_logps(logits, tokens, temperature: float = 1.0, logps=None, ws=None):
    """log p of a token per row of logits [..., vocab] under
    softmax(logits / temperature) (aspis_token_logps), float32 of the tokens'
    shape: what policy_loss takes as old and ref.  0 where the token is outside
    the vocabulary.  A row's result does not depend on the others of the call.
    The result carries no autograd graph."""
    at, rows, vocab, ld, code, index = _place("logits", logits)
    ids, wide = _token_place(tokens, rows, index)
    if logps is None:
        logps = _torch().empty(tokens.shape, dtype=_float32(), device=logits.device)
    if ws is None:
        ws = policy_workspace(logits)
    _enqueue(index, lib().aspis_token_logps, at, rows, vocab, ld, code, ids, wide, temperature,
             _floats("logps", logps, rows, index), _scratch_at(ws, index), ws.numel())
    return logps


def policy_loss(logits, tokens, old, advantage, weight, ref=None, clip=(0.2, 0.2), kl: float = 0.0,
                temperature: float = 1.0, grad=None, grad_scale: float = 1.0,
                bufs: PolicyBuffers | None = None, ws=None) -> PolicyBuffers:
    """The clipped policy loss of tokens under logits [..., vocab], with a KL
    term towards a reference, and its gradient by the logits in the same call
    (aspis_policy_loss has the formulas).  old, advantage, weight and ref are
    float32, a number per position: log-probabilities when sampled, the
    advantage, what the position counts (its mask over the number of
    positions; 0 leaves it out) and log-probabilities under the reference.
    clip is (below, above) 1.  grad receives grad_scale times the gradient: a
    tensor like logits, or logits themselves.  A row's gradient does not depend
    on the others of the call.  Nothing is synchronised.

    Autograd does not see it: hand grad to the layer below (or to autograd, as
    torch.autograd.backward(logits, grad))."""
    at, rows, vocab, ld, code, index = _place("logits", logits)
    ids, wide = _token_place(tokens, rows, index)
    if bufs is None:
        bufs = PolicyBuffers.empty(rows, logits.device)
    if ws is None:
        ws = policy_workspace(logits)
    to, ldg = None, 0
    if grad is not None:
        to, _, _, ldg, grad_code, grad_index = _place("grad", grad)
        if grad.shape != logits.shape or grad_code != code or grad_index != index:
            raise AspisError(ERR_INVALID_ARG, "grad must have the shape, type and device of logits")
    opt = PolicyOptions(clip[0], clip[1], kl, temperature, grad_scale)
    _enqueue(index, lib().aspis_policy_loss, at, rows, vocab, ld, code, ids, wide,
             _floats("old", old, rows, index), _floats("advantage", advantage, rows, index),
             _floats("weight", weight, rows, index),
             _floats("ref", ref, rows, index) if ref is not None else None, ctypes.byref(opt),
             _floats("bufs.sums", bufs.sums, 3, index, False),
             _floats("bufs.logps", bufs.logps, rows, index, False), to, ldg, _scratch_at(ws, index),
             ws.numel())
    return bufs
