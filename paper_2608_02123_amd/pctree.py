"""Python binding of ``libpctree.so`` (the C ABI declared in include/pctree.h).

Argument marshalling only: every step of a round runs in the library's HIP
kernels.  torch supplies device memory and the current HIP stream.  If the
library has not been built this module raises; there is no fallback path.
"""
from __future__ import annotations

import ctypes
import math
import operator
import os

import torch

__all__ = [
    "PCTreeError",
    "RoundAborted",
    "lib",
    "Shape",
    "workspace_bytes",
    "build_tree",
    "build_mask",
    "chain_decode",
    "build_retrieve",
    "accept_greedy",
    "compact_kv",
    "AttnShape",
    "attention_workspace_bytes",
    "tree_attention",
    "TreeAttention",
    "PagedBatch",
    "rope_table",
    "append_paged",
    "PagedAttention",
    "paged_attention",
    "compact_paged",
    "Sampler",
    "sample",
    "rms_norm",
    "adjust_logits",
    "TreeBuilder",
    "timeline_available",
    "timeline_read",
    "status_string",
    "DebugConfig",
    "debug_set",
    "F32",
    "BF16",
    "F16",
    "MODE_PARENT",
    "MODE_SHARED",
    "MODE_INDEPENDENT",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
# (PCTREE_LIB: another build of the same library, e.g. the host-sanitizer one)
LIB_PATH = os.environ.get("PCTREE_LIB") or os.path.join(_HERE, "libpctree.so")
# the stage-timeline build of the same library (include/pctree_profile.h)
TIMELINE_LIB_PATH = os.path.join(_HERE, "libpctree_timeline.so")
TIMELINE_WHO, TIMELINE_STAGES, TIMELINE_EVENTS = 5, 65, 8

OK, ERR_INVALID_ARGUMENT, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = range(5)
F32, BF16, F16 = 0, 1, 2
NOALLOC_SCRATCH_BYTES = 32 << 20  # PCTREE_NOALLOC_SCRATCH_BYTES
MODE_PARENT, MODE_SHARED, MODE_INDEPENDENT = 0, 1, 2  # pctree_mode


class PCTreeError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_string(status)}")
        self.status = status


class RoundAborted(RuntimeError):
    """A round was abandoned on the device (count = -1, every row padded)."""

    def __init__(self, requests):
        super().__init__(f"round abandoned for requests {list(requests)} (count = -1): a "
                         "workgroup of the single-launch round did not start in time")
        self.requests = list(requests)


class Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("vocab", "block", "budget", "topk", "rank", "requests", "dtype", "mode")]


class AttnShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("requests", "budget", "q_heads", "kv_heads", "head_dim", "capacity")] + \
               [("scale", ctypes.c_float)]


class _PagedCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("page_stride", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in
                ("pages", "page_size", "kv_heads", "head_dim", "dtype")]


class _PagedBatch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("row_start", "row_count", "prefix_len", "page_table")] + \
               [(n, ctypes.c_int32) for n in ("requests", "max_pages", "rows", "max_rows")]


class _Append(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "v", "q_out")] + \
               [(n, ctypes.c_int64) for n in
                ("q_stride", "k_stride", "v_stride", "q_out_stride")] + \
               [(n, ctypes.c_void_p) for n in ("q_norm", "k_norm", "rope", "position")] + \
               [("eps", ctypes.c_float)] + \
               [(n, ctypes.c_int32) for n in ("q_heads", "rot_dim", "positions", "interleaved")]


class _PagedCache8(ctypes.Structure):
    _fields_ = [("pages", _PagedCache), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("scale_stride", ctypes.c_int64),
                ("block", ctypes.c_int32)]


class _Norm(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "weight", "residual", "out", "scale")] + \
               [(n, ctypes.c_int64) for n in ("x_stride", "residual_stride", "out_stride")] + \
               [(n, ctypes.c_int32) for n in ("rows", "width", "group", "dtype")] + \
               [("eps", ctypes.c_float)]


class _Adjust(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("row_stride", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in
                ("row_start", "row_count", "history", "history_start", "history_count",
                 "prompt_count", "repetition", "frequency", "presence", "bias_token",
                 "bias_value", "bias_start", "bias_count", "token", "mask", "allowed",
                 "allowed_row")] + \
               [(n, ctypes.c_int32) for n in
                ("rows", "vocab", "requests", "max_rows", "history_total", "bias_total", "budget",
                 "masks", "dtype")]


class _Inputs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("base_logits", "emb", "proj_t", "depth_feat", "root_token", "prefix_len")]


class _Tree(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("token", "parent", "depth", "position", "logprob", "count", "mask")]


class _Trace(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("token", "parent_slot", "score")]


class DebugConfig(ctypes.Structure):
    """pctree_debug_config of include/pctree_profile.h (test-only launch overrides)."""
    _fields_ = [("wait_ticks", ctypes.c_int64), ("force_multilaunch", ctypes.c_int32),
                ("round_slices", ctypes.c_int32), ("wide_unbounded", ctypes.c_int32)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; "
                "g.build()'` (the HIP library is required; there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        L.pctree_workspace_bytes.argtypes = [ctypes.POINTER(Shape)]
        L.pctree_workspace_bytes.restype = sz
        L.pctree_build_tree.argtypes = [ctypes.POINTER(Shape), ctypes.POINTER(_Inputs),
                                        ctypes.POINTER(_Tree), ctypes.POINTER(_Trace), vp, sz, vp]
        L.pctree_build_tree.restype = ctypes.c_int
        L.pctree_build_tree_noalloc.argtypes = [ctypes.POINTER(Shape), ctypes.POINTER(_Inputs),
                                                ctypes.POINTER(_Tree), ctypes.POINTER(_Trace), vp]
        L.pctree_build_tree_noalloc.restype = ctypes.c_int
        L.pctree_build_mask.argtypes = [vp, vp, ctypes.c_int32, ctypes.c_int32, vp, vp]
        L.pctree_build_mask.restype = ctypes.c_int
        L.pctree_chain_decode.argtypes = [ctypes.POINTER(Shape), ctypes.POINTER(_Inputs), vp, vp,
                                          vp, sz, vp]
        L.pctree_chain_decode.restype = ctypes.c_int
        i32, i64 = ctypes.c_int32, ctypes.c_int64
        L.pctree_build_retrieve.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp]
        L.pctree_build_retrieve.restype = ctypes.c_int
        L.pctree_accept_greedy.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp]
        L.pctree_accept_greedy.restype = ctypes.c_int
        L.pctree_compact_kv.argtypes = [vp, i64, i64, i32, i32, i32, vp, vp, vp, i32, i32, i32,
                                        vp]
        L.pctree_compact_kv.restype = ctypes.c_int
        L.pctree_attention_workspace_bytes.argtypes = [ctypes.POINTER(AttnShape)]
        L.pctree_attention_workspace_bytes.restype = sz
        L.pctree_tree_attention.argtypes = [ctypes.POINTER(AttnShape), vp, vp, vp, vp, vp, vp, vp,
                                            vp, sz, vp]
        L.pctree_tree_attention.restype = ctypes.c_int
        cache, batch = ctypes.POINTER(_PagedCache), ctypes.POINTER(_PagedBatch)
        L.pctree_append_paged.argtypes = [cache, batch, ctypes.POINTER(_Append), vp]
        L.pctree_append_paged.restype = ctypes.c_int
        L.pctree_paged_attention_workspace_bytes.argtypes = [cache, batch, i32]
        L.pctree_paged_attention_workspace_bytes.restype = sz
        L.pctree_paged_attention.argtypes = [cache, batch, vp, i32, ctypes.c_float, vp, i32, vp,
                                             vp, sz, vp]
        L.pctree_paged_attention.restype = ctypes.c_int
        L.pctree_sample_workspace_bytes.argtypes = [i32, i32]
        L.pctree_sample_workspace_bytes.restype = sz
        L.pctree_sample.argtypes = [vp, i32, i32, i32, i64] + [vp] * 8 + [sz, vp]
        L.pctree_sample.restype = ctypes.c_int
        L.pctree_compact_paged.argtypes = [vp, i64, i64, i32, i32, i32, i32, i32, vp, i32, vp, vp,
                                           vp, i32, i32, i32, vp]
        L.pctree_compact_paged.restype = ctypes.c_int
        cache8 = ctypes.POINTER(_PagedCache8)
        L.pctree_append_paged8.argtypes = [cache8, batch, ctypes.POINTER(_Append), vp]
        L.pctree_append_paged8.restype = ctypes.c_int
        L.pctree_paged_attention8_workspace_bytes.argtypes = [cache8, batch, i32]
        L.pctree_paged_attention8_workspace_bytes.restype = sz
        L.pctree_paged_attention8.argtypes = [cache8, *L.pctree_paged_attention.argtypes[1:]]
        L.pctree_paged_attention8.restype = ctypes.c_int
        L.pctree_compact_paged8.argtypes = [vp, i64, i64, vp, i64, i64] + [i32] * 6 + \
            [vp, i32, vp, vp, vp, i32, i32, i32, vp]
        L.pctree_compact_paged8.restype = ctypes.c_int
        L.pctree_rms_norm.argtypes = [ctypes.POINTER(_Norm), vp]
        L.pctree_rms_norm.restype = ctypes.c_int
        L.pctree_adjust_logits.argtypes = [ctypes.POINTER(_Adjust), vp]
        L.pctree_adjust_logits.restype = ctypes.c_int
        L.pctree_status_string.argtypes = [ctypes.c_int]
        L.pctree_status_string.restype = ctypes.c_char_p
        L.pctree_abi_version.argtypes = []
        L.pctree_abi_version.restype = ctypes.c_int32
        L.pctree_profile_enable.argtypes = [ctypes.c_int32]
        L.pctree_profile_enable.restype = ctypes.c_int
        L.pctree_profile_read.argtypes = [ctypes.POINTER(ctypes.c_double),
                                          ctypes.POINTER(ctypes.c_int64),
                                          ctypes.POINTER(ctypes.c_char_p)]
        L.pctree_profile_read.restype = ctypes.c_int
        L.pctree_debug_set.argtypes = [ctypes.POINTER(DebugConfig)]
        L.pctree_debug_set.restype = ctypes.c_int
        L.pctree_timeline_available.argtypes = []
        L.pctree_timeline_available.restype = ctypes.c_int32
        L.pctree_timeline_read.argtypes = [vp, ctypes.POINTER(ctypes.c_double)]
        L.pctree_timeline_read.restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().pctree_status_string(status).decode()


def _check(status: int, what: str) -> None:
    if status != OK:
        raise PCTreeError(status, what)


# (addresses go to the C entry points as plain integers, which their argument
# types convert: wrapping each one, and a stream object per call, took as long
# as a small kernel)
def _ptr(t):
    return None if t is None else t.data_ptr()


# (the current stream's handle without a stream object, where this torch has it)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None):
    if stream is None and _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return (stream if stream is not None else torch.cuda.current_stream()).cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}: float32 or bfloat16 expected")


def make_shape(V, B, N, k, r, R, dtype, mode=0) -> Shape:
    return Shape(V, B, N, k, r, R, dtype, mode)


def workspace_bytes(V, B, N, k, r, R=1, dtype=BF16) -> int:
    return int(lib().pctree_workspace_bytes(ctypes.byref(make_shape(V, B, N, k, r, R, dtype))))


_TORCH_DTYPE = {F32: torch.float32, BF16: torch.bfloat16}


def check_inputs(shape: Shape, L, E, Wt, h, root, prefix_len, *, device=True) -> None:
    """Raise unless every input has exactly the layout ``shape`` describes:
    ``L [R][B][V]``, ``E [V][r]`` and ``Wt [V][r]`` in the shape's dtype,
    ``h [R][B][r]`` float32, ``root [R]`` and ``prefix_len [R]`` int32, all
    contiguous (and on a GPU when ``device``).  The kernels index these
    tensors by the shape alone, so a smaller tensor would be read past its end.
    """
    V, B, r, R = shape.vocab, shape.block, shape.rank, shape.requests
    dt = _TORCH_DTYPE.get(shape.dtype)
    _check_input("L", L, (R, B, V), dt, device)
    _check_input("E", E, (V, r), dt, device)
    _check_input("Wt", Wt, (V, r), dt, device)
    _check_input("h", h, (R, B, r), torch.float32, device)
    _check_input("root", root, (R,), torch.int32, device)
    _check_input("prefix_len", prefix_len, (R,), torch.int32, device)


def _check_input(name, t, shp, dt, device):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if dt is None or t.dtype != dt:
        raise TypeError(f"{name} must be {dt}, got {t.dtype}")
    if t.shape != shp:
        raise ValueError(f"{name} must have shape {shp}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if device and not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")


def _inputs(shape, L, E, Wt, h, root, prefix_len):
    check_inputs(shape, L, E, Wt, h, root, prefix_len)
    return _Inputs(*(t.data_ptr() for t in (L, E, Wt, h, root, prefix_len)))


def check_counts(count) -> None:
    """Raise RoundAborted if a request's count is -1 (waits for the stream)."""
    c = count.cpu()
    bad = (c == -1).nonzero().flatten().tolist()
    if bad:
        raise RoundAborted(bad)


class TreeBuilder:
    """Pre-allocated outputs and workspace for repeated rounds of one shape.

    ``run(L, E, Wt, h, root, prefix_len)`` enqueues one round on the current
    stream and returns the output tensors (overwritten by the next call).
    With ``check=True`` it then waits for the round and raises
    :class:`RoundAborted` if the device abandoned it (count = -1).
    """

    def __init__(self, V, B, N, k, r, R=1, dtype=BF16, device="cuda", mask=True, trace=False,
                 mode=MODE_PARENT, workspace=True):
        self.shape = make_shape(V, B, N, k, r, R, dtype, mode)
        nbytes = int(lib().pctree_workspace_bytes(ctypes.byref(self.shape)))
        if nbytes == 0:
            _check(lib().pctree_build_tree(ctypes.byref(self.shape), None, None, None, None, 0,
                                           None), "shape")
        # workspace=False: only run_noalloc() (the library's own scratch array)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device) if workspace \
            else None
        i32 = dict(dtype=torch.int32, device=device)
        self.out = {
            "token": torch.empty(R, N, **i32),
            "parent": torch.empty(R, N, **i32),
            "depth": torch.empty(R, N, **i32),
            "position": torch.empty(R, N, **i32),
            "logprob": torch.empty(R, N, dtype=torch.float32, device=device),
            "count": torch.empty(R, **i32),
        }
        if mask:
            self.out["mask"] = torch.empty(R, N, (N + 31) // 32, **i32)
        self._tree = _Tree(*(self.out[n].data_ptr() for n in
                             ("token", "parent", "depth", "position", "logprob", "count")),
                           self.out["mask"].data_ptr() if mask else None)
        self._trace = None
        if trace:
            self.out["trace_token"] = torch.empty(R, B, k, **i32)
            self.out["trace_parent_slot"] = torch.empty(R, B, k, **i32)
            self.out["trace_score"] = torch.empty(R, B, k, dtype=torch.float32, device=device)
            self._trace = _Trace(self.out["trace_token"].data_ptr(),
                                 self.out["trace_parent_slot"].data_ptr(),
                                 self.out["trace_score"].data_ptr())

    def run(self, L, E, Wt, h, root, prefix_len, stream=None, check=False):
        self.bind(L, E, Wt, h, root, prefix_len)
        return self.launch(stream, check=check)

    def bind(self, L, E, Wt, h, root, prefix_len):
        """Check and remember the inputs once; ``launch()`` then only enqueues."""
        self._inp = _inputs(self.shape, L, E, Wt, h, root, prefix_len)
        self._keep = (L, E, Wt, h, root, prefix_len)
        self._args = (ctypes.byref(self.shape), ctypes.byref(self._inp), ctypes.byref(self._tree),
                      ctypes.byref(self._trace) if self._trace is not None else None)

    def launch(self, stream=None, check=False):
        if self.workspace is None:
            raise RuntimeError("this builder has no workspace: use run_noalloc()")
        st = lib().pctree_build_tree(*self._args, self.workspace.data_ptr(),
                                     self.workspace.numel(), _stream(stream))
        _check(st, "pctree_build_tree")
        if check:
            check_counts(self.out["count"])
        return self.out

    def run_noalloc(self, L, E, Wt, h, root, prefix_len, stream=None, check=False):
        """The same round through pctree_build_tree_noalloc: no workspace
        argument, the library's fixed per-device scratch array instead."""
        self.bind(L, E, Wt, h, root, prefix_len)
        st = lib().pctree_build_tree_noalloc(*self._args, _stream(stream))
        _check(st, "pctree_build_tree_noalloc")
        if check:
            check_counts(self.out["count"])
        return self.out


def build_tree(L, E, Wt, h, root, prefix_len, k, N, *, mask=True, trace=False, stream=None,
               mode=MODE_PARENT, check=True):
    """One round for tensors ``L [R][B][V]``, ``E [V][r]``, ``Wt [V][r]``, ``h [R][B][r]``.

    Returns a dict of freshly allocated output tensors (see include/pctree.h).
    With ``check`` (the default) it waits for the round and raises
    :class:`RoundAborted` if the device abandoned it.
    """
    R, B, V = L.shape
    r = E.shape[1]
    b = TreeBuilder(V, B, N, k, r, R, _dtype_code(L), device=L.device, mask=mask, trace=trace,
                    mode=mode)
    return b.run(L, E, Wt, h, root, prefix_len, stream=stream, check=check)


def debug_set(wait_ticks: int = -1, force_multilaunch: bool = False,
              round_slices: int = 0, wide_unbounded: bool = False) -> None:
    """Test-only launch overrides (pctree_debug_set); no arguments restores the defaults."""
    cfg = DebugConfig(int(wait_ticks), 1 if force_multilaunch else 0, int(round_slices),
                      1 if wide_unbounded else 0)
    _check(lib().pctree_debug_set(ctypes.byref(cfg)), "pctree_debug_set")


def profile_enable(on: bool = True) -> None:
    """Bracket the dominant kernel's launches with hipEvents (include/pctree_profile.h)."""
    _check(lib().pctree_profile_enable(1 if on else 0), "pctree_profile_enable")


def profile_read():
    """(total milliseconds, launches, kernel name) recorded since enabling; clears them."""
    ms, n, name = ctypes.c_double(), ctypes.c_int64(), ctypes.c_char_p()
    _check(lib().pctree_profile_read(ctypes.byref(ms), ctypes.byref(n), ctypes.byref(name)),
           "pctree_profile_read")
    return ms.value, n.value, name.value.decode()


def timeline_available() -> bool:
    """Whether the loaded library is the stage-timeline build."""
    return bool(lib().pctree_timeline_available())


def timeline_read():
    """The stage timeline's stamps in microseconds, as a float64 array
    [who][stage][event] (NaN where not stamped), zeroing them
    (pctree_timeline_read; waits for the current device first)."""
    import numpy as np

    torch.cuda.synchronize()
    n = TIMELINE_WHO * TIMELINE_STAGES * TIMELINE_EVENTS
    buf = (ctypes.c_int64 * n)()
    rate = ctypes.c_double()
    _check(lib().pctree_timeline_read(ctypes.cast(buf, ctypes.c_void_p), ctypes.byref(rate)),
           "pctree_timeline_read")
    ticks = np.frombuffer(buf, dtype=np.int64).reshape(TIMELINE_WHO, TIMELINE_STAGES,
                                                       TIMELINE_EVENTS)
    return np.where(ticks > 0, ticks / rate.value, np.nan)


def build_mask(parent, count, stream=None):
    """Ancestor mask ``[R][N][ceil(N/32)]`` (int32 view of uint32 words)."""
    if parent.dtype != torch.int32 or count.dtype != torch.int32:
        raise TypeError("parent and count must be int32")
    if not (parent.is_cuda and count.is_cuda and parent.is_contiguous()):
        raise ValueError("parent and count must be contiguous device tensors")
    R, N = parent.shape
    mask = torch.empty(R, N, (N + 31) // 32, dtype=torch.int32, device=parent.device)
    st = lib().pctree_build_mask(_ptr(parent), _ptr(count), R, N, _ptr(mask), _stream(stream))
    _check(st, "pctree_build_mask")
    return mask


def chain_decode(L, E, Wt, h, root, prefix_len=None, stream=None, mode=MODE_PARENT):
    """The greedy chain of Eq. 1: returns (tokens [R][B+1], cumulative logprobs [R][B+1])."""
    R, B, V = L.shape
    r = E.shape[1]
    if prefix_len is None:
        prefix_len = torch.zeros(R, dtype=torch.int32, device=L.device)
    shape = make_shape(V, B, 1, 1, r, R, _dtype_code(L), mode)
    nbytes = int(lib().pctree_workspace_bytes(ctypes.byref(shape)))
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=L.device)
    toks = torch.empty(R, B + 1, dtype=torch.int32, device=L.device)
    lps = torch.empty(R, B + 1, dtype=torch.float32, device=L.device)
    inp = _inputs(shape, L, E, Wt, h, root, prefix_len)
    st = lib().pctree_chain_decode(ctypes.byref(shape), ctypes.byref(inp), _ptr(toks), _ptr(lps),
                                   ws.data_ptr(), ws.numel(), _stream(stream))
    _check(st, "pctree_chain_decode")
    return toks, lps


def _int32_dev(name, t):
    if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous int32 device tensor")


def build_retrieve(parent, count, max_depth, stream=None):
    """Retrieve rows of emitted trees: (rows [R][N][max_depth+1], nrows [R]) int32."""
    _int32_dev("parent", parent)
    _int32_dev("count", count)
    R, N = parent.shape
    dev = parent.device
    rows = torch.empty((R, N, max_depth + 1), dtype=torch.int32, device=dev)
    nrows = torch.empty((R,), dtype=torch.int32, device=dev)
    st = lib().pctree_build_retrieve(_ptr(parent), _ptr(count), R, N, max_depth, _ptr(rows),
                                     _ptr(nrows), _stream(stream))
    _check(st, "pctree_build_retrieve")
    return rows, nrows


def accept_greedy(token, rows, nrows, target_next, stream=None):
    """Greedy tree acceptance over retrieve rows; returns a dict of int32 tensors
    ``accept_len [R]``, ``accept_row [R]``, ``accept_node [R][W]``, ``bonus [R]``."""
    for name, t in (("token", token), ("rows", rows), ("nrows", nrows),
                    ("target_next", target_next)):
        _int32_dev(name, t)
    R, N, W = rows.shape
    if token.shape != (R, N) or target_next.shape != (R, N):
        raise ValueError("token and target_next must be [R][N] like the rows")
    i32 = dict(dtype=torch.int32, device=rows.device)
    out = {"accept_len": torch.empty(R, **i32), "accept_row": torch.empty(R, **i32),
           "accept_node": torch.empty(R, W, **i32), "bonus": torch.empty(R, **i32)}
    st = lib().pctree_accept_greedy(_ptr(token), _ptr(rows), _ptr(nrows), _ptr(target_next), R, N,
                                    W - 1, _ptr(out["accept_len"]), _ptr(out["accept_row"]),
                                    _ptr(out["accept_node"]), _ptr(out["bonus"]), _stream(stream))
    _check(st, "pctree_accept_greedy")
    return out


def compact_kv(cache, prefix_len, accept_node, accept_len, budget, stream=None):
    """Move each request's accepted cache slots right after its prefix, in place.

    ``cache [R][groups][capacity][...]`` is any contiguous device tensor whose
    trailing dimensions form one slot (a multiple of 16 bytes).
    """
    if not cache.is_cuda or not cache.is_contiguous() or cache.dim() < 3:
        raise ValueError("cache must be a contiguous [R][groups][capacity][...] device tensor")
    for name, t in (("prefix_len", prefix_len), ("accept_node", accept_node),
                    ("accept_len", accept_len)):
        _int32_dev(name, t)
    R, G, T = cache.shape[:3]
    es = cache.element_size()
    slot = math.prod(cache.shape[3:]) * es
    st = lib().pctree_compact_kv(_ptr(cache), cache.stride(0) * es, cache.stride(1) * es, G, T,
                                 slot, _ptr(prefix_len), _ptr(accept_node), _ptr(accept_len), R,
                                 budget, accept_node.shape[1] - 1, _stream(stream))
    _check(st, "pctree_compact_kv")
    return cache


def attention_workspace_bytes(R, N, Hq, Hkv, D, C, scale=None) -> int:
    sc = float(scale) if scale is not None else D ** -0.5
    return int(lib().pctree_attention_workspace_bytes(ctypes.byref(
        AttnShape(R, N, Hq, Hkv, D, C, sc))))


class TreeAttention:
    """One tree-attention layer shape with its workspace, for repeated calls."""

    def __init__(self, R, N, Hq, Hkv, D, C, scale=None, device="cuda"):
        self.shape = AttnShape(R, N, Hq, Hkv, D, C,
                               float(scale) if scale is not None else D ** -0.5)
        nb = int(lib().pctree_attention_workspace_bytes(ctypes.byref(self.shape)))
        self.workspace = torch.empty(max(nb, 1), dtype=torch.uint8, device=device)
        self.ws_bytes = nb
        self.device = device

    def __call__(self, q, k, v, mask, count, prefix_len, out=None, stream=None):
        s = self.shape
        R, N, Hq, Hkv, D, C = s.requests, s.budget, s.q_heads, s.kv_heads, s.head_dim, s.capacity
        for name, t, shp in (("q", q, (R, N, Hq, D)), ("k", k, (R, Hkv, C, D)),
                             ("v", v, (R, Hkv, C, D))):
            if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() \
                    or t.shape != shp:
                raise ValueError(f"{name} must be a contiguous bf16 device tensor {shp}")
        if mask.dtype != torch.int32 and mask.dtype != torch.uint32:
            raise TypeError("mask must be the [R][N][(N+31)/32] words of build_mask")
        if mask.shape != (R, N, (N + 31) // 32) or not mask.is_contiguous() \
                or not mask.is_cuda:
            raise ValueError("mask must be [R][N][(N+31)/32] and contiguous")
        _int32_dev("count", count)
        _int32_dev("prefix_len", prefix_len)
        if out is None:
            out = torch.empty((R, N, Hq, D), dtype=torch.bfloat16, device=q.device)
        st = lib().pctree_tree_attention(ctypes.byref(s), _ptr(q), _ptr(k), _ptr(v), _ptr(mask),
                                         _ptr(count), _ptr(prefix_len), _ptr(out),
                                         _ptr(self.workspace), self.ws_bytes, _stream(stream))
        _check(st, "pctree_tree_attention")
        return out


def tree_attention(q, k, v, mask, count, prefix_len, scale=None, stream=None):
    """Tree-masked attention of one target layer: q [R][N][Hq][D], k and v
    [R][Hkv][C][D] bf16, mask from ``build_mask``; returns out [R][N][Hq][D] bf16."""
    R, N, Hq, D = q.shape
    Hkv, C = k.shape[1], k.shape[2]
    return TreeAttention(R, N, Hq, Hkv, D, C, scale, device=q.device)(
        q, k, v, mask, count, prefix_len, stream=stream)


# ---------------------------------------------------------------------------
# the verification step over a paged cache
# ---------------------------------------------------------------------------

_HALVES = {torch.bfloat16: BF16, torch.float16: F16}


class _Here:
    """The calls' device and stream: device ``idx`` (an int, which is compared in a
    tenth of a device object's time), and its current stream or the one that is passed
    (what a call allocates is then that stream's)."""
    __slots__ = ("ctx", "idx")

    def __init__(self, idx, stream):
        self.ctx, self.idx = None, idx
        if stream is not None:
            if stream.device.index != idx:
                raise ValueError(f"the stream is one of {stream.device}, the tensors of cuda:{idx}")
            self.ctx = torch.cuda.stream(stream)
        elif idx != torch.cuda.current_device():
            self.ctx = torch.cuda.device(idx)

    def __enter__(self):
        if self.ctx is not None:
            self.ctx.__enter__()
        return _stream() if _raw_stream is None else _raw_stream(self.idx)

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.__exit__(*exc)


class _Workspace:
    """An object's workspace.  On a stream other than the one that it was made on the
    allocator is told, or a freed object's memory could have a new owner while that
    stream's kernels still use it."""
    __slots__ = ("tensor", "ptr", "bytes", "home")

    def __init__(self, nbytes, device):
        self.tensor = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)
        self.ptr, self.bytes = self.tensor.data_ptr(), nbytes
        self.home = (torch.cuda.current_stream(self.tensor.device).cuda_stream
                     if self.tensor.is_cuda else None)  # (without, calls are refused)

    def on(self, st):
        if st != self.home:
            self.tensor.record_stream(torch.cuda.current_stream())
        return self.ptr


def _size(name, x):
    """``x`` as an int that the C interface can take (ctypes keeps the low 32 bits of
    another one)."""
    x = operator.index(x)
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name} must lie in [-2^31, 2^31), got {x}")
    return x


def _device_tensor(name, t, dtype, shape, idx):
    """``t`` must be a contiguous tensor of that type and shape on device ``idx``."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype:
        raise TypeError(f"{name} must be a {dtype} tensor")
    if t.get_device() != idx or idx < 0:
        raise ValueError(f"{name} must be on the device of the other tensors")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


class PagedBatch:
    """Which rows of a call belong to which request, and the requests' pages.

    Row ``row_start[r] + i`` (``i < row_count[r]``) is request ``r``'s i-th new
    row and sits at slot ``prefix_len[r] + i``, that is slot ``% page_size`` of
    page ``page_table[r][slot // page_size]`` (an entry that is no page's index
    stands for no page).  All are int32 device tensors whose contents may change
    from call to call; ``rows`` is the row count of q, k, v and out, ``max_rows``
    the most rows any request has.  Give it: without it one request may have them
    all, and the attention is planned for that (64 single tokens 174 us for 144).
    """

    def __init__(self, row_start, row_count, prefix_len, page_table, rows, max_rows=None):
        self.rows = _size("rows", int(rows))
        self.max_rows = self.rows if max_rows is None else _size("max_rows", int(max_rows))
        if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
            raise ValueError("page_table must be an [R][max_pages] tensor")
        R, W = page_table.shape
        self.idx = page_table.get_device()
        for name, t, shp in (("page_table", page_table, (R, W)), ("row_start", row_start, (R,)),
                             ("row_count", row_count, (R,)), ("prefix_len", prefix_len, (R,))):
            _device_tensor(name, t, torch.int32, shp, self.idx)
        self.requests, self.max_pages = R, W
        self.device = page_table.device
        self._keep = (row_start, row_count, prefix_len, page_table)
        self.sizes = self.requests, self.max_pages, self.rows, self.max_rows
        self._c = _PagedBatch(*(t.data_ptr() for t in self._keep), *(R, W, self.rows, self.max_rows))
        self._ref = ctypes.byref(self._c)


_HELD, _SCALE = torch.float8_e4m3fn, torch.float8_e8m0fnu
_HELD_ONLY = (_HELD,)


def _paged_cache(k, v, idx, rows=None):
    """The C view of one layer's pages [pages][Hkv][page_size][D]; the pages may lie
    apart (stride 0 is free, the same for both).  ``rows``: the new rows' type, where
    the pages are held in 8 bits."""
    types = _HALVES if rows is None else _HELD_ONLY
    for name, t in (("k_cache", k), ("v_cache", v)):
        if not isinstance(t, torch.Tensor) or t.dtype not in types:
            raise TypeError(f"{name} must be a bfloat16 or float16 tensor" if rows is None else
                            f"{name} must be a float8_e4m3fn tensor")
        if t.dim() != 4 or t.get_device() != idx or idx < 0:
            raise ValueError(f"{name} must be a [pages][Hkv][page_size][D] tensor on the batch's "
                             "device")
    pages, Hkv, P, D = shape = k.shape
    ks, vs = k.stride(), v.stride()
    if shape != v.shape or k.dtype is not v.dtype or (pages > 1 and ks[0] != vs[0]):
        raise ValueError("k_cache and v_cache must have one shape, type and page stride")
    inner = (P * D, D, 1)
    if (ks[1:] != inner and not k[0].is_contiguous()) or \
            (vs[1:] != inner and not v[0].is_contiguous()):
        raise ValueError("a page's [Hkv][page_size][D] must be contiguous")
    return _PagedCache(k.data_ptr(), v.data_ptr(), ks[0] if pages > 1 else Hkv * P * D, pages, P,
                       Hkv, D, _HALVES[rows or k.dtype])


def _held_cache(k, v, k_scale, v_scale, rows, idx):
    """The C view of one layer's pages in 8 bits, with their scales [pages][Hkv][page_size /
    block]; ``rows``: the type of the new rows."""
    if rows not in _HALVES:
        raise TypeError("the rows must be bfloat16 or float16 tensors")
    for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
        if not isinstance(t, torch.Tensor) or t.dtype is not _SCALE:
            raise TypeError(f"{name} must be a float8_e8m0fnu tensor beside pages in 8 bits")
    c = _paged_cache(k, v, idx, rows)
    if k_scale.dim() != 3 or k_scale.get_device() != idx or v_scale.get_device() != idx:
        raise ValueError("k_scale and v_scale must be [pages][Hkv][page_size / block] tensors on the "
                         "batch's device")
    pages, Hkv, n = shape = k_scale.shape
    ks, vs = k_scale.stride(), v_scale.stride()
    if pages != c.pages or Hkv != c.kv_heads or shape != v_scale.shape or \
            (pages > 1 and ks[0] != vs[0]):
        raise ValueError("k_scale and v_scale must be of the pages' and heads' number, with one shape "
                         "and page stride")
    if n < 1 or c.page_size % n:
        raise ValueError(f"{n} scales do not divide a page of {c.page_size} slots")
    if (ks[1:] != (n, 1) and not k_scale[0].is_contiguous()) or \
            (vs[1:] != (n, 1) and not v_scale[0].is_contiguous()):
        raise ValueError("a page's scales must be contiguous")
    return _PagedCache8(c, k_scale.data_ptr(), v_scale.data_ptr(), ks[0] if pages > 1 else Hkv * n,
                        c.page_size // n)


def _row_tensor(name, t, T, D, dtype, idx):
    """Row stride of a [T][heads][D] tensor whose rows may lie apart, and its heads."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype:
        raise TypeError(f"{name} must be a {dtype} tensor")
    if t.dim() != 3 or t.get_device() != idx:
        raise ValueError(f"{name} must be a [{T}][heads][{D}] tensor on the batch's device")
    rows, heads, d = t.shape
    if rows != T or d != D:
        raise ValueError(f"{name} must be a [{T}][heads][{D}] tensor, got {tuple(t.shape)}")
    st = t.stride()
    if (st[1] != D or st[2] != 1) and not t[0].is_contiguous():
        raise ValueError(f"a row of {name} must be contiguous")
    return (st[0] if T > 1 else heads * D), heads


def rope_table(positions, rot_dim, theta=10000.0, device="cuda"):
    """The table that :func:`append_paged` rotates by: ``[positions][rot_dim]`` float32,
    the cosines of a position's ``rot_dim / 2`` angles ``p * theta^(-2 i / rot_dim)``,
    then their sines.  The angles are float64: far positions have many turns."""
    if rot_dim < 16 or rot_dim % 16:
        raise ValueError("rot_dim must be a multiple of 16")
    inv = float(theta) ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device)
                           / rot_dim)
    a = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * inv
    return torch.cat([a.cos(), a.sin()], 1).float()


def append_paged(batch, k_cache, v_cache, k, v, q=None, *, q_norm=None, k_norm=None, eps=1e-6,
                 rope=None, interleaved=False, position=None, q_out=None, k_scale=None,
                 v_scale=None, stream=None):
    """New rows into their pages: ``k``, ``v [T][Hkv][D]`` and, if given, ``q [T][Hq][D]``
    (views of a fused projection will do) are normed per head (``q_norm``, ``k_norm
    [D]``: root mean square), rotated by ``rope`` (:func:`rope_table`) at ``position
    [T]`` (a row's slot if not given); keys and values go to the rows' slots.
    Returns the normed and rotated q in ``q_out`` (a new tensor if not given; rows
    of no request are not written).

    Pages of float8_e4m3fn are held in 8 bits, with scales ``k_scale, v_scale
    [pages][Hkv][page_size / block]`` float8_e8m0fnu, a block being 8, 16, 32 or 64 slots
    (include/pctree.h)."""
    idx, T = batch.idx, batch.rows
    if k_scale is None and v_scale is None:
        c = whole = _paged_cache(k_cache, v_cache, idx)
        dt, call = k_cache.dtype, lib().pctree_append_paged
    else:
        dt, call = getattr(k, "dtype", None), lib().pctree_append_paged8
        whole = _held_cache(k_cache, v_cache, k_scale, v_scale, dt, idx)
        c = whole.pages
    D = c.head_dim
    ks, kh = _row_tensor("k", k, T, D, dt, idx)
    vs, vh = _row_tensor("v", v, T, D, dt, idx)
    if kh != c.kv_heads or vh != kh:
        raise ValueError(f"k and v must have the cache's {c.kv_heads} heads")
    if q_norm is not None:
        _device_tensor("q_norm", q_norm, dt, (D,), idx)
    if k_norm is not None:
        _device_tensor("k_norm", k_norm, dt, (D,), idx)
    if position is not None:
        _device_tensor("position", position, torch.int32, (T,), idx)
    rot = npos = 0
    if rope is not None:
        if not isinstance(rope, torch.Tensor) or rope.dim() != 2:
            raise ValueError("rope must be a [positions][rot_dim] tensor")
        npos, rot = rope.shape
        _device_tensor("rope", rope, torch.float32, (npos, rot), idx)
    if q is None and (q_out is not None or q_norm is not None):
        raise ValueError("q_out and q_norm go with q")
    with _Here(idx, stream) as st:
        qs = os_ = Hq = 0
        if q is not None:
            qs, Hq = _row_tensor("q", q, T, D, dt, idx)
            if q_out is None:
                q_out = q.new_empty((T, Hq, D))
            os_, oh = _row_tensor("q_out", q_out, T, D, dt, idx)
            if oh != Hq:
                raise ValueError("q_out must have q's shape")
        a = _Append(_ptr(q), k.data_ptr(), v.data_ptr(), _ptr(q_out), qs, ks, vs, os_,
                    _ptr(q_norm), _ptr(k_norm), _ptr(rope), _ptr(position), eps, Hq, rot, npos,
                    1 if interleaved else 0)
        status = call(ctypes.byref(whole), batch._ref, ctypes.byref(a), st)
    _check(status, call.__name__)
    return q_out


class PagedAttention:
    """Attention of a batch's new rows over paged caches, with its workspace, for
    repeated calls of one size (calls that may overlap need an object each), over pages in
    16 bits and in 8."""

    def __init__(self, batch, q_heads, kv_heads, head_dim, page_size, scale=None):
        self.sizes = batch.sizes
        self.q_heads, self.kv_heads = _size("q_heads", q_heads), _size("kv_heads", kv_heads)
        self.head_dim, self.page_size = _size("head_dim", head_dim), _size("page_size", page_size)
        self.scale = float(scale) if scale is not None else head_dim ** -0.5
        Hkv, P, D = self.kv_heads, self.page_size, self.head_dim
        c = _PagedCache(None, None, Hkv * P * D, 1, P, Hkv, D, BF16)
        held = _PagedCache8(_PagedCache(None, None, -(-Hkv * P * D // 16) * 16, 1, P, Hkv, D, BF16),
                            None, None, max(Hkv * P, 1), 8)
        self.ws_bytes = max(int(lib().pctree_paged_attention_workspace_bytes(
            ctypes.byref(c), batch._ref, self.q_heads)), int(
                lib().pctree_paged_attention8_workspace_bytes(ctypes.byref(held), batch._ref,
                                                              self.q_heads)))
        self.idx = batch.idx
        self._ws = _Workspace(self.ws_bytes, batch.device)
        self.workspace = self._ws.tensor

    def __call__(self, q, k_cache, v_cache, batch, mask=None, out=None, stream=None, *,
                 k_scale=None, v_scale=None):
        """``q [T][Hq][D]`` over ``k_cache, v_cache [pages][Hkv][page_size][D]``; causal, or
        with ``mask`` (:func:`build_mask`) the tree's.  Returns ``out [T][Hq][D]``
        (rows of no request are not written).  Pages in 8 bits come with their
        scales, as in :func:`append_paged`."""
        idx = self.idx
        if batch.sizes != self.sizes or batch.idx != idx:
            raise ValueError("the batch is not of this object's sizes")
        if k_scale is None and v_scale is None:
            c = whole = _paged_cache(k_cache, v_cache, idx)
            dt, call = k_cache.dtype, lib().pctree_paged_attention
        else:
            dt, call = getattr(q, "dtype", None), lib().pctree_paged_attention8
            whole = _held_cache(k_cache, v_cache, k_scale, v_scale, dt, idx)
            c = whole.pages
        if c.kv_heads != self.kv_heads or c.head_dim != self.head_dim or \
                c.page_size != self.page_size:
            raise ValueError("the pages are not of this object's sizes")
        shp = (batch.rows, self.q_heads, self.head_dim)
        _device_tensor("q", q, dt, shp, idx)
        budget = 0
        if mask is not None:
            if mask.dtype != torch.int32 and mask.dtype != torch.uint32:
                raise TypeError("mask must be the [R][N][(N+31)/32] words of build_mask")
            budget = mask.shape[1] if mask.dim() == 3 else 0
            _device_tensor("mask", mask, mask.dtype,
                           (batch.requests, budget, (budget + 31) // 32), idx)
        if out is not None:
            _device_tensor("out", out, dt, shp, idx)
        with _Here(idx, stream) as st:
            if out is None:
                out = torch.empty(shp, dtype=q.dtype, device=q.device)
            status = call(
                ctypes.byref(whole), batch._ref, q.data_ptr(), self.q_heads, self.scale, _ptr(mask),
                budget, out.data_ptr(), self._ws.on(st), self.ws_bytes, st)
        _check(status, call.__name__)
        return out


def paged_attention(q, k_cache, v_cache, batch, mask=None, scale=None, out=None, stream=None, *,
                    k_scale=None, v_scale=None):
    """One call of :class:`PagedAttention`."""
    with _Here(batch.idx, stream):
        layer = PagedAttention(batch, q.shape[1], k_cache.shape[1], k_cache.shape[3],
                               k_cache.shape[2], scale)
        return layer(q, k_cache, v_cache, batch, mask=mask, out=out, k_scale=k_scale,
                     v_scale=v_scale)


def compact_paged(pool, page_table, prefix_len, accept_node, accept_len, budget, stream=None, *,
                  scale=None):
    """Move each request's accepted slots right after its prefix, in place.

    ``pool [groups][pages][heads][page_size][...]`` (e.g. every layer's K and V):
    the dimensions past ``page_size`` form a slot of a head, a multiple of 16 bytes;
    groups and pages may lie apart.  Pages in 8 bits (``pool [groups][pages][heads]
    [page_size][D]`` float8_e4m3fn) come with ``scale [groups][pages][heads][page_size /
    block]`` float8_e8m0fnu, which moves and grows with them."""
    budget = _size("budget", budget)
    if not isinstance(pool, torch.Tensor) or not pool.is_cuda or pool.dim() < 5 or \
            not (pool.is_contiguous() or pool[0, 0].is_contiguous()):
        raise ValueError("pool must be a [groups][pages][heads][page_size][...] device tensor "
                         "with contiguous pages")
    G, pages, heads, P = shape = pool.shape[:4]
    idx = pool.get_device()
    R, W = accept_node.shape
    _device_tensor("page_table", page_table, torch.int32, (R, page_table.shape[-1]), idx)
    _device_tensor("accept_node", accept_node, torch.int32, (R, W), idx)
    _device_tensor("prefix_len", prefix_len, torch.int32, (R,), idx)
    _device_tensor("accept_len", accept_len, torch.int32, (R,), idx)
    es = pool.element_size()
    slot = math.prod(pool.shape[4:]) * es
    stride = pool.stride()
    page_stride = stride[1] * es if pages > 1 else heads * P * slot
    group_stride = stride[0] * es if G > 1 else 0
    if scale is not None:
        if pool.dtype is not _HELD or pool.dim() != 5:
            raise ValueError("scales go with a float8_e4m3fn pool [groups][pages][heads][page_size][D]")
        return _compact_held(pool, group_stride, page_stride, scale, page_table, prefix_len,
                             accept_node, accept_len, budget, stream)
    with _Here(idx, stream) as st:
        status = lib().pctree_compact_paged(
            pool.data_ptr(), group_stride, page_stride, *shape, slot, page_table.data_ptr(),
            page_table.shape[1], prefix_len.data_ptr(), accept_node.data_ptr(),
            accept_len.data_ptr(), R, budget, W - 1, st)
    _check(status, "pctree_compact_paged")
    return pool


def _compact_held(pool, group_stride, page_stride, scale, page_table, prefix_len, accept_node,
                  accept_len, budget, stream):
    G, pages, heads, P, D = pool.shape
    idx = pool.get_device()
    if not isinstance(scale, torch.Tensor) or scale.dtype is not _SCALE:
        raise TypeError("scale must be a float8_e8m0fnu tensor")
    n, ss = scale.shape[-1] if scale.dim() == 4 else 0, scale.stride()
    if n < 1 or P % n or scale.shape != (G, pages, heads, n) or scale.get_device() != idx or \
            (ss[2:] != (n, 1) and not scale[0, 0].is_contiguous()):
        raise ValueError(f"scale must be a [{G}][{pages}][{heads}][{P} / block] tensor on the pool's "
                         "device, a page's scales contiguous")
    R, W = accept_node.shape
    with _Here(idx, stream) as st:
        status = lib().pctree_compact_paged8(
            pool.data_ptr(), group_stride, page_stride, scale.data_ptr(), ss[0] if G > 1 else 0,
            ss[1] if pages > 1 else heads * n, G, pages, heads, P, D, P // n,
            page_table.data_ptr(), page_table.shape[1], prefix_len.data_ptr(),
            accept_node.data_ptr(), accept_len.data_ptr(), R, budget, W - 1, st)
    _check(status, "pctree_compact_paged8")
    return pool


_LOGITS = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


class Sampler:
    """Sampling of up to ``rows`` rows over ``vocab`` tokens, with its workspace, for
    repeated calls (calls that may overlap need an object each)."""

    def __init__(self, rows, vocab, device="cuda"):
        self.rows, self.vocab = _size("rows", rows), _size("vocab", vocab)
        nb = int(lib().pctree_sample_workspace_bytes(rows, vocab))
        if nb == 0:
            _check(lib().pctree_sample(None, F32, rows, vocab, vocab, *([None] * 8), 0, None),
                   "sizes")
        self._ws = _Workspace(nb, device)
        self.workspace = self._ws.tensor
        self.idx = self.workspace.get_device()

    def __call__(self, logits, uniform, *, temperature=None, top_k=None, top_p=None, min_p=None,
                 token=None, logprob=None, stream=None):
        """A token per row of ``logits [T][V]`` (float32, bfloat16 or float16; rows may lie
        apart) from ``uniform [T]`` in [0, 1).  ``temperature``, ``top_p``, ``min_p``
        (float32) and ``top_k`` (int32) are ``[T]`` or None; see include/pctree.h.
        Returns ``(token [T] int32, logprob [T] float32)``."""
        idx = self.idx
        if not isinstance(logits, torch.Tensor) or logits.dtype not in _LOGITS:
            raise TypeError("logits must be a float32, bfloat16 or float16 tensor")
        if logits.dim() != 2 or logits.get_device() != idx or logits.shape[1] != self.vocab or \
                not 1 <= logits.shape[0] <= self.rows:
            raise ValueError(f"logits must be a [T][{self.vocab}] tensor on {self.workspace.device}"
                             f", T at most {self.rows}")
        T, V = logits.shape
        stride = logits.stride()
        if (V > 1 and stride[1] != 1) or (T > 1 and stride[0] < V):
            raise ValueError("a row of logits must be contiguous, rows must not overlap")
        one = (T,)
        _device_tensor("uniform", uniform, torch.float32, one, idx)
        if temperature is not None:
            _device_tensor("temperature", temperature, torch.float32, one, idx)
        if top_k is not None:
            _device_tensor("top_k", top_k, torch.int32, one, idx)
        if top_p is not None:
            _device_tensor("top_p", top_p, torch.float32, one, idx)
        if min_p is not None:
            _device_tensor("min_p", min_p, torch.float32, one, idx)
        if token is not None:
            _device_tensor("token", token, torch.int32, one, idx)
        if logprob is not None:
            _device_tensor("logprob", logprob, torch.float32, one, idx)
        with _Here(idx, stream) as st:
            if token is None:
                token = torch.empty(T, dtype=torch.int32, device=logits.device)
            if logprob is None:
                logprob = torch.empty(T, dtype=torch.float32, device=logits.device)
            status = lib().pctree_sample(
                logits.data_ptr(), _LOGITS[logits.dtype], T, V, stride[0] if T > 1 else V,
                uniform.data_ptr(), _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p),
                token.data_ptr(), logprob.data_ptr(), self._ws.on(st), self._ws.bytes, st)
        _check(status, "pctree_sample")
        return token, logprob


def sample(logits, uniform, *, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
    """One call of :class:`Sampler`."""
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2 or not logits.is_cuda:
        raise ValueError("logits must be a [T][V] device tensor")
    with _Here(logits.get_device(), stream):
        return Sampler(*logits.shape, device=logits.device)(
            logits, uniform, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)


def _rows_2d(name, t, dtype, T, H, idx):
    """Row stride of a [T][H] tensor whose rows may lie apart."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype:
        raise TypeError(f"{name} must be a {dtype} tensor")
    if t.shape != (T, H) or t.get_device() != idx or idx < 0:
        raise ValueError(f"{name} must be a [{T}][{H}] tensor on the device of the other tensors, "
                         f"got {tuple(t.shape)}")
    st = t.stride()
    if (H > 1 and st[1] != 1) or (T > 1 and st[0] < H):
        raise ValueError(f"a row of {name} must be contiguous, rows must not overlap")
    return st[0] if T > 1 else H


def _list_size(name, t):
    return _size(name, t.numel()) if isinstance(t, torch.Tensor) else 0


def rms_norm(x, weight=None, residual=None, *, eps=1e-6, group=None, out=None, scale=None,
             stream=None):
    """``v = x + residual`` (``residual`` becomes ``v``), then ``v / sqrt(mean(v^2) + eps) *
    weight`` of every row of ``x [T][H]`` (bfloat16 or float16; rows may lie apart).

    Returns it in x's type (in ``out`` if given, which may be ``x``) or, with ``group``, as
    ``(out, scale)``: float8_e4m3fn, and float32 scales ``[T][ceil(H / group)]`` that a group's
    values are to be multiplied by (``group`` 32, 64, 128 or 256 elements, 0: a whole row)."""
    if not isinstance(x, torch.Tensor) or x.dtype not in _HALVES:
        raise TypeError("x must be a bfloat16 or float16 tensor")
    if x.dim() != 2 or not x.is_cuda:
        raise ValueError("x must be a [T][H] device tensor")
    T, H = x.shape
    idx, dt = x.get_device(), x.dtype
    xs = _rows_2d("x", x, dt, T, H, idx)
    if weight is not None:
        _device_tensor("weight", weight, dt, (H,), idx)
    rs = 0 if residual is None else _rows_2d("residual", residual, dt, T, H, idx)
    held = group is not None
    if held:
        group = _size("group", group)
        if group < 0:
            raise ValueError(f"group must be 32, 64, 128, 256 or 0, got {group}")
        n = -(-H // group) if group else 1
    elif scale is not None:
        raise ValueError("scale goes with group")
    with _Here(idx, stream) as st:
        if out is None:
            out, os_ = x.new_empty((T, H), dtype=_HELD if held else dt), H
        else:
            os_ = _rows_2d("out", out, _HELD if held else dt, T, H, idx)
        if held:
            if scale is None:
                scale = x.new_empty((T, n), dtype=torch.float32)
            else:
                _device_tensor("scale", scale, torch.float32, (T, n), idx)
        a = _Norm(x.data_ptr(), _ptr(weight), _ptr(residual), out.data_ptr(), _ptr(scale), xs, rs,
                  os_, T, H, group if held else 0, _HALVES[dt], eps)
        status = lib().pctree_rms_norm(ctypes.byref(a), st)
    _check(status, "pctree_rms_norm")
    return (out, scale) if held else out


def adjust_logits(logits, row_start, row_count, *, max_rows=None, history=None, history_start=None,
                  history_count=None, prompt_count=None, repetition=None, frequency=None,
                  presence=None, bias_token=None, bias_value=None, bias_start=None,
                  bias_count=None, token=None, mask=None, allowed=None, allowed_row=None,
                  stream=None):
    """Penalties for repeated tokens, biases and a grammar's mask, on ``logits [T][V]`` (float32,
    bfloat16 or float16; rows may lie apart) in place, before :class:`Sampler`.

    Request ``r`` has rows ``row_start[r] + i``, ``i < row_count[r]`` (``max_rows``: the most any
    has).  Its tokens so far are ``history_count[r]`` of ``history`` from ``history_start[r]``, the
    first ``prompt_count[r]`` of them its prompt; with ``token [R][N]`` and ``mask``
    (:func:`build_mask`) row ``i`` is a tree's node and counts its ancestors and itself too.
    ``repetition`` (divides or multiplies the logits of tokens that were there, the prompt's
    too), ``frequency`` (times the count since the prompt) and ``presence`` are ``[R]`` float32.
    ``bias_value`` is added to the logits of ``bias_token``, ``bias_count[r]`` entries from
    ``bias_start[r]`` (of a token's entries the last).  ``allowed [M][ceil(V / 32)]`` (int32
    words): tokens whose bit is not set become -inf; row ``t`` takes mask ``allowed_row[t]`` (no
    mask where that is none's index) or ``t``.  See include/pctree.h.  Returns ``logits``."""
    if not isinstance(logits, torch.Tensor) or logits.dtype not in _LOGITS:
        raise TypeError("logits must be a float32, bfloat16 or float16 tensor")
    if logits.dim() != 2 or not logits.is_cuda:
        raise ValueError("logits must be a [T][V] device tensor")
    T, V = logits.shape
    idx = logits.get_device()
    stride = _rows_2d("logits", logits, logits.dtype, T, V, idx)
    i32, f32 = torch.int32, torch.float32
    if not isinstance(row_start, torch.Tensor) or row_start.dim() != 1:
        raise ValueError("row_start must be an [R] tensor")
    R = row_start.shape[0]
    one = (R,)
    _device_tensor("row_start", row_start, i32, one, idx)
    _device_tensor("row_count", row_count, i32, one, idx)
    most = T if max_rows is None else _size("max_rows", max_rows)

    # lists over all requests (empty where no request has any), and each request's part
    total = biases = 0
    if history is not None:
        total = _list_size("history", history)
        _device_tensor("history", history, i32, (total,), idx)
        if not total:
            history = history_start = history_count = prompt_count = None
    if bias_token is not None:
        biases = _list_size("bias_token", bias_token)
        _device_tensor("bias_token", bias_token, i32, (biases,), idx)
        if bias_value is not None:
            _device_tensor("bias_value", bias_value, f32, (biases,), idx)
        if not biases:
            bias_token = bias_value = bias_start = bias_count = None
    for name, t in (("history_start", history_start), ("history_count", history_count),
                    ("prompt_count", prompt_count), ("bias_start", bias_start),
                    ("bias_count", bias_count)):
        if t is not None:
            _device_tensor(name, t, i32, one, idx)
    for name, t in (("repetition", repetition), ("frequency", frequency), ("presence", presence)):
        if t is not None:
            _device_tensor(name, t, f32, one, idx)
    budget = masks = 0
    if token is not None:
        budget = token.shape[1] if isinstance(token, torch.Tensor) and token.dim() == 2 else 0
        _device_tensor("token", token, i32, (R, budget), idx)
    if mask is not None:
        if mask.dtype != torch.int32 and mask.dtype != torch.uint32:
            raise TypeError("mask must be the [R][N][(N+31)/32] words of build_mask")
        _device_tensor("mask", mask, mask.dtype, (R, budget, (budget + 31) // 32), idx)
    if allowed is not None:
        if not isinstance(allowed, torch.Tensor) or \
                (allowed.dtype != torch.int32 and allowed.dtype != torch.uint32):
            raise TypeError("allowed must be an int32 or uint32 tensor of words")
        masks = _size("masks", allowed.shape[0] if allowed.dim() == 2 else 0)
        _device_tensor("allowed", allowed, allowed.dtype, (masks, (V + 31) // 32), idx)
    if allowed_row is not None:
        _device_tensor("allowed_row", allowed_row, i32, (T,), idx)
    if allowed is not None and not masks:
        allowed = allowed_row = None
    given = (row_start, row_count, history, history_start, history_count, prompt_count, repetition,
             frequency, presence, bias_token, bias_value, bias_start, bias_count, token, mask,
             allowed, allowed_row)
    with _Here(idx, stream) as st:
        a = _Adjust(logits.data_ptr(), stride, *map(_ptr, given), T, V, R, most, total, biases,
                    budget, masks, _LOGITS[logits.dtype])
        status = lib().pctree_adjust_logits(ctypes.byref(a), st)
    _check(status, "pctree_adjust_logits")
    return logits


def device_inputs(inp: dict, device="cuda") -> dict:
    """Upload one round's host inputs (the dict returned by ``synth.make_inputs``).

    The head matrix is stored transposed, ``Wt [V][r]`` (each token's rank
    vector contiguous, the same layout as ``E``); this packing is done once,
    when the drafter's weights are loaded, not per round.
    """
    import numpy as np

    dt = torch.bfloat16 if inp["workload"].dtype == "bf16" else torch.float32

    def up(a, dtype):
        return torch.from_numpy(np.ascontiguousarray(a)).to(device=device).to(dtype)

    return {
        "L": up(inp["L"], dt),
        "E": up(inp["E"], dt),
        "Wt": up(inp["W"].T, dt),
        "h": up(inp["h"], torch.float32),
        "root": up(inp["root"], torch.int32),
        "prefix_len": up(inp["prefix_len"], torch.int32),
    }
