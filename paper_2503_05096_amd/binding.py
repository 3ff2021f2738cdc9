"""Thin Python binding of libadaspec.so (see include/adaspec.h).

Argument marshalling only: every step of the verification path runs inside the
library's HIP kernels.  PyTorch supplies device memory and streams.  There is
no CPU fallback: if the library has not been built, importing it fails.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libadaspec.so")

F32, F16, BF16 = 0, 1, 2
PATH_AUTO, PATH_VECTOR, PATH_FAST = 0, 1, 2
PLAN_BUILD_AND_RUN, PLAN_BUILD_ONLY, PLAN_REUSE = 0, 1, 2
_PLAN = {"run": PLAN_BUILD_AND_RUN, "build": PLAN_BUILD_ONLY, "reuse": PLAN_REUSE}
PATH_STREAM, PATH_TWO_PASS = 3, 4
_PATHS = {"auto": PATH_AUTO, "vector": PATH_VECTOR, "fast": PATH_FAST, "stream": PATH_STREAM,
          "two_pass": PATH_TWO_PASS}

EXPORTS = (
    "adaspec_verify_attn_workspace_bytes", "adaspec_verify_attn",
    "adaspec_accept_workspace_bytes", "adaspec_accept", "adaspec_accept_noalloc", "adaspec_accept_resolved_path",
    "adaspec_verify_attn_tree", "adaspec_accept_tree", "adaspec_kv_compact_path", "adaspec_check_tree_parents", "adaspec_check_accept_inputs",
    "adaspec_check_ragged_inputs", "adaspec_kv_append", "adaspec_commit",
    "adaspec_verify_attn_window_workspace_bytes", "adaspec_verify_attn_window", "adaspec_check_window_inputs",
    "adaspec_kv_remap_workspace_bytes", "adaspec_kv_remap", "adaspec_kv_compact_pages_workspace_bytes", "adaspec_kv_compact_pages",
    "adaspec_kv_copy_pages",
    "adaspec_rope", "adaspec_kv_append_rope", "adaspec_verify_attn_scaled_workspace_bytes", "adaspec_verify_attn_scaled",
    "adaspec_kv_copy_pages_scaled", "adaspec_kv_compact_path_scaled",
    "adaspec_draft_sample_workspace_bytes", "adaspec_draft_sample",
    "adaspec_status_string", "adaspec_version",
)


class AttnDims(C.Structure):
    _fields_ = [("batch", C.c_int32), ("total_q", C.c_int32), ("max_spec_len", C.c_int32),
                ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_size", C.c_int32), ("num_pages", C.c_int32), ("max_pages_per_req", C.c_int32),
                ("dtype", C.c_int32), ("out_dtype", C.c_int32), ("path", C.c_int32),
                ("scale", C.c_float), ("plan_mode", C.c_int32),
                ("timing_start", C.c_void_p), ("timing_stop", C.c_void_p)]


class AcceptDims(C.Structure):
    _fields_ = [("batch", C.c_int32), ("total_q", C.c_int32), ("total_draft", C.c_int32),
                ("max_spec_len", C.c_int32), ("vocab", C.c_int32), ("logits_dtype", C.c_int32),
                ("probs_dtype", C.c_int32), ("out_stride", C.c_int32),
                ("logits_row_stride", C.c_int64), ("probs_row_stride", C.c_int64),
                ("path", C.c_int32), ("reserved", C.c_int32),
                ("timing_start", C.c_void_p), ("timing_stop", C.c_void_p)]


class CommitDims(C.Structure):
    _fields_ = [("batch", C.c_int32), ("max_spec_len", C.c_int32), ("out_stride", C.c_int32),
                ("seq_stride", C.c_int32)]


class DraftDims(C.Structure):
    _fields_ = [("rows", C.c_int32), ("vocab", C.c_int32), ("logits_dtype", C.c_int32),
                ("probs_dtype", C.c_int32), ("logits_row_stride", C.c_int64), ("probs_row_stride", C.c_int64),
                ("path", C.c_int32), ("reserved", C.c_int32),
                ("timing_start", C.c_void_p), ("timing_stop", C.c_void_p)]


class PagesDims(C.Structure):
    _fields_ = [("batch", C.c_int32), ("old_batch", C.c_int32), ("max_pages_per_req", C.c_int32), ("num_pages", C.c_int32),
                ("page_size", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32), ("max_moves", C.c_int32)]


class CopyDims(C.Structure):
    _fields_ = [("layers", C.c_int32), ("num_pages", C.c_int32), ("n_kv_heads", C.c_int32), ("page_size", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class RopeDims(C.Structure):
    _fields_ = [("batch", C.c_int32), ("total_q", C.c_int32), ("max_spec_len", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("page_size", C.c_int32), ("num_pages", C.c_int32),
                ("max_pages_per_req", C.c_int32), ("dtype", C.c_int32), ("rot_dim", C.c_int32), ("interleaved", C.c_int32),
                ("attn_factor", C.c_float), ("reserved", C.c_int32),
                ("q_row_stride", C.c_int64), ("k_row_stride", C.c_int64), ("v_row_stride", C.c_int64), ("q_out_row_stride", C.c_int64)]


class AdaspecError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None
_fast = None        # the _fastcall module once the library is loaded

# entry points the native call path uses, in the order it expects their addresses
_FAST_ENTRIES = ("adaspec_verify_attn_workspace_bytes", "adaspec_verify_attn", "adaspec_verify_attn_tree",
                 "adaspec_accept_workspace_bytes", "adaspec_accept", "adaspec_accept_tree", "adaspec_kv_append",
                 "adaspec_kv_compact_path", "adaspec_commit", "adaspec_draft_sample_workspace_bytes",
                 "adaspec_draft_sample",
                 "adaspec_verify_attn_window_workspace_bytes", "adaspec_verify_attn_window", "adaspec_kv_remap_workspace_bytes",
                 "adaspec_kv_remap", "adaspec_kv_compact_pages_workspace_bytes", "adaspec_kv_compact_pages", "adaspec_kv_copy_pages",
                 "adaspec_rope", "adaspec_kv_append_rope", "adaspec_verify_attn_scaled_workspace_bytes", "adaspec_verify_attn_scaled")


def _native():
    """The native call path (csrc_python/fastcall.cpp): its functions make an ordinary call in full, or return
    NotImplemented without having done anything, and the wrapper goes on in Python.  Where the module is missing or was
    built for another torch, every call goes on in Python: the same kernels, some microseconds later."""
    global _fast
    if _fast is None:
        L = lib()
        import torch
        try:
            from . import _fastcall
            if _fastcall.torch_version != torch.__version__:
                raise ImportError(f"it was built for torch {_fastcall.torch_version}")
            _fastcall.setup(tuple(C.cast(getattr(L, n), C.c_void_p).value for n in _FAST_ENTRIES), _workspace,
                            torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice, AdaspecError)
            _fast = _fastcall
        except (ImportError, AttributeError) as e:
            import warnings
            warnings.warn(f"no native call path, calls go through Python ({e}); build it together with the library: "
                          "python paper_2503_05096_amd/build.py", RuntimeWarning, stacklevel=3)
            _fast = _PythonOnly()
    return _fast


class _PythonOnly:
    """Stands in for the native call path where there is none."""
    def _decline(*args):
        return NotImplemented
    verify_attn = accept = accept_tree = kv_append = kv_compact_path = commit = draft_sample = _decline
    verify_attn_window = kv_remap = kv_compact_pages = kv_copy_pages = _decline
    rope = kv_append_rope = verify_attn_scaled = _decline


def lib() -> C.CDLL:
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; "
                "g.build()' or python paper_2503_05096_amd/build.py). There is no fallback path.")
        _lib = _open(LIB_PATH)
    return _lib


def _open(path: str) -> C.CDLL:
    """The library at `path`, with the C ABI's signatures."""
    # The process must hold ONE HIP runtime.  PyTorch ships its own copy and loads it by path;
    # the loader shares it with this library only if it is already mapped when the library is
    # opened (same SONAME).  Opened the other way round, the library would bind to the system
    # copy and launch kernels through a runtime that knows nothing of torch's streams and memory.
    import torch  # noqa: F401
    L = C.CDLL(path)
    vp = C.c_void_p
    L.adaspec_verify_attn_workspace_bytes.restype = C.c_size_t
    L.adaspec_verify_attn_workspace_bytes.argtypes = [C.POINTER(AttnDims)]
    L.adaspec_verify_attn.restype = C.c_int
    L.adaspec_verify_attn.argtypes = [vp] * 7 + [C.POINTER(AttnDims), vp, C.c_size_t, vp]
    L.adaspec_verify_attn_window_workspace_bytes.restype = C.c_size_t
    L.adaspec_verify_attn_window_workspace_bytes.argtypes = [C.POINTER(AttnDims), C.c_int32, C.c_int32]
    L.adaspec_verify_attn_window.restype = C.c_int
    L.adaspec_verify_attn_window.argtypes = [vp] * 7 + [C.POINTER(AttnDims), C.c_int32, C.c_int32, vp, C.c_size_t, vp]
    L.adaspec_check_window_inputs.restype = C.c_int
    L.adaspec_check_window_inputs.argtypes = [vp, vp, vp, C.POINTER(AttnDims), C.c_int32, C.c_int32, vp, vp]
    L.adaspec_accept_workspace_bytes.restype = C.c_size_t
    L.adaspec_accept_workspace_bytes.argtypes = [C.POINTER(AcceptDims)]
    L.adaspec_accept.restype = C.c_int
    L.adaspec_accept.argtypes = [vp] * 8 + [C.POINTER(AcceptDims), vp, C.c_size_t, vp]
    L.adaspec_accept_noalloc.restype = C.c_int
    L.adaspec_accept_noalloc.argtypes = [vp] * 8 + [C.POINTER(AcceptDims), vp]
    L.adaspec_accept_resolved_path.restype = C.c_int
    L.adaspec_accept_resolved_path.argtypes = [vp, vp, C.POINTER(AcceptDims)]
    L.adaspec_verify_attn_tree.restype = C.c_int
    L.adaspec_verify_attn_tree.argtypes = [vp] * 8 + [C.POINTER(AttnDims), vp, C.c_size_t, vp]
    L.adaspec_accept_tree.restype = C.c_int
    L.adaspec_accept_tree.argtypes = [vp] * 10 + [C.POINTER(AcceptDims), vp, C.c_size_t, vp]
    L.adaspec_kv_compact_path.restype = C.c_int
    L.adaspec_kv_compact_path.argtypes = [vp] * 7 + [C.POINTER(AttnDims), C.c_int32, vp]
    L.adaspec_check_accept_inputs.restype = C.c_int
    L.adaspec_check_accept_inputs.argtypes = [vp, vp, vp, C.POINTER(AcceptDims), vp, vp]
    L.adaspec_check_tree_parents.restype = C.c_int
    L.adaspec_check_tree_parents.argtypes = [vp, vp, C.c_int32, C.c_int32, C.c_int32, vp, vp]
    L.adaspec_check_ragged_inputs.restype = C.c_int
    L.adaspec_check_ragged_inputs.argtypes = [vp, vp, vp, C.POINTER(AttnDims), vp, vp]
    L.adaspec_kv_append.restype = C.c_int
    L.adaspec_kv_append.argtypes = [vp] * 7 + [C.POINTER(AttnDims), vp]
    L.adaspec_commit.restype = C.c_int
    L.adaspec_commit.argtypes = [vp] * 10 + [C.POINTER(CommitDims), vp]
    L.adaspec_draft_sample.restype = C.c_int
    L.adaspec_draft_sample.argtypes = [vp] * 7 + [C.POINTER(DraftDims), vp, C.c_size_t, vp]
    L.adaspec_draft_sample_workspace_bytes.restype = C.c_size_t
    L.adaspec_draft_sample_workspace_bytes.argtypes = [C.POINTER(DraftDims)]
    L.adaspec_kv_remap_workspace_bytes.restype = C.c_size_t
    L.adaspec_kv_remap_workspace_bytes.argtypes = [C.POINTER(PagesDims)]
    L.adaspec_kv_remap.restype = C.c_int
    L.adaspec_kv_remap.argtypes = [vp] * 10 + [C.POINTER(PagesDims), vp, C.c_size_t, vp]
    L.adaspec_kv_compact_pages_workspace_bytes.restype = C.c_size_t
    L.adaspec_kv_compact_pages_workspace_bytes.argtypes = [C.POINTER(PagesDims)]
    L.adaspec_kv_compact_pages.restype = C.c_int
    L.adaspec_kv_compact_pages.argtypes = [vp] * 8 + [C.POINTER(PagesDims), vp, C.c_size_t, vp]
    L.adaspec_kv_copy_pages.restype = C.c_int
    L.adaspec_kv_copy_pages.argtypes = [vp] * 4 + [C.c_int32, C.POINTER(CopyDims), vp]
    L.adaspec_rope.restype = C.c_int
    L.adaspec_rope.argtypes = [vp] * 6 + [C.POINTER(RopeDims), vp]
    L.adaspec_kv_append_rope.restype = C.c_int
    L.adaspec_kv_append_rope.argtypes = [vp] * 13 + [C.POINTER(RopeDims), vp]
    L.adaspec_verify_attn_scaled_workspace_bytes.restype = C.c_size_t
    L.adaspec_verify_attn_scaled_workspace_bytes.argtypes = [C.POINTER(AttnDims)]
    L.adaspec_verify_attn_scaled.restype = C.c_int
    L.adaspec_verify_attn_scaled.argtypes = [vp] * 10 + [C.POINTER(AttnDims), vp, C.c_size_t, vp]
    L.adaspec_kv_copy_pages_scaled.restype = C.c_int
    L.adaspec_kv_copy_pages_scaled.argtypes = [vp] * 6 + [C.c_int32, C.POINTER(CopyDims), vp]
    L.adaspec_kv_compact_path_scaled.restype = C.c_int
    L.adaspec_kv_compact_path_scaled.argtypes = [vp] * 9 + [C.POINTER(AttnDims), C.c_int32, vp]
    L.adaspec_status_string.restype = C.c_char_p
    L.adaspec_status_string.argtypes = [C.c_int]
    L.adaspec_version.restype = C.c_int
    return L


def hip_runtime() -> C.CDLL:
    """The HIP runtime this process already uses (the copy torch loaded), for callers that need
    raw HIP calls such as hipEventCreate: opening "libamdhip64.so" by name could map a second copy."""
    lib()
    with open("/proc/self/maps") as f:
        paths = {line.split()[-1] for line in f if "libamdhip64" in line}
    if len(paths) != 1:
        raise RuntimeError(f"expected exactly one HIP runtime in the process, found {sorted(paths)}")
    return C.CDLL(paths.pop())


def status_string(status: int) -> str:
    return lib().adaspec_status_string(int(status)).decode()


def version() -> int:
    return int(lib().adaspec_version())


# --------------------------------------------------------------------------
# torch-facing wrappers
# --------------------------------------------------------------------------
def _int32(n) -> int:
    """n, cut to 32 bits: a window of more tokens than there are"""
    return max(min(int(n), 2 ** 31 - 1), -2 ** 31)


def _dtype_code(t) -> int:
    import torch
    return {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}[t.dtype]


def _torch_dtype(code: int):
    import torch
    return {F32: torch.float32, F16: torch.float16, BF16: torch.bfloat16}[code]


def _stream_ptr(stream) -> int:
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return int(s.cuda_stream)


# Default workspaces of attention, acceptance and draft sampling: one per (device, call family), grown on demand.
# The three never share one (a planned attention pass keeps its metadata in its workspace across calls).
# A buffer that is outgrown stays referenced until the process ends: a kernel on a caller-supplied,
# non-current stream may still be using it, and torch's allocator would hand a freed block to the next
# tensor at once.  Callers that issue calls on several streams must pass their own `workspace` per
# stream: calls that share a workspace have to be ordered on one stream.
_ws_cache = {}
_ws_retired = []


def _on_device(t, device, what: str) -> None:
    """A caller's buffer that kernels write to: an address of another device, or of the host, would be written to all the same."""
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, the call's tensors are on {device}")


def _workspace(nbytes: int, device, workspace, family: str):
    import torch
    if workspace is not None:
        _on_device(workspace, device, "workspace=")
        return workspace
    key = (str(device), family)
    ws = _ws_cache.get(key)
    if ws is None or ws.numel() < nbytes:
        if ws is not None:
            _ws_retired.append(ws)
        ws = torch.empty(max(nbytes, 1 << 20), dtype=torch.uint8, device=device)
        _ws_cache[key] = ws
    return ws


def _scratch(nbytes: int, device, workspace, stream):
    """The caller's workspace, or memory of this call alone: what its kernels leave there for each other is safe from calls on other
    streams, from other threads and from graphs that are replayed meanwhile.  It is allocated on the call's stream, to whose memory it
    goes back when the call has been made, behind its kernels."""
    import torch
    if workspace is not None:
        _on_device(workspace, device, "workspace=")
        return workspace
    if stream is not None and not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream.cuda_stream), device=device)
    with torch.cuda.stream(stream):                     # (None: the current one)
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def _with_timing(dims, timing):
    """timing = (start, stop): raw hipEvent_t handles (ints or c_void_p) the library records around the call's
    main kernel(s) on the call's stream; None = no events."""
    if timing is not None:
        start, stop = timing
        dims.timing_start = start.value if isinstance(start, C.c_void_p) else start
        dims.timing_stop = stop.value if isinstance(stop, C.c_void_p) else stop
    return dims


def attn_dims(q, k_pages, block_table, *, max_spec_len: int, scale: float = 0.0,
              out_dtype: Optional[int] = None, path: str = "auto", plan: str = "run") -> AttnDims:
    dt = _dtype_code(q)
    TQ, Hq, d = q.shape
    num_pages, Hkv, P, _ = k_pages.shape
    B, max_pages = block_table.shape
    return AttnDims(B, TQ, int(max_spec_len), Hq, Hkv, d, P, num_pages, max_pages, dt,
                    dt if out_dtype is None else int(out_dtype), _PATHS[path], float(scale), _PLAN[plan])


def verify_attn(q, k_pages, v_pages, block_table, ctx_lens, spec_lens, out=None, *,
                max_spec_len: int, scale: float = 0.0, out_dtype: Optional[int] = None,
                path: str = "auto", plan: str = "run", workspace=None, stream=None, parents=None, timing=None,
                window: Optional[int] = None, sinks: int = 0, k_scales=None, v_scales=None):
    """adaspec_verify_attn on device tensors; returns `out` [TQ][Hq][d].

    plan: "run" (build the ragged metadata, then run), "build" (metadata only; returns None) or
    "reuse" (run with the metadata a previous call left in the same workspace).  "build" and "reuse"
    require `workspace`: a tensor of at least adaspec_verify_attn_workspace_bytes that the caller owns
    and that no other call touches between the build and the last reuse.
    parents [TQ] int32 (a draft tree): adaspec_verify_attn_tree instead.
    window, sinks: adaspec_verify_attn_window instead: a row sees the last `window` tokens up to its own and the request's
    first `sinks`; block_table entries of pages that no row sees are never read.  Not with parents.  Such a call has no plan of
    its own and overwrites its workspace: not the one that holds a plan for calls without a window.
    workspace: calls without a window share a default one per device, and have to be ordered on one stream; on several streams each
    needs its own.  Windowed calls without workspace= may overlap: each that keeps something there has its own.
    k_scales, v_scales [num_pages][Hkv] float32: adaspec_verify_attn_scaled instead, over k_pages and v_pages of
    torch.float8_e4m3fn.  Not with a window.  Calls without workspace= may overlap: each has its own."""
    if k_scales is not None or v_scales is not None:
        if window is not None or sinks != 0:
            raise ValueError("verify_attn(k_scales=, v_scales=) takes no window")
        return _verify_attn_scaled(q, k_pages, v_pages, k_scales, v_scales, block_table, ctx_lens, spec_lens, out, max_spec_len, scale,
                                   out_dtype, path, plan, workspace, stream, parents, timing)
    if window is not None or sinks != 0:
        if window is None:
            raise ValueError("verify_attn(sinks=...) needs a window: without one every token is visible")
        if parents is not None:
            raise ValueError("verify_attn(window=...) takes chains of drafts, not trees (parents=)")
        window, sinks = _int32(window), _int32(sinks)
        if path == "auto" and timing is None:
            r = (_fast or _native()).verify_attn_window(q, k_pages, v_pages, block_table, ctx_lens, spec_lens, out, max_spec_len,
                                                        scale, out_dtype, plan, workspace, stream, window, sinks)
            if r is not NotImplemented:
                return r
    elif path == "auto" and timing is None:
        r = (_fast or _native()).verify_attn(q, k_pages, v_pages, block_table, ctx_lens, spec_lens, out, max_spec_len,
                                             scale, out_dtype, plan, workspace, stream, parents)
        if r is not NotImplemented:
            return r
    import torch
    dims = _with_timing(attn_dims(q, k_pages, block_table, max_spec_len=max_spec_len, scale=scale,
                                  out_dtype=out_dtype, path=path, plan=plan), timing)
    for t in (q, k_pages, v_pages, block_table, ctx_lens, spec_lens):
        assert t.is_cuda and t.is_contiguous()
    assert block_table.dtype == torch.int32 and ctx_lens.dtype == torch.int32 and spec_lens.dtype == torch.int32
    assert v_pages.shape == k_pages.shape and v_pages.dtype == k_pages.dtype == q.dtype
    assert k_pages.shape[3] == q.shape[2]
    if out is not None:
        _on_device(out, q.device, "out")
    elif plan != "build":
        out = torch.empty(q.shape, dtype=_torch_dtype(dims.out_dtype), device=q.device)
    L = lib()
    if window is not None:
        return _verify_attn_window(q, k_pages, v_pages, block_table, ctx_lens, spec_lens, out, dims, window, sinks, plan,
                                   workspace, stream)
    need = L.adaspec_verify_attn_workspace_bytes(C.byref(dims))
    if need == 0 and dims.batch > 0:
        raise AdaspecError(L.adaspec_verify_attn(None, None, None, None, None, None, None, C.byref(dims),
                                                 None, 0, None) or -2, "adaspec_verify_attn (dims)")
    if plan != "run" and workspace is None:
        # the metadata of a planned pass lives in the workspace between the calls: it has to be the
        # caller's own buffer, one that nothing else writes to meanwhile
        raise ValueError("verify_attn(plan='build' / 'reuse') needs an explicit workspace= tensor that the "
                         "caller keeps for the whole pass")
    ws = _workspace(need, q.device, workspace, "attn")
    if parents is not None:
        assert parents.is_cuda and parents.is_contiguous() and parents.dtype == torch.int32
        assert parents.shape == (q.shape[0],)
        rc = L.adaspec_verify_attn_tree(q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                        block_table.data_ptr(), ctx_lens.data_ptr(), spec_lens.data_ptr(),
                                        parents.data_ptr(), None if out is None else out.data_ptr(),
                                        C.byref(dims), ws.data_ptr(), ws.numel(), _stream_ptr(stream))
        if rc != 0:
            raise AdaspecError(rc, "adaspec_verify_attn_tree")
        return out
    rc = L.adaspec_verify_attn(q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                               block_table.data_ptr(), ctx_lens.data_ptr(), spec_lens.data_ptr(),
                               None if out is None else out.data_ptr(), C.byref(dims), ws.data_ptr(), ws.numel(),
                               _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_verify_attn")
    return out


def _verify_attn_window(q, k_pages, v_pages, block_table, ctx_lens, spec_lens, out, dims, window, sinks, plan, workspace, stream):
    """the windowed call of verify_attn, whose checks have been made"""
    L = lib()
    _on_current_device(q)
    assert all(t.device == q.device for t in (k_pages, v_pages, block_table, ctx_lens, spec_lens))
    assert ctx_lens.shape == spec_lens.shape == (dims.batch,)
    assert out is None or (out.is_contiguous() and out.shape == q.shape and _dtype_code(out) == dims.out_dtype)
    need = L.adaspec_verify_attn_window_workspace_bytes(C.byref(dims), window, sinks)
    if need == 0 and dims.batch > 0:
        raise AdaspecError(L.adaspec_verify_attn_window(None, None, None, None, None, None, None, C.byref(dims), window, sinks, None,
                                                        0, None) or -2, "adaspec_verify_attn_window (dims)")
    if plan != "run" and workspace is None:
        raise ValueError("verify_attn(plan='build' / 'reuse') needs an explicit workspace= tensor that the "
                         "caller keeps for the whole pass")
    # (256 bytes: the call is not cut into parts, and writes none of them)
    ws = _scratch(need, q.device, workspace, stream) if need > 256 else _workspace(need, q.device, workspace, "attn")
    rc = L.adaspec_verify_attn_window(q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), block_table.data_ptr(),
                                      ctx_lens.data_ptr(), spec_lens.data_ptr(), None if out is None else out.data_ptr(),
                                      C.byref(dims), window, sinks, ws.data_ptr(), ws.numel(), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_verify_attn_window")
    return out


def _verify_attn_scaled(q, k_pages, v_pages, k_scales, v_scales, block_table, ctx_lens, spec_lens, out, max_spec_len, scale, out_dtype,
                        path, plan, workspace, stream, parents, timing):
    """verify_attn over a cache of 8 bits"""
    if path == "auto" and timing is None:
        r = (_fast or _native()).verify_attn_scaled(q, k_pages, v_pages, k_scales, v_scales, block_table, ctx_lens, spec_lens, out,
                                                    max_spec_len, scale, out_dtype, plan, workspace, stream, parents)
        if r is not NotImplemented:
            return r
    import torch
    for t in (q, block_table, ctx_lens, spec_lens):
        assert t.is_cuda and t.is_contiguous()
    assert q.dim() == 3 and k_pages.dim() == 4 and block_table.dim() == 2
    _scaled_cache(k_pages, v_pages, k_scales, v_scales)
    _dense_ints(block_table, ctx_lens, spec_lens)
    _on_current_device(q)
    assert k_pages.device == block_table.device == q.device
    assert ctx_lens.shape == spec_lens.shape == block_table.shape[:1] and k_pages.shape[3] == q.shape[2]
    dims = _with_timing(attn_dims(q, k_pages, block_table, max_spec_len=max_spec_len, scale=scale, out_dtype=out_dtype, path=path,
                                  plan=plan), timing)
    if parents is not None:
        _dense_ints(block_table, parents)
        assert parents.shape == (q.shape[0],)
    if plan != "run" and workspace is None:
        raise ValueError("verify_attn(plan='build' / 'reuse') needs an explicit workspace= tensor that the "
                         "caller keeps for the whole pass")
    if out is not None:
        _on_device(out, q.device, "out")
        assert out.is_contiguous() and out.shape == q.shape and _dtype_code(out) == dims.out_dtype
    elif plan != "build":
        out = torch.empty(q.shape, dtype=_torch_dtype(dims.out_dtype), device=q.device)
    L = lib()
    need = L.adaspec_verify_attn_scaled_workspace_bytes(C.byref(dims))
    ptr = lambda t: None if t is None else t.data_ptr()
    args = [ptr(t) for t in (q, k_pages, v_pages, k_scales, v_scales, block_table, ctx_lens, spec_lens, parents, out)]
    if need == 0 and dims.batch > 0:
        raise AdaspecError(L.adaspec_verify_attn_scaled(*args, C.byref(dims), None, 0, None) or -2, "adaspec_verify_attn_scaled (dims)")
    ws = _scratch(need, q.device, workspace, stream)
    rc = L.adaspec_verify_attn_scaled(*args, C.byref(dims), ws.data_ptr(), ws.numel(), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_verify_attn_scaled")
    return out


def _scaled_cache(k_pages, v_pages, k_scales, v_scales) -> None:
    """a cache of 8 bits: pages [..., num_pages][Hkv][P][d] of e4m3, scales [..., num_pages][Hkv]"""
    import torch
    if k_scales is None or v_scales is None:
        raise ValueError("k_scales= and v_scales= go together")
    for t in (k_pages, v_pages, k_scales, v_scales):
        assert t.is_cuda and t.is_contiguous() and t.device == k_pages.device
    assert k_pages.dtype == v_pages.dtype == torch.float8_e4m3fn and k_scales.dtype == v_scales.dtype == torch.float32
    assert v_pages.shape == k_pages.shape and v_scales.shape == k_scales.shape == k_pages.shape[:-2]


def accept_dims(target_logits, draft_probs, draft_tokens, spec_lens, max_spec_len, out_stride, path):
    """(dims, draft_probs pointer, draft_tokens pointer) of an acceptance call: marshalling only."""
    import torch
    TQ, V = target_logits.shape
    B = spec_lens.shape[0]
    TD = TQ - B
    out_stride = int(max_spec_len) + 1 if out_stride is None else int(out_stride)
    assert target_logits.is_cuda and spec_lens.is_cuda
    assert target_logits.stride(1) == 1 and spec_lens.dtype == torch.int32
    if TD > 0:
        assert draft_probs.shape == (TD, V) and draft_probs.stride(1) == 1
        assert draft_tokens.dtype == torch.int32 and draft_tokens.shape == (TD,)
        pdt, pstride = _dtype_code(draft_probs), draft_probs.stride(0)
        pp, tp = draft_probs.data_ptr(), draft_tokens.data_ptr()
    else:
        pdt, pstride, pp, tp = _dtype_code(target_logits), V, None, None
    dims = AcceptDims(B, TQ, TD, int(max_spec_len), V, _dtype_code(target_logits), pdt, out_stride,
                      target_logits.stride(0), pstride, _PATHS[path], 0)
    return dims, pp, tp


def accept_resolved_path(target_logits, draft_probs, draft_tokens, spec_lens, *, max_spec_len: int,
                         out_stride: Optional[int] = None, path: str = "auto") -> str:
    """adaspec_accept_resolved_path: the kernel path adaspec_accept takes for these tensors ("stream" and "vector" as the
    answer to "auto": the per-row path of the shape; the header says which of those calls run in row parts)."""
    dims, pp, _ = accept_dims(target_logits, draft_probs, draft_tokens, spec_lens, max_spec_len, out_stride, path)
    rc = lib().adaspec_accept_resolved_path(target_logits.data_ptr(), pp, C.byref(dims))
    if rc < 0:
        raise AdaspecError(rc, "adaspec_accept_resolved_path")
    return {v: k for k, v in _PATHS.items()}[rc]


def accept(target_logits, draft_probs, draft_tokens, uniforms, spec_lens, temperature, *,
           max_spec_len: int, out_tokens=None, out_accept_len=None, out_stride: Optional[int] = None,
           path: str = "auto", workspace=None, stream=None, timing=None) -> Tuple[object, object]:
    """adaspec_accept on device tensors; returns (out_tokens [B][out_stride], out_accept_len [B]).
    workspace: the default one is shared by all calls of a device, which have to be ordered on one stream (accept_tree too)."""
    if path == "auto" and timing is None:
        r = (_fast or _native()).accept(target_logits, draft_probs, draft_tokens, uniforms, spec_lens, temperature,
                                        max_spec_len, out_tokens, out_accept_len, out_stride, workspace, stream)
        if r is not NotImplemented:
            return r
    import torch
    for t in (uniforms, temperature):
        assert t.is_cuda
    assert uniforms.is_contiguous() and uniforms.dtype == torch.float32 and temperature.dtype == torch.float32
    dims, pp, tp = accept_dims(target_logits, draft_probs, draft_tokens, spec_lens, max_spec_len, out_stride, path)
    _with_timing(dims, timing)
    B, out_stride = dims.batch, dims.out_stride
    if out_tokens is None:
        out_tokens = torch.empty((B, out_stride), dtype=torch.int32, device=target_logits.device)
    if out_accept_len is None:
        out_accept_len = torch.empty((B,), dtype=torch.int32, device=target_logits.device)
    L = lib()
    need = L.adaspec_accept_workspace_bytes(C.byref(dims))
    ws = _workspace(max(need, 256), target_logits.device, workspace, "accept")
    rc = L.adaspec_accept(target_logits.data_ptr(), pp, tp, uniforms.data_ptr(), spec_lens.data_ptr(),
                          temperature.data_ptr(), out_tokens.data_ptr(), out_accept_len.data_ptr(),
                          C.byref(dims), ws.data_ptr(), ws.numel(), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_accept")
    return out_tokens, out_accept_len


NOALLOC_SCRATCH_BYTES = 8 << 20


def accept_noalloc(target_logits, draft_probs, draft_tokens, uniforms, spec_lens, temperature, out_tokens,
                   out_accept_len, *, max_spec_len: int, out_stride: Optional[int] = None, path: str = "auto",
                   stream=None) -> None:
    """adaspec_accept_noalloc: acceptance into the caller's output tensors, on the library's built-in
    scratch memory.  Nothing is allocated here either: the outputs are required arguments."""
    import torch
    assert uniforms.is_cuda and uniforms.is_contiguous() and uniforms.dtype == torch.float32
    assert temperature.is_cuda and temperature.dtype == torch.float32
    dims, pp, tp = accept_dims(target_logits, draft_probs, draft_tokens, spec_lens, max_spec_len, out_stride, path)
    assert out_tokens.is_cuda and out_tokens.dtype == torch.int32 and out_tokens.is_contiguous()
    assert tuple(out_tokens.shape) == (dims.batch, dims.out_stride)
    assert out_accept_len.is_cuda and out_accept_len.dtype == torch.int32 and tuple(out_accept_len.shape) == (dims.batch,)
    rc = lib().adaspec_accept_noalloc(target_logits.data_ptr(), pp, tp, uniforms.data_ptr(), spec_lens.data_ptr(),
                                      temperature.data_ptr(), out_tokens.data_ptr(), out_accept_len.data_ptr(),
                                      C.byref(dims), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_accept_noalloc")


def accept_tree(target_logits, draft_probs, draft_tokens, parents, uniforms, spec_lens, temperature, *,
                max_spec_len: int, out_tokens=None, out_accept_len=None, out_path=None,
                out_stride: Optional[int] = None, path: str = "auto", workspace=None, stream=None, timing=None):
    """adaspec_accept_tree; returns (out_tokens [B][out_stride], out_accept_len [B], out_path [B][out_stride]).
    path: "auto", "vector" (portable per-node kernel) or "fast" (node statistics, then the walk of every request)."""
    if path == "auto" and timing is None:
        r = (_fast or _native()).accept_tree(target_logits, draft_probs, draft_tokens, parents, uniforms, spec_lens,
                                             temperature, max_spec_len, out_tokens, out_accept_len, out_path, out_stride,
                                             workspace, stream)
        if r is not NotImplemented:
            return r
    import torch
    for t in (uniforms, temperature, parents):
        assert t.is_cuda and t.is_contiguous()
    assert uniforms.dtype == torch.float32 and temperature.dtype == torch.float32 and parents.dtype == torch.int32
    assert parents.shape == (target_logits.shape[0],)
    dims, pp, tp = accept_dims(target_logits, draft_probs, draft_tokens, spec_lens, max_spec_len, out_stride, path)
    _with_timing(dims, timing)
    B, out_stride = dims.batch, dims.out_stride
    dev = target_logits.device
    if out_tokens is None:
        out_tokens = torch.empty((B, out_stride), dtype=torch.int32, device=dev)
    if out_accept_len is None:
        out_accept_len = torch.empty((B,), dtype=torch.int32, device=dev)
    if out_path is None:
        out_path = torch.empty((B, out_stride), dtype=torch.int32, device=dev)
    L = lib()
    need = L.adaspec_accept_workspace_bytes(C.byref(dims))
    ws = _workspace(max(need, 256), dev, workspace, "accept")
    rc = L.adaspec_accept_tree(target_logits.data_ptr(), pp, tp, parents.data_ptr(), uniforms.data_ptr(),
                               spec_lens.data_ptr(), temperature.data_ptr(), out_tokens.data_ptr(),
                               out_accept_len.data_ptr(), out_path.data_ptr(), C.byref(dims), ws.data_ptr(),
                               ws.numel(), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_accept_tree")
    return out_tokens, out_accept_len, out_path


def kv_compact_path(k_pages, v_pages, block_table, ctx_lens, spec_lens, out_path, out_accept_len, *,
                    max_spec_len: int, stream=None, k_scales=None, v_scales=None) -> None:
    """adaspec_kv_compact_path: moves the accepted nodes' K/V rows to chain positions, in place.
    k_scales, v_scales [num_pages][Hkv]: adaspec_kv_compact_path_scaled instead, for a cache of 8 bits."""
    if k_scales is not None or v_scales is not None:
        return _kv_compact_path_scaled(k_pages, v_pages, k_scales, v_scales, block_table, ctx_lens, spec_lens, out_path, out_accept_len,
                                       max_spec_len, stream)
    if (_fast or _native()).kv_compact_path(k_pages, v_pages, block_table, ctx_lens, spec_lens, out_path, out_accept_len,
                                            max_spec_len, stream) is not NotImplemented:
        return
    import torch
    num_pages, Hkv, P, d = k_pages.shape
    B, max_pages = block_table.shape
    for t in (k_pages, v_pages, block_table, ctx_lens, spec_lens, out_path, out_accept_len):
        assert t.is_cuda and t.is_contiguous()
    for t in (block_table, ctx_lens, spec_lens, out_path, out_accept_len):
        assert t.dtype == torch.int32
    assert v_pages.shape == k_pages.shape and v_pages.dtype == k_pages.dtype
    dt = _dtype_code(k_pages)
    dims = AttnDims(B, B, int(max_spec_len), Hkv, Hkv, d, P, num_pages, max_pages, dt, dt, PATH_AUTO, 0.0)
    rc = lib().adaspec_kv_compact_path(k_pages.data_ptr(), v_pages.data_ptr(), block_table.data_ptr(),
                                       ctx_lens.data_ptr(), spec_lens.data_ptr(), out_path.data_ptr(),
                                       out_accept_len.data_ptr(), C.byref(dims), out_path.shape[1],
                                       _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_kv_compact_path")


def _kv_compact_path_scaled(k_pages, v_pages, k_scales, v_scales, block_table, ctx_lens, spec_lens, out_path, out_accept_len, max_spec_len,
                            stream) -> None:
    assert k_pages.dim() == 4 and block_table.dim() == 2 and out_path.dim() == 2
    _scaled_cache(k_pages, v_pages, k_scales, v_scales)
    _dense_ints(block_table, ctx_lens, spec_lens, out_path, out_accept_len)
    _on_current_device(k_pages)
    assert block_table.device == k_pages.device
    assert ctx_lens.shape == spec_lens.shape == out_accept_len.shape == block_table.shape[:1] == out_path.shape[:1]
    num_pages, Hkv, P, d = k_pages.shape
    B, max_pages = block_table.shape
    dims = AttnDims(B, B, int(max_spec_len), Hkv, Hkv, d, P, num_pages, max_pages, BF16, BF16, PATH_AUTO, 0.0)
    rc = lib().adaspec_kv_compact_path_scaled(k_pages.data_ptr(), v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(),
                                              block_table.data_ptr(), ctx_lens.data_ptr(), spec_lens.data_ptr(), out_path.data_ptr(),
                                              out_accept_len.data_ptr(), C.byref(dims), out_path.shape[1], _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_kv_compact_path_scaled")


def check_accept_inputs(draft_tokens, spec_lens, temperature, *, vocab: int, max_spec_len: int, stream=None) -> int:
    """Runs the device-side check of the acceptance inputs and returns the flag word (synchronises)."""
    import torch
    for t in (draft_tokens, spec_lens):
        assert t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()
    assert temperature.is_cuda and temperature.dtype == torch.float32
    B, TD = spec_lens.shape[0], draft_tokens.shape[0]
    dims = AcceptDims(B, TD + B, TD, int(max_spec_len), int(vocab), BF16, BF16, int(max_spec_len) + 1, int(vocab),
                      int(vocab), PATH_AUTO, 0)
    flags = torch.zeros(1, dtype=torch.int32, device=spec_lens.device)
    rc = lib().adaspec_check_accept_inputs(draft_tokens.data_ptr(), spec_lens.data_ptr(), temperature.data_ptr(),
                                           C.byref(dims), flags.data_ptr(), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_check_accept_inputs")
    return int(flags.item())


def check_tree_parents(parents, spec_lens, *, max_spec_len: int, stream=None) -> int:
    """Runs the device-side check of a parent array and returns the flag word (synchronises)."""
    import torch
    assert parents.is_cuda and parents.dtype == torch.int32 and spec_lens.dtype == torch.int32
    flags = torch.zeros(1, dtype=torch.int32, device=parents.device)
    rc = lib().adaspec_check_tree_parents(parents.data_ptr(), spec_lens.data_ptr(), spec_lens.shape[0],
                                          parents.shape[0], int(max_spec_len), flags.data_ptr(), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_check_tree_parents")
    return int(flags.item())


def check_ragged_inputs(block_table, ctx_lens, spec_lens, dims: AttnDims, stream=None, *, window: Optional[int] = None,
                        sinks: int = 0) -> int:
    """Runs the device-side metadata check and returns the flag word (synchronises).  window, sinks: the check of a windowed
    call, which leaves out the entries that such a call never reads."""
    import torch
    if window is None and sinks != 0:
        raise ValueError("check_ragged_inputs(sinks=...) needs a window: without one every token is visible")
    flags = torch.zeros(1, dtype=torch.int32, device=block_table.device)
    if window is not None:
        rc = lib().adaspec_check_window_inputs(block_table.data_ptr(), ctx_lens.data_ptr(), spec_lens.data_ptr(), C.byref(dims),
                                               _int32(window), _int32(sinks), flags.data_ptr(), _stream_ptr(stream))
        if rc != 0:
            raise AdaspecError(rc, "adaspec_check_window_inputs")
        return int(flags.item())
    rc = lib().adaspec_check_ragged_inputs(block_table.data_ptr(), ctx_lens.data_ptr(),
                                           spec_lens.data_ptr(), C.byref(dims), flags.data_ptr(),
                                           _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_check_ragged_inputs")
    return int(flags.item())


def _rope_dims(rows, heads, kv_heads, d, table_shape, num_pages, max_spec_len, dtype, inv_freq, interleaved, attn_factor) -> RopeDims:
    import torch
    rot = 0
    if inv_freq is not None:
        assert inv_freq.is_cuda and inv_freq.is_contiguous() and inv_freq.dtype == torch.float32 and inv_freq.dim() == 1
        rot = 2 * inv_freq.shape[0]
    if not C.c_float(float(attn_factor)).value > 0:                # (0 in fp32 would mean 1 to the library)
        raise ValueError("attn_factor= is more than 0, in fp32")
    B, max_pages = table_shape
    return RopeDims(B, rows, int(max_spec_len), heads, kv_heads, d, 16, num_pages, max_pages, dtype, rot, int(bool(interleaved)),
                    float(attn_factor), 0, 0, 0, 0, 0)


def _ragged_rows(x, like=None):
    """rows [TQ][heads][d] whose heads lie side by side; the rows may be apart, as slices of a wider array are"""
    assert x.is_cuda and x.dim() == 3 and x.stride(2) == 1 and (x.stride(1) == x.shape[2] or x.shape[1] == 1)
    if like is not None:
        assert x.dtype == like.dtype and x.device == like.device and x.shape[0] == like.shape[0] and x.shape[2] == like.shape[2]
    return x.stride(0) if x.shape[0] > 1 else max(x.stride(0), x.shape[1] * x.shape[2]) // 8 * 8


def rope(x, inv_freq, ctx_lens, spec_lens, *, max_spec_len: int, interleaved: bool = False, attn_factor: float = 1.0, parents=None,
         out=None, stream=None):
    """adaspec_rope: the rows x [TQ][heads][d] turned by the angles of their positions; returns `out` (new and contiguous unless
    given; may be x itself).  inv_freq [rot_dim / 2] float32 (rope_frequencies makes it).  parents [TQ] int32: nodes of draft trees
    stand at the depth they have.  x (and out) may be slices of wider rows, e.g. of a projection's output."""
    r = (_fast or _native()).rope(x, inv_freq, ctx_lens, spec_lens, max_spec_len, interleaved, attn_factor, parents, out, stream)
    if r is not NotImplemented:
        return r
    import torch
    stride = _ragged_rows(x)
    _dense_ints(ctx_lens, spec_lens, *([] if parents is None else [parents]))
    _on_current_device(x)
    assert ctx_lens.device == inv_freq.device == x.device and spec_lens.dim() == 1 and ctx_lens.shape == spec_lens.shape
    assert parents is None or parents.shape == x.shape[:1]
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    else:
        _on_device(out, x.device, "out")
        assert out.shape == x.shape
    dims = _rope_dims(x.shape[0], x.shape[1], 0, x.shape[2], (spec_lens.shape[0], 0), 0, max_spec_len, _dtype_code(x), inv_freq,
                      interleaved, attn_factor)
    dims.q_row_stride, dims.q_out_row_stride = stride, _ragged_rows(out, x)
    rc = lib().adaspec_rope(x.data_ptr(), inv_freq.data_ptr(), out.data_ptr(), ctx_lens.data_ptr(), spec_lens.data_ptr(),
                            None if parents is None else parents.data_ptr(), C.byref(dims), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_rope")
    return out


def kv_append_rope(q, k_new, v_new, inv_freq, k_pages, v_pages, block_table, ctx_lens, spec_lens, *, max_spec_len: int, k_scales=None,
                   v_scales=None, interleaved: bool = False, attn_factor: float = 1.0, parents=None, q_out=None, stream=None):
    """adaspec_kv_append_rope: keys k_new [TQ][Hkv][d] turned by the angles of their positions and written into the pages with v_new,
    in place; returns the queries q [TQ][Hq][d] turned likewise (q_out if given, which may be q itself; None where q is None).
    k_scales, v_scales [num_pages][Hkv] float32: the pages are held in 8 bits (torch.float8_e4m3fn) with these scales, which are
    updated.  inv_freq, interleaved, attn_factor, parents, and rows that are slices: as for rope; inv_freq None: nothing is turned
    (then q is None too)."""
    r = (_fast or _native()).kv_append_rope(q, k_new, v_new, inv_freq, k_pages, v_pages, block_table, ctx_lens, spec_lens, max_spec_len,
                                            k_scales, v_scales, interleaved, attn_factor, parents, q_out, stream)
    if r is not NotImplemented:
        return r
    import torch
    if q is not None and inv_freq is None:
        raise ValueError("kv_append_rope(q=...) needs inv_freq: without it nothing is turned")
    if q is None and q_out is not None:
        raise ValueError("kv_append_rope(q_out=...) needs q")
    TQ, Hkv, d = k_new.shape
    strides = [0, _ragged_rows(k_new), _ragged_rows(v_new, k_new), 0]
    assert v_new.shape == k_new.shape and k_pages.dim() == 4 and block_table.dim() == 2
    if k_scales is not None or v_scales is not None:
        _scaled_cache(k_pages, v_pages, k_scales, v_scales)
    else:
        for t in (k_pages, v_pages):
            assert t.is_cuda and t.is_contiguous() and t.dtype == k_new.dtype
    assert v_pages.shape == k_pages.shape and v_pages.device == k_pages.device == k_new.device
    num_pages, Hkv2, P, d2 = k_pages.shape
    assert (Hkv2, d2) == (Hkv, d)
    _dense_ints(block_table, ctx_lens, spec_lens, *([] if parents is None else [parents]))
    _on_current_device(k_new)
    assert block_table.device == k_new.device and (inv_freq is None or inv_freq.device == k_new.device)
    assert ctx_lens.shape == spec_lens.shape == block_table.shape[:1] and (parents is None or parents.shape == (TQ,))
    if q is not None:
        strides[0] = _ragged_rows(q, k_new)
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        else:
            _on_device(q_out, q.device, "q_out")
            assert q_out.shape == q.shape
        strides[3] = _ragged_rows(q_out, q)
    dims = _rope_dims(TQ, 0 if q is None else q.shape[1], Hkv, d, tuple(block_table.shape), num_pages, max_spec_len, _dtype_code(k_new),
                      inv_freq, interleaved, attn_factor)
    dims.page_size = P
    dims.q_row_stride, dims.k_row_stride, dims.v_row_stride, dims.q_out_row_stride = strides
    ptr = lambda t: None if t is None else t.data_ptr()
    rc = lib().adaspec_kv_append_rope(*[ptr(t) for t in (q, k_new, v_new, inv_freq, q_out, k_pages, v_pages, k_scales, v_scales,
                                                         block_table, ctx_lens, spec_lens, parents)], C.byref(dims), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_kv_append_rope")
    return q_out


def kv_append(k_new, v_new, k_pages, v_pages, block_table, ctx_lens, spec_lens, *, max_spec_len: int,
              stream=None, k_scales=None, v_scales=None) -> None:
    """adaspec_kv_append: writes the new tokens' K/V rows [TQ][Hkv][d] into the pages, in place.
    k_scales, v_scales [num_pages][Hkv]: into a cache of 8 bits (kv_append_rope without turning)."""
    if k_scales is not None or v_scales is not None:
        kv_append_rope(None, k_new, v_new, None, k_pages, v_pages, block_table, ctx_lens, spec_lens, max_spec_len=max_spec_len,
                       k_scales=k_scales, v_scales=v_scales, stream=stream)
        return
    if (_fast or _native()).kv_append(k_new, v_new, k_pages, v_pages, block_table, ctx_lens, spec_lens, max_spec_len,
                                      stream) is not NotImplemented:
        return
    import torch
    TQ, Hkv, d = k_new.shape
    num_pages, Hkv2, P, d2 = k_pages.shape
    B, max_pages = block_table.shape
    assert (Hkv2, d2) == (Hkv, d) and v_new.shape == k_new.shape and v_pages.shape == k_pages.shape
    assert k_new.dtype == v_new.dtype == k_pages.dtype == v_pages.dtype
    for t in (k_new, v_new, k_pages, v_pages, block_table, ctx_lens, spec_lens):
        assert t.is_cuda and t.is_contiguous()
    assert block_table.dtype == torch.int32 and ctx_lens.dtype == torch.int32 and spec_lens.dtype == torch.int32
    dt = _dtype_code(k_new)
    dims = AttnDims(B, TQ, int(max_spec_len), Hkv, Hkv, d, P, num_pages, max_pages, dt, dt, PATH_AUTO, 0.0)
    rc = lib().adaspec_kv_append(k_new.data_ptr(), v_new.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                 block_table.data_ptr(), ctx_lens.data_ptr(), spec_lens.data_ptr(),
                                 C.byref(dims), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_kv_append")


def commit(out_tokens, out_accept_len, spec_lens, ctx_lens, *, max_spec_len: int, next_spec_lens=None,
           committed_lens=None, next_ctx_lens=None, last_token=None, seq_tokens=None, seq_lens=None,
           stream=None):
    """adaspec_commit; returns (committed_lens, next_ctx_lens or None, last_token)."""
    r = (_fast or _native()).commit(out_tokens, out_accept_len, spec_lens, ctx_lens, max_spec_len, next_spec_lens,
                                    committed_lens, next_ctx_lens, last_token, seq_tokens, seq_lens, stream)
    if r is not NotImplemented:
        return r
    import torch
    B, out_stride = out_tokens.shape
    dev = out_tokens.device
    for t in (out_tokens, out_accept_len, spec_lens, ctx_lens):
        assert t.is_cuda and t.is_contiguous() and t.dtype == torch.int32
    if committed_lens is None:
        committed_lens = torch.empty((B,), dtype=torch.int32, device=dev)
    if last_token is None:
        last_token = torch.empty((B,), dtype=torch.int32, device=dev)
    if next_spec_lens is not None and next_ctx_lens is None:
        next_ctx_lens = torch.empty((B,), dtype=torch.int32, device=dev)
    seq_stride = 0
    if seq_tokens is not None:
        assert seq_lens is not None and seq_tokens.is_contiguous() and seq_tokens.dtype == torch.int32
        assert seq_lens.dtype == torch.int32
        seq_stride = seq_tokens.shape[1]
    dims = CommitDims(B, int(max_spec_len), out_stride, seq_stride)
    ptr = lambda t: None if t is None else t.data_ptr()
    rc = lib().adaspec_commit(out_tokens.data_ptr(), out_accept_len.data_ptr(), spec_lens.data_ptr(),
                              ctx_lens.data_ptr(), ptr(next_spec_lens), committed_lens.data_ptr(),
                              ptr(next_ctx_lens), last_token.data_ptr(), ptr(seq_tokens), ptr(seq_lens),
                              C.byref(dims), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_commit")
    return committed_lens, next_ctx_lens, last_token


def _on_current_device(t) -> None:
    import torch
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"tensors on {t.device}, but the current device is cuda:{torch.cuda.current_device()}: make the call under "
                         f"torch.cuda.device({t.device.index})")


def _dense_ints(*tensors):
    import torch
    for t in tensors:
        assert t.is_cuda and t.is_contiguous() and t.dtype == torch.int32 and t.device == tensors[0].device


def _ints_like(given, shape, like):
    """the caller's output tensor, or a new one"""
    import torch
    if given is None:
        return torch.empty(shape, dtype=torch.int32, device=like.device)
    _dense_ints(like, given)
    assert tuple(given.shape) == tuple(shape)
    return given


def kv_remap(block_table, page_refs, sources, lens, new_lens, *, window: Optional[int] = None, sinks: int = 0, page_size: int = 16,
             out_table=None, out_refs=None, copy_src=None, copy_dst=None, status=None, workspace=None, stream=None):
    """adaspec_kv_remap: the block table of the next batch; returns (out_table [batch][max_pages], out_refs [num_pages],
    copy_src [batch], copy_dst [batch], status [2]).

    block_table [old_batch][max_pages], page_refs [num_pages], sources [batch], lens [old_batch], new_lens [batch], all int32.
    window, sinks: pages that no later row of verify_attn(window=, sinks=) sees are given back as well.  out_refs may be
    page_refs; out_table must not overlap block_table.  Results that are not given are new tensors of one allocation, which lasts, with
    the call's workspace behind them, until the last of them is gone.  Calls without workspace= may overlap: each has its own."""
    if window is None and sinks != 0:
        raise ValueError("kv_remap(sinks=...) needs a window: without one every token is visible")
    if window is not None and window < 1:
        raise ValueError("kv_remap(window=...) is at least 1 (None: no window)")
    window, sinks = 0 if window is None else _int32(window), _int32(sinks)
    r = (_fast or _native()).kv_remap(block_table, page_refs, sources, lens, new_lens, window, sinks, page_size, out_table, out_refs,
                                      copy_src, copy_dst, status, workspace, stream)
    if r is not NotImplemented:
        return r
    old_batch, max_pages = block_table.shape
    batch, num_pages = sources.shape[0], page_refs.shape[0]
    _dense_ints(block_table, page_refs, sources, lens, new_lens)
    _on_current_device(block_table)
    assert sources.shape == new_lens.shape == (batch,) and lens.shape == (old_batch,) and page_refs.shape == (num_pages,)
    out_table = _ints_like(out_table, (batch, max_pages), block_table)
    out_refs = _ints_like(out_refs, (num_pages,), block_table)
    copy_src = _ints_like(copy_src, (batch,), block_table)
    copy_dst = _ints_like(copy_dst, (batch,), block_table)
    status = _ints_like(status, (2,), block_table)
    dims = PagesDims(batch, old_batch, max_pages, num_pages, int(page_size), window, sinks, 0)
    L = lib()
    ws = _scratch(L.adaspec_kv_remap_workspace_bytes(C.byref(dims)), block_table.device, workspace, stream)
    rc = L.adaspec_kv_remap(block_table.data_ptr(), page_refs.data_ptr(), sources.data_ptr(), lens.data_ptr(), new_lens.data_ptr(),
                            out_table.data_ptr(), out_refs.data_ptr(), copy_src.data_ptr(), copy_dst.data_ptr(), status.data_ptr(),
                            C.byref(dims), ws.data_ptr(), ws.numel(), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_kv_remap")
    return out_table, out_refs, copy_src, copy_dst, status


def kv_compact_pages(block_table, page_refs, *, max_moves: Optional[int] = None, out_table=None, out_refs=None, page_map=None,
                     copy_src=None, copy_dst=None, status=None, page_size: int = 16, workspace=None, stream=None):
    """adaspec_kv_compact_pages: used pages to the front of the pool; returns (out_table, out_refs, page_map [num_pages],
    copy_src [max_moves], copy_dst [max_moves], status [2]).  max_moves: half of the pool's pages unless given, which is always
    enough.  out_table may be block_table, out_refs may be page_refs.  Results and workspace as for kv_remap."""
    batch, max_pages = block_table.shape
    num_pages = page_refs.shape[0]
    max_moves = max(1, num_pages // 2) if max_moves is None else int(max_moves)
    r = (_fast or _native()).kv_compact_pages(block_table, page_refs, max_moves, page_size, out_table, out_refs, page_map, copy_src,
                                              copy_dst, status, workspace, stream)
    if r is not NotImplemented:
        return r
    _dense_ints(block_table, page_refs)
    _on_current_device(block_table)
    assert page_refs.shape == (num_pages,)
    if max_moves < 1:
        raise ValueError("kv_compact_pages(max_moves=...) is at least 1")
    out_table = _ints_like(out_table, (batch, max_pages), block_table)
    out_refs = _ints_like(out_refs, (num_pages,), block_table)
    page_map = _ints_like(page_map, (num_pages,), block_table)
    copy_src = _ints_like(copy_src, (max_moves,), block_table)
    copy_dst = _ints_like(copy_dst, (max_moves,), block_table)
    status = _ints_like(status, (2,), block_table)
    dims = PagesDims(0, batch, max_pages, num_pages, int(page_size), 0, 0, max_moves)
    L = lib()
    ws = _scratch(L.adaspec_kv_compact_pages_workspace_bytes(C.byref(dims)), block_table.device, workspace, stream)
    rc = L.adaspec_kv_compact_pages(block_table.data_ptr(), page_refs.data_ptr(), out_table.data_ptr(), out_refs.data_ptr(),
                                    page_map.data_ptr(), copy_src.data_ptr(), copy_dst.data_ptr(), status.data_ptr(), C.byref(dims),
                                    ws.data_ptr(), ws.numel(), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_kv_compact_pages")
    return out_table, out_refs, page_map, copy_src, copy_dst, status


def kv_copy_pages(k_pages, v_pages, copy_src, copy_dst, *, stream=None, k_scales=None, v_scales=None) -> None:
    """adaspec_kv_copy_pages: pages copy_src[c] -> copy_dst[c] of K and V, in place; pairs with -1 are left out.
    k_pages, v_pages: the pages of one layer [num_pages][Hkv][P][d], or of several [layers][num_pages][Hkv][P][d].
    k_scales, v_scales [num_pages][Hkv] or [layers][num_pages][Hkv]: adaspec_kv_copy_pages_scaled instead, for a cache of 8 bits."""
    if k_scales is not None or v_scales is not None:
        return _kv_copy_pages_scaled(k_pages, v_pages, k_scales, v_scales, copy_src, copy_dst, stream)
    if (_fast or _native()).kv_copy_pages(k_pages, v_pages, copy_src, copy_dst, stream) is not NotImplemented:
        return
    assert k_pages.dim() in (4, 5)
    layers = k_pages.shape[0] if k_pages.dim() == 5 else 1
    num_pages, Hkv, P, d = k_pages.shape[-4:]
    assert k_pages.is_cuda and k_pages.is_contiguous() and v_pages.is_cuda and v_pages.is_contiguous()
    assert v_pages.shape == k_pages.shape and v_pages.dtype == k_pages.dtype
    _dense_ints(copy_src, copy_dst)
    _on_current_device(k_pages)
    assert v_pages.device == copy_src.device == k_pages.device
    assert copy_src.dim() == 1 and copy_dst.shape == copy_src.shape
    dims = CopyDims(layers, num_pages, Hkv, P, d, _dtype_code(k_pages))
    rc = lib().adaspec_kv_copy_pages(k_pages.data_ptr(), v_pages.data_ptr(), copy_src.data_ptr(), copy_dst.data_ptr(),
                                     copy_src.shape[0], C.byref(dims), _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_kv_copy_pages")


def _kv_copy_pages_scaled(k_pages, v_pages, k_scales, v_scales, copy_src, copy_dst, stream) -> None:
    assert k_pages.dim() in (4, 5)
    layers = k_pages.shape[0] if k_pages.dim() == 5 else 1
    num_pages, Hkv, P, d = k_pages.shape[-4:]
    _scaled_cache(k_pages, v_pages, k_scales, v_scales)
    _dense_ints(copy_src, copy_dst)
    _on_current_device(k_pages)
    assert copy_src.device == k_pages.device and copy_src.dim() == 1 and copy_dst.shape == copy_src.shape
    dims = CopyDims(layers, num_pages, Hkv, P, d, BF16)
    rc = lib().adaspec_kv_copy_pages_scaled(k_pages.data_ptr(), v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(),
                                            copy_src.data_ptr(), copy_dst.data_ptr(), copy_src.shape[0], C.byref(dims),
                                            _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_kv_copy_pages_scaled")


def draft_sample(draft_logits, temperature, uniforms, *, probs_dtype=None, draft_probs=None, out_rows=None,
                 draft_tokens=None, confidence=None, path: str = "auto", workspace=None, stream=None, timing=None):
    """adaspec_draft_sample; returns (draft_probs, draft_tokens [R] int32, confidence [R] float32).
    path "split" (ADASPEC_PATH_TWO_PASS for this call) shares long rows between workgroups.
    workspace: the default one is shared by all calls of a device, which have to be ordered on one stream."""
    if path == "auto" and timing is None:
        r = (_fast or _native()).draft_sample(draft_logits, temperature, uniforms, probs_dtype, draft_probs, out_rows,
                                              draft_tokens, confidence, workspace, stream)
        if r is not NotImplemented:
            return r
    import torch
    R, V = draft_logits.shape
    dev = draft_logits.device
    assert draft_logits.is_cuda and draft_logits.stride(1) == 1
    assert temperature.dtype == torch.float32 and uniforms.dtype == torch.float32
    if draft_probs is None:
        assert out_rows is None
        draft_probs = torch.empty((R, V), dtype=probs_dtype or draft_logits.dtype, device=dev)
    assert draft_probs.stride(1) == 1 and draft_probs.shape[1] == V
    if draft_tokens is None:
        draft_tokens = torch.empty((R,), dtype=torch.int32, device=dev)
    if confidence is None:
        confidence = torch.empty((R,), dtype=torch.float32, device=dev)
    dims = DraftDims(R, V, _dtype_code(draft_logits), _dtype_code(draft_probs), draft_logits.stride(0),
                     draft_probs.stride(0), PATH_TWO_PASS if path == "split" else _PATHS[path], 0)
    _with_timing(dims, timing)
    L = lib()
    need = L.adaspec_draft_sample_workspace_bytes(C.byref(dims))
    ws = _workspace(need, dev, workspace, "draft") if need else None
    rc = L.adaspec_draft_sample(draft_logits.data_ptr(), temperature.data_ptr(), uniforms.data_ptr(),
                                None if out_rows is None else out_rows.data_ptr(), draft_probs.data_ptr(),
                                draft_tokens.data_ptr(), confidence.data_ptr(), C.byref(dims),
                                None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(),
                                _stream_ptr(stream))
    if rc != 0:
        raise AdaspecError(rc, "adaspec_draft_sample")
    return draft_probs, draft_tokens, confidence
