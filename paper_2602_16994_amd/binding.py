"""ctypes binding of libmpv.so: argument marshalling only.

Function names and argument order follow include/mpv.h.  torch is used for
device memory (tensor.data_ptr()) and for the current HIP stream; every step of
the computation runs in the library's kernels.  There is no CPU fallback: if the
library is missing, loading raises.
"""

import contextlib
import ctypes
import os
from dataclasses import dataclass
from typing import Optional

MPV_METHOD_SPECINFER = 0
MPV_METHOD_TRAVERSAL = 1
MPV_METHOD_NSS = 2
MPV_METHOD_NAIVE = 3
MPV_METHOD_SPECTR = 4
# indices into the counters array of a call
MPV_COUNTER_NEAR_TIE_ACCEPT = 0
MPV_COUNTER_NEAR_TIE_BONUS = 1
MPV_COUNTER_ZERO_MASS = 2
MPV_COUNTER_BAD_TOKEN = 3
MPV_COUNTER_DEPENDENCY_TIMEOUT = 4
MPV_COUNTER_NODE_TASKS_RUN = 5
MPV_COUNTER_NODE_TASKS_CANCELLED = 6
MPV_COUNTER_NODE_TASKS_RESUMED = 7
MPV_DTYPE_F32 = 0
MPV_DTYPE_BF16 = 1
MPV_DTYPE_F16 = 2           # mpv_tree_attention, mpv_verify_chains and mpv_append_paths only

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))


def lib_path():
    return os.path.join(_PKG_DIR, "libmpv.so")


class MpvError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        extra = f", hipError {mpv_last_hip_error()}" if code == -9 else ""
        super().__init__(f"{where}: {mpv_strerror(code)} (code {code}{extra})")


class _Problem(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("N", ctypes.c_int32), ("V", ctypes.c_int32),
        ("method", ctypes.c_int32), ("logit_dtype", ctypes.c_int32),
        ("temperature", ctypes.c_float), ("max_depth", ctypes.c_int32),
        ("parent", ctypes.POINTER(ctypes.c_int32)),
    ]


class _Buffers(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in (
        "target_logits", "draft_logits", "tokens", "uniforms",
        "accept_len", "path_nodes", "path_tokens", "bonus_token", "counters",
        "stats", "edge_probs", "accept_prob", "final_residual", "draw_uniforms")]


class _Attention(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "N", "heads", "kv_heads", "head_dim", "dtype", "num_pages", "page_size", "table_width",
                                               "window", "sinks")]
                + [("scale", ctypes.c_float)]
                + [(n, ctypes.c_int64) for n in ("q_stride", "kv_stride", "out_stride", "page_stride", "slot_stride")]
                + [("parent", ctypes.POINTER(ctypes.c_int32))])


class _AttentionBuffers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "tree_k", "tree_v", "cache_k", "cache_v", "block_table", "context_len", "num_nodes",
                                               "tree_parent", "out")]


class _Chains(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "N", "V", "dtype", "max_depth")]
                + [(n, ctypes.c_int64) for n in ("target_stride", "draft_stride")])


class _ChainBuffers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("target_probs", "draft_probs", "tokens", "uniforms", "num_nodes", "accept_len", "path_nodes",
                                               "path_tokens", "bonus_token", "counters")]


class _Tables(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "page_size", "table_width", "num_pages", "extra", "packed")]
                + [("slot_width", ctypes.c_int64)])


class _TableBuffers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("new_len", "context_len", "block_table", "free_pages", "free_count", "context_len_out",
                                               "free_count_out", "slot_map", "granted", "offsets")]


class _Append(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("layers", "B", "N", "dtype", "row", "max_depth", "slot_width", "num_pages", "page_size")]
                + [(n, ctypes.c_int64) for n in ("tree_layer_stride", "tree_stride", "cache_layer_stride", "page_stride", "slot_stride")])


class _AppendBuffers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("tree_k", "tree_v", "cache_k", "cache_v", "slot_map", "accept_len", "path_nodes")]


_lib = None


def load_library(path=None):
    """Load libmpv.so (built by paper_2602_16994_amd.build) and declare prototypes."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    # torch ships its own HIP runtime; import it first so that libmpv.so binds to
    # the same runtime instance (device memory and streams come from torch).
    import torch  # noqa: F401
    path = path or lib_path()
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} not found: build it with `python -m paper_2602_16994_amd.build` "
            "(there is no fallback implementation)")
    lib = ctypes.CDLL(path)
    lib.mpv_version.restype = ctypes.c_int
    lib.mpv_version.argtypes = []
    lib.mpv_strerror.restype = ctypes.c_char_p
    lib.mpv_strerror.argtypes = [ctypes.c_int]
    lib.mpv_last_hip_error.restype = ctypes.c_int
    lib.mpv_last_hip_error.argtypes = []
    lib.mpv_workspace_bytes.restype = ctypes.c_int
    lib.mpv_workspace_bytes.argtypes = [ctypes.POINTER(_Problem), ctypes.POINTER(ctypes.c_size_t)]
    lib.mpv_verify.restype = ctypes.c_int
    lib.mpv_verify.argtypes = [ctypes.POINTER(_Problem), ctypes.POINTER(_Buffers),
                               ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    lib.mpv_verify_static.restype = ctypes.c_int
    lib.mpv_verify_static.argtypes = [ctypes.POINTER(_Problem), ctypes.POINTER(_Buffers), ctypes.c_void_p]
    lib.mpv_merge_duplicates.restype = ctypes.c_int
    lib.mpv_merge_duplicates.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32,
                                         ctypes.c_void_p, ctypes.c_void_p]
    lib.mpv_verify_merged.restype = ctypes.c_int
    lib.mpv_verify_merged.argtypes = [ctypes.POINTER(_Problem), ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_Buffers),
                                      ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    lib.mpv_block_efficiency.restype = ctypes.c_int
    lib.mpv_block_efficiency.argtypes = [ctypes.POINTER(_Problem), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_void_p]
    lib.mpv_block_efficiency_merged.restype = ctypes.c_int
    lib.mpv_block_efficiency_merged.argtypes = [ctypes.POINTER(_Problem), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                                ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                                ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.mpv_acceptance_rates.restype = ctypes.c_int
    lib.mpv_acceptance_rates.argtypes = [ctypes.POINTER(_Problem), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.mpv_acceptance_rates_merged.restype = ctypes.c_int
    lib.mpv_acceptance_rates_merged.argtypes = [ctypes.POINTER(_Problem), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                                ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p,
                                                ctypes.c_void_p]
    lib.mpv_nucleus_mask.restype = ctypes.c_int
    lib.mpv_nucleus_mask.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_int32,
                                     ctypes.c_float, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.mpv_row_stats.restype = ctypes.c_int
    lib.mpv_row_stats.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_int32,
                                  ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p]
    lib.mpv_fill_uniforms.restype = ctypes.c_int
    lib.mpv_fill_uniforms.argtypes = [ctypes.c_uint64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]
    for name, shape, bufs in (("mpv_tree_attention", _Attention, _AttentionBuffers), ("mpv_verify_chains", _Chains, _ChainBuffers),
                              ("mpv_extend_tables", _Tables, _TableBuffers)):
        call, size = getattr(lib, name), getattr(lib, name + "_workspace_bytes")
        call.restype = size.restype = ctypes.c_int
        call.argtypes = [ctypes.POINTER(shape), ctypes.POINTER(bufs), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        size.argtypes = [ctypes.POINTER(shape), ctypes.POINTER(ctypes.c_size_t)]
    lib.mpv_append_paths.restype = ctypes.c_int
    lib.mpv_append_paths.argtypes = [ctypes.POINTER(_Append), ctypes.POINTER(_AppendBuffers), ctypes.c_void_p]
    lib.mpv_timing_enable.restype = ctypes.c_int
    lib.mpv_timing_enable.argtypes = [ctypes.c_int32]
    lib.mpv_timing_read.restype = ctypes.c_int
    lib.mpv_timing_read.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int32),
                                    ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]
    _lib = lib
    return lib


def mpv_version():
    return load_library().mpv_version()


def mpv_strerror(code):
    return load_library().mpv_strerror(int(code)).decode()


def mpv_last_hip_error():
    return load_library().mpv_last_hip_error()


def _make_problem(B, N, V, method, logit_dtype, temperature, max_depth, parent):
    arr = (ctypes.c_int32 * len(parent))(*[int(x) for x in parent]) if parent is not None else None
    prob = _Problem(int(B), int(N), int(V), int(method), int(logit_dtype), float(temperature),
                    int(max_depth), arr)
    prob._keepalive = arr
    return prob


def mpv_workspace_bytes(B, N, V, method, logit_dtype, temperature, max_depth, parent):
    prob = _make_problem(B, N, V, method, logit_dtype, temperature, max_depth, parent)
    out = ctypes.c_size_t(0)
    rc = load_library().mpv_workspace_bytes(ctypes.byref(prob), ctypes.byref(out))
    if rc != 0:
        raise MpvError(rc, "mpv_workspace_bytes")
    return out.value


def _stream_ptr(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


_nothing = contextlib.nullcontext()


def _allocating(stream):
    """What a call allocates, its results and workspace, is allocated on the stream that it runs on: memory that was given back on
    another one may still be in use by work that was enqueued there before, and the call's stream does not wait for that."""
    if stream is None:
        return _nothing
    import torch
    return torch.cuda.stream(stream)


def _workspace(out, need, device, stream, raw):
    """out.workspace, of at least `need` bytes, for a call on `stream` (handle `raw`)."""
    import torch
    ws = out.workspace
    if ws is None or ws.numel() < need or ws.get_device() != device:
        with _allocating(stream):
            ws = out.workspace = torch.empty(need, dtype=torch.uint8, device=torch.device("cuda", device))
    elif getattr(out, "_workspace_stream", None) != raw:           # it is used on another stream than the one before
        ws.record_stream(torch.cuda.current_stream() if stream is None else stream)
    out._workspace_stream = raw
    return ws


def _used_on(stream, out, workspace=None):
    """Tells the allocator of a call on `stream`: what was allocated elsewhere is in use there, and results that were allocated on it are
    used on the current one next; neither must be given away before that is done."""
    import torch
    if stream is None:
        return
    current = torch.cuda.current_stream()
    if stream.cuda_stream == current.cuda_stream:
        return
    for t in out:
        if isinstance(t, torch.Tensor) and t.is_cuda:
            t.record_stream(stream)
            if t is not workspace:
                t.record_stream(current)


def _no_counts(stream, counters):
    """The counters of a batch of none: the library writes nothing then."""
    with _allocating(stream):
        counters.zero_()


def _dtype_id(t):
    import torch
    if t.dtype == torch.float32:
        return MPV_DTYPE_F32
    if t.dtype == torch.bfloat16:
        return MPV_DTYPE_BF16
    raise TypeError(f"logits must be float32 or bfloat16, got {t.dtype}")


class MpvTimeout(RuntimeError):
    """A wait inside the kernels ran into its time limit: the outputs of that call are invalid."""


def _raise_on_timeout(counters, where):
    """Reads the call's counters (this synchronises with the stream the call ran on) and raises
    if the library reported a dependency timeout."""
    n = int(counters[MPV_COUNTER_DEPENDENCY_TIMEOUT].item())
    if n:
        raise MpvTimeout(f"{where}: {n} waits inside the kernels timed out; the outputs are invalid")


@dataclass
class VerifyResult:
    accept_len: "object"
    path_nodes: "object"
    path_tokens: "object"
    bonus_token: "object"
    counters: "object"
    stats: Optional["object"] = None
    edge_probs: Optional["object"] = None
    accept_prob: Optional["object"] = None
    final_residual: Optional["object"] = None
    workspace: Optional["object"] = None

    def raise_on_timeout(self):
        """Synchronises and raises MpvTimeout if the call gave up on a wait (counters[4] != 0)."""
        _raise_on_timeout(self.counters, "mpv_verify")


def mpv_merge_duplicates(parent, tokens):
    """Host call (see include/mpv.h): parent list of N ints, tokens an int32 array [B,N] on the host
    (numpy, or a CPU torch tensor).  Returns (merged_parent, context_node), numpy int32 [B,N]."""
    import numpy as np
    tok = np.ascontiguousarray(np.asarray(tokens), dtype=np.int32)
    if tok.ndim != 2 or tok.shape[1] != len(parent):
        raise ValueError("tokens must be [B,N] with N = len(parent)")
    B, N = tok.shape
    par = np.ascontiguousarray(np.asarray(parent, dtype=np.int32))
    merged = np.empty((B, N), dtype=np.int32)
    context = np.empty((B, N), dtype=np.int32)
    rc = load_library().mpv_merge_duplicates(par.ctypes.data, tok.ctypes.data, B, N,
                                             merged.ctypes.data, context.ctypes.data)
    if rc != 0:
        raise MpvError(rc, "mpv_merge_duplicates")
    return merged, context


def mpv_verify(parent, tokens, target_logits, draft_logits, temperature, uniforms, method,
               max_depth=None, debug=False, out=None, workspace=None, stream=None, draw_uniforms=None,
               static_scratch=False, merged_parent=None, context_node=None):
    """Enqueue one batched verification on the current (or given) torch stream.

    parent: list of N ints (host).  tokens int32 [B,N], target_logits / draft_logits
    [B,N,V] float32 or bfloat16, uniforms float32 [B,N]: CUDA tensors, contiguous.
    Returns a VerifyResult of CUDA tensors (asynchronous; synchronise before reading
    on the host).  `out` may be a previous VerifyResult whose buffers are reused.
    draw_uniforms float32 [B,N] is needed by MPV_METHOD_NSS, MPV_METHOD_NAIVE and MPV_METHOD_SPECTR (the draw at
    each visited node); with those methods debug=True provides accept_prob and final_residual only.
    static_scratch=True calls mpv_verify_static: no workspace tensor, the library's own device array.
    merged_parent (numpy int32 [B,N] on the host, one parent array per tree) calls mpv_verify_merged;
    `parent` then only serves to size the outputs and the workspace.  MPV_METHOD_SPECTR also needs
    context_node: an int32 CUDA tensor [B,N] (what mpv_merge_duplicates returned, copied to the device).
    """
    import torch
    from .trees import tree_depth
    B, N, V = target_logits.shape
    for t, name in ((tokens, "tokens"), (target_logits, "target_logits"),
                    (draft_logits, "draft_logits"), (uniforms, "uniforms")):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous CUDA tensor")
    if tokens.dtype != torch.int32 or uniforms.dtype != torch.float32:
        raise TypeError("tokens must be int32 and uniforms float32")
    if draft_logits.shape != target_logits.shape or draft_logits.dtype != target_logits.dtype:
        raise ValueError("target and draft logits must have the same shape and dtype")
    if tuple(tokens.shape) != (B, N) or tuple(uniforms.shape) != (B, N):
        raise ValueError("tokens and uniforms must be [B,N]")
    if draw_uniforms is not None:
        if (not draw_uniforms.is_cuda or not draw_uniforms.is_contiguous() or draw_uniforms.dtype != torch.float32
                or tuple(draw_uniforms.shape) != (B, N)):
            raise ValueError("draw_uniforms must be a contiguous float32 CUDA tensor [B,N]")
    if max_depth is None:
        max_depth = max(1, tree_depth(list(parent)) if len(parent) == N and N > 0 else 1)
    dev = target_logits.device
    prob = _make_problem(B, N, V, method, _dtype_id(target_logits), temperature, max_depth, parent)
    if out is None:
        i32 = dict(dtype=torch.int32, device=dev)
        with _allocating(stream):
            out = VerifyResult(
                accept_len=torch.empty(B, **i32),
                path_nodes=torch.empty(B, max_depth, **i32),
                path_tokens=torch.empty(B, max_depth, **i32),
                bonus_token=torch.empty(B, **i32),
                counters=torch.empty(8, dtype=torch.int32, device=dev),
            )
            if debug:
                f32 = dict(dtype=torch.float32, device=dev)
                if method in (MPV_METHOD_SPECINFER, MPV_METHOD_TRAVERSAL):
                    out.stats = torch.empty(B, N, 4, **f32)
                    out.edge_probs = torch.empty(B, N, 2, **f32)
                out.accept_prob = torch.empty(B, N, **f32)
                out.final_residual = torch.empty(B, V, **f32)
    if not B:
        _no_counts(stream, out.counters)
    lib, on = load_library(), _stream_ptr(stream)

    def ptr(t):
        return ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)

    if not static_scratch:
        need = ctypes.c_size_t(0)
        rc = lib.mpv_workspace_bytes(ctypes.byref(prob), ctypes.byref(need))
        if rc != 0:
            raise MpvError(rc, "mpv_workspace_bytes")
        if workspace is not None and workspace is not out.workspace:
            out.workspace, out._workspace_stream = workspace, None
        workspace = _workspace(out, max(need.value, 256), target_logits.get_device(), stream, on.value)

    bufs = _Buffers(ptr(target_logits), ptr(draft_logits), ptr(tokens), ptr(uniforms),
                    ptr(out.accept_len), ptr(out.path_nodes), ptr(out.path_tokens),
                    ptr(out.bonus_token), ptr(out.counters),
                    ptr(out.stats), ptr(out.edge_probs), ptr(out.accept_prob), ptr(out.final_residual),
                    ptr(draw_uniforms))
    if merged_parent is not None:
        import numpy as np
        rows = np.ascontiguousarray(np.asarray(merged_parent), dtype=np.int32)
        if static_scratch or rows.shape != (B, N):
            raise ValueError("merged_parent must be [B,N] and cannot be combined with static_scratch")
        if context_node is not None and (not context_node.is_cuda or not context_node.is_contiguous()
                                         or context_node.dtype != torch.int32 or tuple(context_node.shape) != (B, N)):
            raise ValueError("context_node must be a contiguous int32 CUDA tensor [B,N]")
        rc = lib.mpv_verify_merged(ctypes.byref(prob), rows.ctypes.data, ptr(context_node), ctypes.byref(bufs),
                                   ptr(workspace), ctypes.c_size_t(workspace.numel()), on)
        if rc != 0:
            raise MpvError(rc, "mpv_verify_merged")
        _used_on(stream, vars(out).values(), workspace)
        return out
    if static_scratch:
        rc = lib.mpv_verify_static(ctypes.byref(prob), ctypes.byref(bufs), on)
    else:
        rc = lib.mpv_verify(ctypes.byref(prob), ctypes.byref(bufs), ptr(workspace),
                            ctypes.c_size_t(workspace.numel()), on)
    if rc != 0:
        raise MpvError(rc, "mpv_verify_static" if static_scratch else "mpv_verify")
    _used_on(stream, vars(out).values(), workspace)
    return out


@dataclass
class BlockEfficiencyResult:
    expected: "object"          # float32 [B]    E[tau + 1 | tree]
    reach_prob: "object"        # float32 [B,N]  P(node on the accepted path)
    counters: "object"
    workspace: Optional["object"] = None

    def raise_on_timeout(self):
        """Synchronises and raises MpvTimeout if the call gave up on a wait (counters[4] != 0)."""
        _raise_on_timeout(self.counters, "mpv_block_efficiency")


def mpv_block_efficiency(parent, tokens, target_logits, draft_logits, temperature, method,
                         out=None, stream=None, merged_parent=None, context_node=None):
    """Expected block efficiency of every tree of the batch (see include/mpv.h): enqueued on the
    current (or given) torch stream; returns a BlockEfficiencyResult of CUDA tensors.  Arguments as
    for mpv_verify, without uniforms.  `out` may be a previous result whose buffers are reused.
    merged_parent (numpy int32 [B,N] on the host) calls mpv_block_efficiency_merged; MPV_METHOD_SPECTR
    then also needs context_node, an int32 CUDA tensor [B,N]."""
    import torch
    from .trees import tree_depth
    B, N, V = target_logits.shape
    for t, name in ((tokens, "tokens"), (target_logits, "target_logits"), (draft_logits, "draft_logits")):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous CUDA tensor")
    if tokens.dtype != torch.int32 or tuple(tokens.shape) != (B, N):
        raise TypeError("tokens must be int32 [B,N]")
    if draft_logits.shape != target_logits.shape or draft_logits.dtype != target_logits.dtype:
        raise ValueError("target and draft logits must have the same shape and dtype")
    dev = target_logits.device
    max_depth = max(1, tree_depth(list(parent)) if len(parent) == N and N > 0 else 1)
    prob = _make_problem(B, N, V, method, _dtype_id(target_logits), temperature, max_depth, parent)
    lib, on = load_library(), _stream_ptr(stream)
    need = ctypes.c_size_t(0)
    rc = lib.mpv_workspace_bytes(ctypes.byref(prob), ctypes.byref(need))
    if rc != 0:
        raise MpvError(rc, "mpv_workspace_bytes")
    if out is None:
        with _allocating(stream):
            out = BlockEfficiencyResult(
                expected=torch.empty(B, dtype=torch.float32, device=dev),
                reach_prob=torch.empty(B, N, dtype=torch.float32, device=dev),
                counters=torch.empty(8, dtype=torch.int32, device=dev))
    _workspace(out, max(need.value, 256), target_logits.get_device(), stream, on.value)
    if not B:
        _no_counts(stream, out.counters)

    def ptr(t):
        return ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)

    if merged_parent is not None:
        import numpy as np
        rows = np.ascontiguousarray(np.asarray(merged_parent), dtype=np.int32)
        if rows.shape != (B, N):
            raise ValueError("merged_parent must be [B,N]")
        if context_node is not None and (not context_node.is_cuda or not context_node.is_contiguous()
                                         or context_node.dtype != torch.int32 or tuple(context_node.shape) != (B, N)):
            raise ValueError("context_node must be a contiguous int32 CUDA tensor [B,N]")
        rc = lib.mpv_block_efficiency_merged(ctypes.byref(prob), rows.ctypes.data, ptr(context_node), ptr(target_logits), ptr(draft_logits),
                                             ptr(tokens), ptr(out.workspace), ctypes.c_size_t(out.workspace.numel()),
                                             ptr(out.reach_prob), ptr(out.expected), ptr(out.counters), on)
        if rc != 0:
            raise MpvError(rc, "mpv_block_efficiency_merged")
        _used_on(stream, vars(out).values(), out.workspace)
        return out
    rc = lib.mpv_block_efficiency(ctypes.byref(prob), ptr(target_logits), ptr(draft_logits), ptr(tokens),
                                  ptr(out.workspace), ctypes.c_size_t(out.workspace.numel()),
                                  ptr(out.reach_prob), ptr(out.expected), ptr(out.counters), on)
    if rc != 0:
        raise MpvError(rc, "mpv_block_efficiency")
    _used_on(stream, vars(out).values(), out.workspace)
    return out


def mpv_acceptance_rates(parent, target_logits, draft_logits, temperature, method, stream=None, merged_parent=None):
    """Acceptance rate of the solver `method` at every internal node (see include/mpv.h): returns
    (alpha float32 [B,N], counters) as CUDA tensors; leaves get 0.  merged_parent (numpy int32 [B,N]
    on the host, one parent array per tree) calls mpv_acceptance_rates_merged."""
    import torch
    from .trees import tree_depth
    B, N, V = target_logits.shape
    for t, name in ((target_logits, "target_logits"), (draft_logits, "draft_logits")):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous CUDA tensor")
    if draft_logits.shape != target_logits.shape or draft_logits.dtype != target_logits.dtype:
        raise ValueError("target and draft logits must have the same shape and dtype")
    dev = target_logits.device
    max_depth = max(1, tree_depth(list(parent)) if len(parent) == N and N > 0 else 1)
    prob = _make_problem(B, N, V, method, _dtype_id(target_logits), temperature, max_depth, parent)
    lib = load_library()
    need = ctypes.c_size_t(0)
    rc = lib.mpv_workspace_bytes(ctypes.byref(prob), ctypes.byref(need))
    if rc != 0:
        raise MpvError(rc, "mpv_workspace_bytes")
    with _allocating(stream):
        workspace = torch.empty(max(need.value, 256), dtype=torch.uint8, device=dev)
        alpha = torch.empty(B, N, dtype=torch.float32, device=dev)
        counters = torch.empty(8, dtype=torch.int32, device=dev)
    if not B:
        _no_counts(stream, counters)
    if merged_parent is not None:
        import numpy as np
        rows = np.ascontiguousarray(np.asarray(merged_parent), dtype=np.int32)
        if rows.shape != (B, N):
            raise ValueError("merged_parent must be [B,N]")
        rc = lib.mpv_acceptance_rates_merged(ctypes.byref(prob), rows.ctypes.data, ctypes.c_void_p(target_logits.data_ptr()),
                                             ctypes.c_void_p(draft_logits.data_ptr()), ctypes.c_void_p(workspace.data_ptr()),
                                             ctypes.c_size_t(workspace.numel()), ctypes.c_void_p(alpha.data_ptr()),
                                             ctypes.c_void_p(counters.data_ptr()), _stream_ptr(stream))
        if rc != 0:
            raise MpvError(rc, "mpv_acceptance_rates_merged")
        _used_on(stream, (alpha, counters))
        return alpha, counters
    rc = lib.mpv_acceptance_rates(ctypes.byref(prob), ctypes.c_void_p(target_logits.data_ptr()),
                                  ctypes.c_void_p(draft_logits.data_ptr()), ctypes.c_void_p(workspace.data_ptr()),
                                  ctypes.c_size_t(workspace.numel()), ctypes.c_void_p(alpha.data_ptr()),
                                  ctypes.c_void_p(counters.data_ptr()), _stream_ptr(stream))
    if rc != 0:
        raise MpvError(rc, "mpv_acceptance_rates")
    _used_on(stream, (alpha, counters))
    return alpha, counters


def mpv_nucleus_mask(logits, temperature, top_p, out=None, inplace=False, stream=None):
    """Nucleus (top-p) transform of every row of a CUDA tensor [..., V] (see include/mpv.h): tokens
    outside the nucleus get the logit -inf.  Returns (masked, threshold[...], kept[...]); with
    inplace=True `masked` is `logits` itself."""
    import torch
    if not logits.is_cuda or not logits.is_contiguous() or logits.dim() < 1:
        raise ValueError("logits must be a contiguous CUDA tensor")
    V = logits.shape[-1]
    rows = logits.numel() // V if V else 0
    lead = tuple(logits.shape[:-1])
    with _allocating(stream):
        if inplace:
            out = logits
        elif out is None:
            out = torch.empty_like(logits)
        thr = torch.empty(lead, dtype=torch.float32, device=logits.device)
        kept = torch.empty(lead, dtype=torch.int32, device=logits.device)
    rc = load_library().mpv_nucleus_mask(ctypes.c_void_p(logits.data_ptr()), ctypes.c_void_p(out.data_ptr()),
                                         _dtype_id(logits), rows, V, float(temperature), float(top_p),
                                         ctypes.c_void_p(thr.data_ptr()), ctypes.c_void_p(kept.data_ptr()),
                                         _stream_ptr(stream))
    if rc != 0:
        raise MpvError(rc, "mpv_nucleus_mask")
    _used_on(stream, (out, thr, kept))
    return out, thr, kept


def mpv_row_stats(logits, temperature, out=None, stream=None):
    """(max, ln sum exp((z-max)/T)) of every row of a [rows, V] CUDA tensor."""
    import torch
    if not logits.is_cuda or not logits.is_contiguous() or logits.dim() != 2:
        raise ValueError("logits must be a contiguous 2-D CUDA tensor")
    rows, V = logits.shape
    if out is None:
        with _allocating(stream):
            out = torch.empty(rows, 2, dtype=torch.float32, device=logits.device)
    rc = load_library().mpv_row_stats(ctypes.c_void_p(logits.data_ptr()), _dtype_id(logits), rows, V,
                                      float(temperature), ctypes.c_void_p(out.data_ptr()), _stream_ptr(stream))
    if rc != 0:
        raise MpvError(rc, "mpv_row_stats")
    _used_on(stream, (out,))
    return out


def mpv_fill_uniforms(seed, count, out=None, device="cuda", stream=None):
    """count counter-based uniforms in [0,1) from `seed` (see include/mpv.h)."""
    import torch
    if out is None:
        with _allocating(stream):
            out = torch.empty(count, dtype=torch.float32, device=device)
    rc = load_library().mpv_fill_uniforms(ctypes.c_uint64(seed & (2 ** 64 - 1)), int(count),
                                          ctypes.c_void_p(out.data_ptr()), _stream_ptr(stream))
    if rc != 0:
        raise MpvError(rc, "mpv_fill_uniforms")
    _used_on(stream, (out,))
    return out


# ------------------------------------------------------------------ the calls around a verification


def _dtype_of(t):
    import torch
    ids = {torch.float32: MPV_DTYPE_F32, torch.bfloat16: MPV_DTYPE_BF16, torch.float16: MPV_DTYPE_F16}
    if t.dtype not in ids:
        raise TypeError(f"tensors must be float32, bfloat16 or float16, got {t.dtype}")
    return ids[t.dtype]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _on_device(dev, **tensors):
    for name, t in tensors.items():
        if t is not None and (not t.is_cuda or t.device != dev):
            raise ValueError(f"{name} must be a CUDA tensor on {dev}")


def _whole(dev, dtype, **tensors):
    """Contiguous tensors of one type on one device: name=(tensor or None, shape)."""
    for name, (t, shape) in tensors.items():
        if t is None:
            continue
        _on_device(dev, **{name: t})
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if not t.is_contiguous() or tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must be a contiguous tensor {list(shape)}, got {list(t.shape)} with strides {list(t.stride())}")


def _int32(**numbers):
    """Numbers that the library takes in 32 bits: ctypes would cut others off without a word."""
    for name, x in numbers.items():
        if not -2 ** 31 <= x < 2 ** 31:
            raise ValueError(f"{name} must fit 32 bits, got {x}")


def _row_stride(name, t, lead, inner):
    """Elements between the rows of a tensor [*lead, *inner] whose rows (the inner dimensions) are contiguous and whose leading
    dimensions follow each other."""
    if tuple(t.shape) != (*lead, *inner):
        raise ValueError(f"{name} must be {[*lead, *inner]}, got {list(t.shape)}")
    n = len(lead)
    want = 1
    for d in range(len(inner) - 1, -1, -1):
        if inner[d] != 1 and t.stride(n + d) != want:
            raise ValueError(f"the rows of {name} must be contiguous, got strides {list(t.stride())}")
        want *= inner[d]
    stride, count = None, 1
    for d in range(n - 1, -1, -1):
        if lead[d] != 1:
            if stride is None:
                if t.stride(d) % count:
                    raise ValueError(f"the rows of {name} must be evenly spaced, got strides {list(t.stride())}")
                stride = t.stride(d) // count
            elif t.stride(d) != stride * count:
                raise ValueError(f"the rows of {name} must be evenly spaced, got strides {list(t.stride())}")
        count *= lead[d]
    return want if stride is None else stride


def _cache_strides(k, v, shape):
    """(page stride, slot stride) of the cache tensors [num_pages, page_size, kv_heads, head_dim]."""
    strides = []
    for name, t in (("cache_k", k), ("cache_v", v)):
        if t.dim() != 4 or tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
        if (shape[3] != 1 and t.stride(3) != 1) or (shape[2] != 1 and t.stride(2) != shape[3]):
            raise ValueError(f"the slots of {name} must be contiguous, got strides {list(t.stride())}")
        slot = t.stride(1) if shape[1] != 1 else shape[2] * shape[3]
        strides.append((t.stride(0) if shape[0] != 1 else slot * shape[1], slot))
    if strides[0] != strides[1]:
        raise ValueError("cache_k and cache_v must have the same strides")
    return strides[0]


class _Plan:
    """What a call derives from the shapes, strides and types of its tensors: checked once, used again for tensors that agree in them."""

    def __init__(self, name, device, shape):
        self.name, self.device, self.shape = name, device, shape
        lib = load_library()
        self.call = getattr(lib, name)
        self.address = ctypes.byref(shape)
        self.need = None
        global _raw_stream
        if _raw_stream is None:              # the current stream's handle without a Stream object around it (2 us a call), where torch has it
            import torch
            _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if name != "mpv_append_paths":
            need = ctypes.c_size_t(0)
            rc = getattr(lib, name + "_workspace_bytes")(self.address, ctypes.byref(need))
            if rc != 0:
                raise MpvError(rc, name + "_workspace_bytes")
            self.need = max(need.value, 256)


_plans = {}
_raw_stream = None


def _kept(key, plan):
    if len(_plans) >= 1024:                  # sizes that change without end: start again
        _plans.clear()
    _plans[key] = plan
    return plan


def _like(t):
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device())


def _launch(plan, bufs, out, stream):
    """The call on its tensors' device; its workspace, if it has one, is kept in out.workspace."""
    import torch
    if torch.cuda.current_device() != plan.device:
        with torch.cuda.device(plan.device):
            return _launch(plan, bufs, out, stream)
    if stream is not None:
        raw = stream.cuda_stream
    elif _raw_stream is not None:
        raw = _raw_stream(plan.device)
    else:
        raw = torch.cuda.current_stream().cuda_stream
    if plan.need is None:
        rc = plan.call(plan.address, ctypes.byref(bufs), raw)
    else:
        ws = _workspace(out, plan.need, plan.device, stream, raw)
        rc = plan.call(plan.address, ctypes.byref(bufs), ws.data_ptr(), ws.numel(), raw)
    if rc != 0:
        raise MpvError(rc, plan.name)
    if stream is not None and out is not None:
        _used_on(stream, vars(out).values(), out.workspace)
    return out


@dataclass
class TreeAttentionResult:
    out: "object"               # [B,N,heads,head_dim]
    workspace: Optional["object"] = None


def mpv_tree_attention(parent, q, tree_k, tree_v, cache_k, cache_v, block_table, context_len, scale=None, window=0, sinks=0,
                       num_nodes=None, tree_parent=None, out=None, stream=None):
    """Attention of the nodes of B draft trees over a paged cache and their own tree (see include/mpv.h), enqueued on the current
    (or given) torch stream; returns a TreeAttentionResult.

    parent: list of N ints (host).  q [B,N,heads,head_dim], tree_k / tree_v [B,N,kv_heads,head_dim], cache_k / cache_v
    [num_pages,page_size,kv_heads,head_dim]: CUDA tensors of one type (float32, bfloat16 or float16).  The rows of a node and the
    slots of a cache are contiguous; nodes may lie further apart (slices of a projection's output), and so may slots and pages.
    block_table int32 [B,table_width], context_len int32 [B].  scale: head_dim ** -0.5 unless given.  num_nodes int32 [B]: only
    so many nodes of a tree exist (rows of `out` behind them are left as they were).  tree_parent int32 [B,N], on the device: a
    parent array per tree, in the place of `parent`.  `out` may be a previous TreeAttentionResult whose buffers are reused."""
    import torch
    key = ("attention", None if tree_parent is not None else tuple(parent), scale, window, sinks, _like(q), _like(tree_k), _like(tree_v),
           _like(cache_k), _like(cache_v), _like(block_table), _like(context_len), _like(num_nodes), _like(tree_parent),
           None if out is None else _like(out.out))
    plan = _plans.get(key)
    if plan is None:
        plan = _kept(key, _attention_plan(parent, q, tree_k, tree_v, cache_k, cache_v, block_table, context_len, scale, window, sinks,
                                          num_nodes, tree_parent, out))
    if out is None:
        with _allocating(stream):
            out = TreeAttentionResult(out=torch.empty(q.shape, dtype=q.dtype, device=q.device))
    bufs = _AttentionBuffers(q.data_ptr(), tree_k.data_ptr(), tree_v.data_ptr(), cache_k.data_ptr(), cache_v.data_ptr(), block_table.data_ptr(),
                             context_len.data_ptr(), _ptr(num_nodes), _ptr(tree_parent), out.out.data_ptr())
    return _launch(plan, bufs, out, stream)


def _attention_plan(parent, q, tree_k, tree_v, cache_k, cache_v, block_table, context_len, scale, window, sinks, num_nodes, tree_parent, out):
    import torch
    _int32(window=window, sinks=sinks)
    if tree_parent is None:
        for n, up in enumerate(parent):
            _int32(**{f"parent[{n}]": up})
    if q.dim() != 4 or tree_k.dim() != 4 or cache_k.dim() != 4 or block_table.dim() != 2:
        raise ValueError("q, tree_k, tree_v, cache_k and cache_v must have 4 dimensions, block_table 2")
    B, N, heads, head_dim = q.shape
    kv_heads, dev = tree_k.shape[2], q.device
    _on_device(dev, q=q, tree_k=tree_k, tree_v=tree_v, cache_k=cache_k, cache_v=cache_v)
    if any(t.dtype != q.dtype for t in (tree_k, tree_v, cache_k, cache_v)):
        raise TypeError("q, tree_k, tree_v, cache_k and cache_v must have the same dtype")
    dtype = _dtype_of(q)
    kv_stride = _row_stride("tree_k", tree_k, (B, N), (kv_heads, head_dim))
    if _row_stride("tree_v", tree_v, (B, N), (kv_heads, head_dim)) != kv_stride:
        raise ValueError("tree_k and tree_v must have the same strides")
    num_pages, page_size = cache_k.shape[0], cache_k.shape[1]
    page_stride, slot_stride = _cache_strides(cache_k, cache_v, (num_pages, page_size, kv_heads, head_dim))
    width = block_table.shape[1]
    _whole(dev, torch.int32, block_table=(block_table, (B, width)), context_len=(context_len, (B,)), num_nodes=(num_nodes, (B,)),
           tree_parent=(tree_parent, (B, N)))
    if tree_parent is None and len(parent) != N:
        raise ValueError("parent must have as many entries as a tree has nodes")
    out_stride = heads * head_dim
    if out is not None:
        _on_device(dev, out=out.out)
        if out.out.dtype != q.dtype:
            raise TypeError("out must have the dtype of q")
        out_stride = _row_stride("out", out.out, (B, N), (heads, head_dim))
    arr = (ctypes.c_int32 * N)(*[int(x) for x in parent]) if tree_parent is None else None
    return _Plan("mpv_tree_attention", dev.index, _Attention(
        B, N, heads, kv_heads, head_dim, dtype, num_pages, page_size, width, int(window), int(sinks),
        float(head_dim ** -0.5 if scale is None else scale), _row_stride("q", q, (B, N), (heads, head_dim)), kv_stride, out_stride,
        page_stride, slot_stride, arr))


def mpv_verify_chains(tokens, target_probs, draft_probs, uniforms, num_nodes=None, max_depth=None, out=None, stream=None):
    """Verification of drafted chains against the target's probabilities (see include/mpv.h), enqueued on the current (or given)
    torch stream; returns a VerifyResult, as mpv_verify does.

    tokens int32 [B,N], uniforms float32 [B,N], target_probs and draft_probs [B,N,V] (float32, bfloat16 or float16; rows may lie
    further apart than V): CUDA tensors.  draft_probs=None: the drafts are certain (looked up, or greedy).  num_nodes int32 [B]: rows
    of each chain, one more than its drafted tokens.  `out` may be a previous VerifyResult whose buffers are reused."""
    import torch
    if max_depth is None:
        max_depth = out.path_nodes.shape[1] if out is not None else max(1, target_probs.shape[1] - 1)
    key = ("chains", max_depth, _like(tokens), _like(target_probs), _like(draft_probs), _like(uniforms), _like(num_nodes),
           None if out is None else (_like(out.accept_len), _like(out.path_nodes), _like(out.path_tokens), _like(out.bonus_token),
                                     _like(out.counters)))
    plan = _plans.get(key)
    if plan is None:
        plan = _kept(key, _chains_plan(tokens, target_probs, draft_probs, uniforms, num_nodes, max_depth, out))
    if out is None:
        B, i32 = target_probs.shape[0], dict(dtype=torch.int32, device=target_probs.device)
        with _allocating(stream):
            out = VerifyResult(accept_len=torch.empty(B, **i32), path_nodes=torch.empty(B, max_depth, **i32),
                               path_tokens=torch.empty(B, max_depth, **i32), bonus_token=torch.empty(B, **i32), counters=torch.empty(8, **i32))
    bufs = _ChainBuffers(target_probs.data_ptr(), _ptr(draft_probs), tokens.data_ptr(), uniforms.data_ptr(), _ptr(num_nodes),
                         out.accept_len.data_ptr(), out.path_nodes.data_ptr(), out.path_tokens.data_ptr(), out.bonus_token.data_ptr(),
                         out.counters.data_ptr())
    _launch(plan, bufs, out, stream)
    if not target_probs.shape[0]:
        _no_counts(stream, out.counters)
    return out


def _chains_plan(tokens, target_probs, draft_probs, uniforms, num_nodes, max_depth, out):
    import torch
    _int32(max_depth=max_depth)
    if target_probs.dim() != 3:
        raise ValueError("target_probs must be [B,N,V]")
    B, N, V = target_probs.shape
    dev = target_probs.device
    _on_device(dev, target_probs=target_probs, draft_probs=draft_probs)
    if draft_probs is not None and draft_probs.dtype != target_probs.dtype:
        raise TypeError("target and draft probabilities must have the same dtype")
    dtype = _dtype_of(target_probs)
    _whole(dev, torch.int32, tokens=(tokens, (B, N)), num_nodes=(num_nodes, (B,)))
    _whole(dev, torch.float32, uniforms=(uniforms, (B, N)))
    if out is not None:
        _whole(dev, torch.int32, accept_len=(out.accept_len, (B,)), path_nodes=(out.path_nodes, (B, max_depth)),
               path_tokens=(out.path_tokens, (B, max_depth)), bonus_token=(out.bonus_token, (B,)), counters=(out.counters, (8,)))
    return _Plan("mpv_verify_chains", dev.index, _Chains(
        B, N, V, dtype, max_depth, _row_stride("target_probs", target_probs, (B, N), (V,)),
        _row_stride("draft_probs", draft_probs, (B, N), (V,)) if draft_probs is not None else 0))


@dataclass
class TablesResult:
    context_len: "object"       # int32 [B]    tokens in the cache after the call
    free_count: "object"        # int32 [1]
    granted: "object"           # int32 [B]    tokens placed; -1: refused
    slot_map: "object"          # int64, the tensor that was passed
    offsets: "object"           # int32 [B+1]  exclusive sums of the tokens placed
    workspace: Optional["object"] = None
    inplace: bool = False       # context_len and free_count are the tensors that were passed


def mpv_extend_tables(block_table, context_len, new_len, free_pages, free_count, page_size, slot_map, extra=0, inplace=False, out=None,
                      stream=None):
    """Room for new tokens in a paged cache: block tables and slot maps from request lengths (see include/mpv.h), enqueued on the
    current (or given) torch stream; returns a TablesResult.

    block_table int32 [B,table_width] and free_pages int32 [num_pages] are changed in place; context_len int32 [B] and
    free_count int32 [1] are, too, with inplace=True, otherwise their new values are in the result alone.  new_len int32 [B]: tokens to
    place beside `extra`, negative for a finished request.  slot_map int64: [B,n] for a row of slots per request, [n] for all of them
    packed.  `out` may be a previous TablesResult whose buffers are reused (without inplace=True, not those that a caller passed).
    """
    import torch
    # a result's lengths and count are written again unless they are a caller's tensors: those of a call in place, or this call's inputs
    lengths, count = context_len.data_ptr(), free_count.data_ptr()
    after = left = None
    if inplace:
        after, left = context_len, free_count
    elif out is not None and not out.inplace and out.context_len.data_ptr() != lengths and out.free_count.data_ptr() != count:
        after, left = out.context_len, out.free_count
    key = ("tables", page_size, extra, _like(block_table), _like(context_len), _like(new_len), _like(free_pages), _like(free_count),
           _like(slot_map), _like(after), _like(left), None if out is None else (_like(out.granted), _like(out.offsets)))
    plan = _plans.get(key)
    if plan is None:
        plan = _kept(key, _tables_plan(block_table, context_len, new_len, free_pages, free_count, page_size, slot_map, extra, after, left, out))
    if after is None or out is None:
        B, i32 = block_table.shape[0], dict(dtype=torch.int32, device=block_table.device)
        with _allocating(stream):
            if after is None:
                after, left = torch.empty(B, **i32), torch.empty(1, **i32)
            if out is None:
                out = TablesResult(context_len=after, free_count=left, granted=torch.empty(B, **i32), slot_map=slot_map,
                                   offsets=torch.empty(B + 1, **i32))
    out.context_len, out.free_count, out.slot_map, out.inplace = after, left, slot_map, inplace
    bufs = _TableBuffers(new_len.data_ptr(), lengths, block_table.data_ptr(), free_pages.data_ptr(), count, after.data_ptr(), left.data_ptr(),
                         slot_map.data_ptr(), out.granted.data_ptr(), out.offsets.data_ptr())
    _launch(plan, bufs, out, stream)
    if not block_table.shape[0]:                   # the library writes nothing then
        with _allocating(stream):
            left.copy_(free_count.clamp(0, free_pages.shape[0]))
            out.offsets.zero_()
    return out


def _tables_plan(block_table, context_len, new_len, free_pages, free_count, page_size, slot_map, extra, after, left, out):
    import torch
    _int32(page_size=page_size, extra=extra)
    if block_table.dim() != 2 or free_pages.dim() != 1 or slot_map.dim() not in (1, 2):
        raise ValueError("block_table must be [B,table_width], free_pages [num_pages], slot_map [B,n] or [n]")
    B, width = block_table.shape
    dev, pages = block_table.device, free_pages.shape[0]
    packed = slot_map.dim() == 1
    _whole(dev, torch.int32, block_table=(block_table, (B, width)), context_len=(context_len, (B,)), new_len=(new_len, (B,)),
           free_pages=(free_pages, (pages,)), free_count=(free_count, (1,)))
    _whole(dev, torch.int64, slot_map=(slot_map, tuple(slot_map.shape) if packed else (B, slot_map.shape[1])))
    _whole(dev, torch.int32, **{"the result's context_len": (after, (B,)), "the result's free_count": (left, (1,))})
    if out is not None:
        _whole(dev, torch.int32, granted=(out.granted, (B,)), offsets=(out.offsets, (B + 1,)))
    return _Plan("mpv_extend_tables", dev.index, _Tables(B, int(page_size), width, pages, int(extra), int(packed), slot_map.shape[-1]))


def mpv_append_paths(tree_k, tree_v, cache_k, cache_v, slot_map, accept_len, path_nodes=None, stream=None):
    """Moves the keys and values of the root and of the accepted path of every tree into the cache (see include/mpv.h), enqueued
    on the current (or given) torch stream.

    tree_k / tree_v [layers,B,N,kv_heads,head_dim] and cache_k / cache_v [layers,num_pages,page_size,kv_heads,head_dim], or all four
    without the first dimension for one layer; slot_map int64 [B,n]; accept_len int32 [B] and path_nodes int32 [B,max_depth] as a
    verification writes them (path_nodes=None: chains, nodes 1, 2, ...)."""
    key = ("append", _like(tree_k), _like(tree_v), _like(cache_k), _like(cache_v), _like(slot_map), _like(accept_len), _like(path_nodes))
    plan = _plans.get(key)
    if plan is None:
        plan = _kept(key, _append_plan(tree_k, tree_v, cache_k, cache_v, slot_map, accept_len, path_nodes))
    bufs = _AppendBuffers(tree_k.data_ptr(), tree_v.data_ptr(), cache_k.data_ptr(), cache_v.data_ptr(), slot_map.data_ptr(),
                          accept_len.data_ptr(), _ptr(path_nodes))
    _launch(plan, bufs, None, stream)


def _append_plan(tree_k, tree_v, cache_k, cache_v, slot_map, accept_len, path_nodes):
    import torch
    if tree_k.dim() == 4 and cache_k.dim() == 4:
        tree_k, tree_v, cache_k, cache_v = (t.unsqueeze(0) for t in (tree_k, tree_v, cache_k, cache_v))
    if tree_k.dim() != 5 or tree_v.dim() != 5 or cache_k.dim() != 5 or cache_v.dim() != 5 or slot_map.dim() != 2:
        raise ValueError("tree_k, tree_v, cache_k and cache_v must all have a dimension of layers or all have none, slot_map is [B,n]")
    layers, B, N, kv_heads, head_dim = tree_k.shape
    num_pages, page_size = cache_k.shape[1], cache_k.shape[2]
    dev = tree_k.device
    _on_device(dev, tree_k=tree_k, tree_v=tree_v, cache_k=cache_k, cache_v=cache_v)
    if any(t.dtype != tree_k.dtype for t in (tree_v, cache_k, cache_v)):
        raise TypeError("tree_k, tree_v, cache_k and cache_v must have the same dtype")
    dtype = _dtype_of(tree_k)
    if tuple(tree_v.shape) != tuple(tree_k.shape) or tuple(cache_v.shape) != tuple(cache_k.shape) or cache_k.shape[0] != layers:
        raise ValueError("keys and values must have the same shapes, tree and cache the same number of layers")
    deep = path_nodes.shape[1] if path_nodes is not None and path_nodes.dim() == 2 else 0
    _whole(dev, torch.int64, slot_map=(slot_map, (B, slot_map.shape[1])))
    _whole(dev, torch.int32, accept_len=(accept_len, (B,)), path_nodes=(path_nodes, (B, deep)))
    shape = _Append(layers, B, N, dtype, kv_heads * head_dim, deep, slot_map.shape[1], num_pages, page_size, 0, 0, 0, 0, 0)
    if layers and B:
        shape.tree_stride = _row_stride("tree_k", tree_k[0], (B, N), (kv_heads, head_dim))
        shape.page_stride, shape.slot_stride = _cache_strides(cache_k[0], cache_v[0], (num_pages, page_size, kv_heads, head_dim))
        if layers > 1:
            shape.tree_layer_stride, shape.cache_layer_stride = tree_k.stride(0), cache_k.stride(0)
        if (_row_stride("tree_v", tree_v[0], (B, N), (kv_heads, head_dim)) != shape.tree_stride
                or (layers > 1 and (tree_v.stride(0) != tree_k.stride(0) or cache_v.stride(0) != cache_k.stride(0)))):
            raise ValueError("keys and values must have the same strides")
    return _Plan("mpv_append_paths", dev.index, shape)


MPV_KERNEL_NAMES = {0: "init", 1: "node_task", 2: "debug_stats"}


def mpv_timing_enable(max_launches):
    """Bracket every kernel of the following mpv_verify calls with HIP events
    (0 turns it off)."""
    rc = load_library().mpv_timing_enable(int(max_launches))
    if rc != 0:
        raise MpvError(rc, "mpv_timing_enable")


def mpv_timing_read(capacity):
    """After synchronising: list of (kernel_id, milliseconds) of the recorded launches."""
    ms = (ctypes.c_float * capacity)()
    ids = (ctypes.c_int32 * capacity)()
    n = ctypes.c_int32(0)
    rc = load_library().mpv_timing_read(ms, ids, capacity, ctypes.byref(n))
    if rc != 0:
        raise MpvError(rc, "mpv_timing_read")
    return [(int(ids[i]), float(ms[i])) for i in range(n.value)]
