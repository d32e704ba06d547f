"""Thin ctypes binding of liblfmmi.so (include/lfmmi.h): argument marshalling
only. Every step of the forward-backward runs in the library's HIP kernels;
there is no CPU fallback, and a missing library is an error.

Functions carry the names of the C entry points. Device arrays are torch
tensors on the GPU (PyTorch only provides device memory and the stream).
"""
from __future__ import annotations

import array
import collections
import contextlib
import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblfmmi.so")

ORD_FWD, ORD_BWD, ORD_OCC = 0, 1, 2

EXPORTS = [
    "lfmmi_graph_create", "lfmmi_graph_pack", "lfmmi_graph_create_batch",
    "lfmmi_graph_pack_batch", "lfmmi_graph_upload", "lfmmi_graph_destroy",
    "lfmmi_forward_backward", "lfmmi_forward_backward_static", "lfmmi_loss", "lfmmi_last_error",
    "lfmmi_graph_info",
    "lfmmi_graph_ordering_info", "lfmmi_graph_ordering_copy",
    "lfmmi_profile_enable", "lfmmi_profile_read",
    "lfmmi_token_logprobs", "lfmmi_token_logprobs_workspace", "lfmmi_token_logprobs_backward",
    "lfmmi_grad_norm", "lfmmi_clip_grads",
]

_lib = None


class LfmmiError(RuntimeError):
    def __init__(self, code, message):
        super().__init__("lfmmi status %d: %s" % (code, message))
        self.code = code


def load_library():
    """Loads the built library; builds it first only if nothing is built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from . import build as _build
        _build.build()
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    pp = ctypes.POINTER(vp)
    single = [i32, i32, i64, vp, vp, vp, vp, vp, vp, pp]
    batch = [i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, pp]
    lib.lfmmi_graph_create.argtypes = single
    lib.lfmmi_graph_pack.argtypes = single
    lib.lfmmi_graph_create_batch.argtypes = batch
    lib.lfmmi_graph_pack_batch.argtypes = batch
    lib.lfmmi_graph_upload.argtypes = [vp]
    lib.lfmmi_graph_destroy.argtypes = [vp]
    lib.lfmmi_graph_destroy.restype = None
    lib.lfmmi_forward_backward.argtypes = [vp, vp, vp, i32, i32, i32, f32, f32,
                                           ctypes.c_int, vp, vp, vp, vp]
    lib.lfmmi_forward_backward_static.argtypes = lib.lfmmi_forward_backward.argtypes
    lib.lfmmi_loss.argtypes = [vp, vp, vp, vp, i32, i32, i32, f32, vp, vp, vp, vp]
    lib.lfmmi_last_error.argtypes = []
    lib.lfmmi_last_error.restype = ctypes.c_char_p
    lib.lfmmi_graph_info.argtypes = [vp, vp]
    lib.lfmmi_graph_ordering_info.argtypes = [vp, i32, i32, vp]
    lib.lfmmi_graph_ordering_copy.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.lfmmi_profile_enable.argtypes = [vp, ctypes.c_int]
    lib.lfmmi_profile_read.argtypes = [vp, vp, vp, vp]
    lib.lfmmi_token_logprobs.argtypes = [vp, i32, i32, i32, i32, i64, i64, vp, vp, i32, f32, i32,
                                         vp, vp, vp, vp, vp, vp, vp, i64, vp]
    lib.lfmmi_token_logprobs_workspace.argtypes = [i32, i32, i32, i32, i32, vp]
    lib.lfmmi_token_logprobs_backward.argtypes = [vp, i32, i32, i32, i32, i64, i64, vp, vp, i32, f32,
                                                  vp, vp, vp, vp, vp, vp]
    lib.lfmmi_grad_norm.argtypes = [i32, vp, vp, vp, vp, vp, i64, vp]
    lib.lfmmi_clip_grads.argtypes = [i32, vp, vp, vp, vp, f32, vp, vp, i64, vp]
    for name in EXPORTS:
        if name not in ("lfmmi_graph_destroy", "lfmmi_last_error"):
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _check(code):
    if code != 0:
        raise LfmmiError(code, lfmmi_last_error())


def lfmmi_last_error():
    return load_library().lfmmi_last_error().decode("utf-8", "replace")


def _host(arr, dtype):
    return np.ascontiguousarray(arr, dtype=dtype)


def _hp(arr):
    return ctypes.c_void_p(arr.ctypes.data) if arr is not None and arr.size else None


class Graph:
    """Owner of an lfmmi_graph handle."""

    def __init__(self, handle, num_graphs, num_pdfs):
        self.handle = handle
        self.num_graphs = num_graphs
        self.num_pdfs = num_pdfs

    def close(self):
        if self.handle:
            lfmmi_graph_destroy(self)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _single(fn_name, g):
    lib = load_library()
    src, dst, pdf = (_host(g[k], np.int32) for k in ("src", "dst", "pdf"))
    logw = _host(g["logw"], np.float32)
    pi = _host(g["init_prob"], np.float32)
    fin = _host(g["final_prob"], np.float32)
    S, P = int(g["num_states"]), int(g["num_pdfs"])
    if not (len(src) == len(dst) == len(pdf) == len(logw)):
        raise ValueError("arc arrays differ in length")
    if len(pi) != S or len(fin) != S:
        raise ValueError("init_prob / final_prob must have num_states entries")
    out = ctypes.c_void_p()
    _check(getattr(lib, fn_name)(S, P, len(src), _hp(src), _hp(dst), _hp(pdf), _hp(logw),
                                 _hp(pi), _hp(fin), ctypes.byref(out)))
    return Graph(out.value, 1, P)


def _batch(fn_name, graphs):
    lib = load_library()
    n = len(graphs)
    P = int(graphs[0]["num_pdfs"])
    for g in graphs:
        if int(g["num_pdfs"]) != P:
            raise ValueError("graphs of a batch must share num_pdfs")
        if len(g["init_prob"]) != int(g["num_states"]) or \
                len(g["final_prob"]) != int(g["num_states"]):
            raise ValueError("init_prob / final_prob must have num_states entries")
    state_off = np.zeros(n + 1, dtype=np.int64)
    arc_off = np.zeros(n + 1, dtype=np.int64)
    for i, g in enumerate(graphs):
        state_off[i + 1] = state_off[i] + int(g["num_states"])
        arc_off[i + 1] = arc_off[i] + len(g["src"])
    cat = lambda k, dt: _host(np.concatenate([np.asarray(g[k]) for g in graphs]), dt)
    src, dst, pdf = cat("src", np.int32), cat("dst", np.int32), cat("pdf", np.int32)
    logw = cat("logw", np.float32)
    pi, fin = cat("init_prob", np.float32), cat("final_prob", np.float32)
    out = ctypes.c_void_p()
    _check(getattr(lib, fn_name)(n, P, _hp(state_off), _hp(arc_off), _hp(src), _hp(dst),
                                 _hp(pdf), _hp(logw), _hp(pi), _hp(fin), ctypes.byref(out)))
    return Graph(out.value, n, P)


def lfmmi_graph_create(graph):
    """Pack one graph (dict of arrays) and upload it to the current device."""
    return _single("lfmmi_graph_create", graph)


def lfmmi_graph_pack(graph):
    """Host-only packing, for inspection."""
    return _single("lfmmi_graph_pack", graph)


def lfmmi_graph_create_batch(graphs):
    return _batch("lfmmi_graph_create_batch", graphs)


def lfmmi_graph_pack_batch(graphs):
    return _batch("lfmmi_graph_pack_batch", graphs)


def lfmmi_graph_upload(graph):
    _check(load_library().lfmmi_graph_upload(graph.handle))


def lfmmi_graph_destroy(graph):
    if graph.handle:
        load_library().lfmmi_graph_destroy(graph.handle)
        graph.handle = None


def lfmmi_graph_info(graph):
    info = np.zeros(8, dtype=np.int64)
    _check(load_library().lfmmi_graph_info(graph.handle, _hp(info)))
    keys = ("num_graphs", "num_pdfs", "total_states", "total_arcs", "rec_waves",
            "occ_waves", "flags", "workspace_bytes")
    out = dict(zip(keys, (int(v) for v in info)))
    out["uploaded"] = out["flags"] & 1
    out["fp64"] = (out["flags"] >> 1) & 1
    out["emission_by_state"] = (out["flags"] >> 2) & 1
    return out


def lfmmi_graph_ordering_info(graph, g, ord_):
    info = np.zeros(12, dtype=np.int64)
    _check(load_library().lfmmi_graph_ordering_info(graph.handle, g, ord_, _hp(info)))
    keys = ("rows", "slices", "waves", "total_slots", "max_wave_slots", "register_slots",
            "emission_replicated", "per_arc_leak", "gather_cycles", "closing_slots", "hub_slices",
            "lds_vector_rows")
    return dict(zip(keys, (int(v) for v in info)))


def lfmmi_graph_ordering_copy(graph, g, ord_):
    info = lfmmi_graph_ordering_info(graph, g, ord_)
    slice_off = np.zeros(info["slices"] + 1, dtype=np.int32)
    wave_first = np.zeros(info["waves"] + 1, dtype=np.int32)
    key = np.zeros(info["total_slots"] * 64, dtype=np.uint32)
    w = np.zeros(info["total_slots"] * 64, dtype=np.float32)
    row_id = np.zeros(info["slices"] * 64, dtype=np.int32)
    slice_hub = np.zeros(info["slices"], dtype=np.int32)
    _check(load_library().lfmmi_graph_ordering_copy(
        graph.handle, g, ord_, _hp(slice_off), _hp(wave_first), _hp(key), _hp(w), _hp(row_id),
        _hp(slice_hub)))
    return dict(info, slice_off=slice_off, wave_first=wave_first, key=key, w=w, row_id=row_id,
                slice_hub=slice_hub)


STATIC_WORKSPACE_BYTES = 64 << 20   # LFMMI_STATIC_WORKSPACE_BYTES
STATIC_MAX_BATCH = 256              # LFMMI_STATIC_MAX_BATCH


def lfmmi_forward_backward_static(graph, logits, lengths, leak, grad_scale, accumulate,
                                  objf, grad, status, stream=None):
    """The entry point that allocates nothing: as lfmmi_forward_backward, with the
    outputs passed in (this wrapper allocates nothing either) and the workspace
    in the library's static device array."""
    return lfmmi_forward_backward(graph, logits, lengths, leak, grad_scale, accumulate,
                                  objf, grad, status, stream,
                                  _entry="lfmmi_forward_backward_static")


def lfmmi_forward_backward(graph, logits, lengths, leak, grad_scale=1.0, accumulate=False,
                           objf=None, grad=None, status=None, stream=None,
                           _entry="lfmmi_forward_backward"):
    """logits: torch float32 CUDA tensor [B, T, P]; lengths: host int array [B].
    Returns (objf [B], grad [B, T, P], status [B]) device tensors (allocated here
    unless passed in). Enqueues on `stream` (default: torch's current stream)."""
    import torch
    if not logits.is_cuda or logits.dtype != torch.float32 or not logits.is_contiguous():
        raise ValueError("logits must be a contiguous float32 CUDA tensor")
    B, T, P = logits.shape
    lens = _host(lengths, np.int32)
    if len(lens) != B:
        raise ValueError("lengths must have B entries")
    dev = logits.device
    if objf is None:
        if accumulate:
            raise ValueError("accumulate needs existing objf / grad")
        objf = torch.empty(B, dtype=torch.float32, device=dev)
    if grad is None:
        if accumulate:
            raise ValueError("accumulate needs existing objf / grad")
        grad = torch.empty((B, T, P), dtype=torch.float32, device=dev)
    if status is None:
        status = torch.zeros(B, dtype=torch.int32, device=dev)
    for t, shape, dt in ((objf, (B,), torch.float32), (grad, (B, T, P), torch.float32),
                         (status, (B,), torch.int32)):
        if tuple(t.shape) != shape or t.dtype != dt or not t.is_contiguous() or t.device != dev:
            raise ValueError("output tensor has the wrong shape, dtype, layout or device")
    if stream is None:
        stream = torch.cuda.current_stream(dev).cuda_stream
    with torch.cuda.device(dev):
        _check(getattr(load_library(), _entry)(
            graph.handle, ctypes.c_void_p(logits.data_ptr()), _hp(lens), B, T, P,
            float(leak), float(grad_scale), 1 if accumulate else 0,
            ctypes.c_void_p(objf.data_ptr()), ctypes.c_void_p(grad.data_ptr()),
            ctypes.c_void_p(status.data_ptr()), ctypes.c_void_p(stream)))
    return objf, grad, status


def lfmmi_loss(num, den, logits, lengths, leak, objf=None, grad=None, status=None, stream=None):
    """Eq. 2 / Eq. 3 in one call: objf = log p(num) - log p(den) per sequence and its
    gradient with respect to `logits` (torch float32 CUDA tensor [B, T, P]).
    Returns (objf [B], grad [B, T, P], status [B]) device tensors."""
    import torch
    if not logits.is_cuda or logits.dtype != torch.float32 or not logits.is_contiguous():
        raise ValueError("logits must be a contiguous float32 CUDA tensor")
    B, T, P = logits.shape
    lens = _host(lengths, np.int32)
    if len(lens) != B:
        raise ValueError("lengths must have B entries")
    dev = logits.device
    if objf is None:
        objf = torch.empty(B, dtype=torch.float32, device=dev)
    if grad is None:
        grad = torch.empty((B, T, P), dtype=torch.float32, device=dev)
    if status is None:
        status = torch.zeros(B, dtype=torch.int32, device=dev)
    for t, shape, dt in ((objf, (B,), torch.float32), (grad, (B, T, P), torch.float32),
                         (status, (B,), torch.int32)):
        if tuple(t.shape) != shape or t.dtype != dt or not t.is_contiguous() or t.device != dev:
            raise ValueError("output tensor has the wrong shape, dtype, layout or device")
    if stream is None:
        stream = torch.cuda.current_stream(dev).cuda_stream
    with torch.cuda.device(dev):
        _check(load_library().lfmmi_loss(
            num.handle, den.handle, ctypes.c_void_p(logits.data_ptr()), _hp(lens), B, T, P,
            float(leak), ctypes.c_void_p(objf.data_ptr()), ctypes.c_void_p(grad.data_ptr()),
            ctypes.c_void_p(status.data_ptr()), ctypes.c_void_p(stream)))
    return objf, grad, status


def lfmmi_profile_enable(graph, enable=True):
    """enable: False / 0 off, True / 1 every kernel, 2 the recursion launches only."""
    _check(load_library().lfmmi_profile_enable(graph.handle, int(enable)))


def lfmmi_profile_read(graph):
    ms = np.zeros(4, dtype=np.float32)
    calls = np.zeros(1, dtype=np.int32)
    launches = np.zeros(1, dtype=np.int32)
    _check(load_library().lfmmi_profile_read(graph.handle, _hp(ms), _hp(calls), _hp(launches)))
    out = dict(zip(("emit", "rec", "scan", "occ"), (float(v) for v in ms)))
    out["calls"] = int(calls[0])
    out["launches"] = int(launches[0])
    return out


MAX_TOP = 64   # LFMMI_MAX_TOP

TokenLogprobs = collections.namedtuple(
    "TokenLogprobs", ["logp", "entropy", "stats", "top_id", "top_logp", "status"])

_NO_CONTEXT = contextlib.nullcontext()
_dtypes = None


def _dtype_codes():
    """lfmmi_dtype of each torch dtype that the library takes."""
    global _dtypes
    if _dtypes is None:
        import torch
        _dtypes = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    return _dtypes


def _on_stream(dev, stream):
    """(context, raw stream): inside the context `dev` is the current device and torch takes
    memory that belongs to `stream` (torch's current stream if None), which may run
    beside torch's current one."""
    import torch
    if stream is None:
        here = torch.cuda.current_device() == dev.index
        return (_NO_CONTEXT if here else torch.cuda.device(dev)), torch.cuda.current_stream(dev.index).cuda_stream
    own = torch.cuda.ExternalStream(stream, device=dev) if stream else torch.cuda.default_stream(dev)
    return torch.cuda.stream(own), stream


def _written(tensors):
    """Tells autograd that the caller's `tensors` have new values, as torch's own operations in
    place do: a graph that has saved one of them then refuses its backward pass."""
    import torch
    torch.autograd.graph.increment_version(tensors)


def _logit_rows(logits, targets, lengths):
    """Checked (dtype code, B, T, V, stride_b, stride_t, lengths, target bytes) of logits
    [B, T, V] or [B, V]."""
    import torch
    code = _dtype_codes().get(logits.dtype)
    if not logits.is_cuda or code is None or logits.dim() not in (2, 3):
        raise ValueError("logits must be a float32, bfloat16 or float16 CUDA tensor [B, T, V] or [B, V]")
    shape = logits.shape
    V = shape[-1]
    if V < 1:
        raise ValueError("logits need at least one column")
    if logits.dim() == 3:
        (B, T), (stride_b, stride_t, step) = shape[:2], logits.stride()
    else:
        B, T = shape[0], 1
        stride_b, step = logits.stride()
        stride_t = V
    if step != 1 and V > 1:
        raise ValueError("the logits of a row must be next to each other")
    if B * T >= 1 << 31 or V > 1 << 30:   # (ctypes would pass on the lowest 32 bits)
        raise ValueError("too many rows or columns")
    bytes_ = 0
    if targets is not None:
        if targets.dtype == torch.int64:
            bytes_ = 8
        elif targets.dtype == torch.int32:
            bytes_ = 4
        else:
            raise ValueError("targets must be int32 or int64")
        if targets.shape != shape[:-1] or targets.device != logits.device or not targets.is_contiguous():
            raise ValueError("targets must be contiguous, on the logits' device, one for each row")
    lens = None
    if lengths is not None:
        lens = _host(lengths, np.int32)
        if lens.shape != (B,):
            raise ValueError("lengths must have B entries")
    return code, B, T, V, stride_b, stride_t, lens, bytes_


def _ptr(t):
    return None if t is None else t.data_ptr()


def lfmmi_token_logprobs(logits, targets=None, lengths=None, top_k=0, scale=1.0, entropy=True,
                         out=None, stream=None):
    """Log probabilities of given tokens, entropies and the top_k best alternatives of rows of
    logits: a float32, bfloat16 or float16 CUDA tensor [B, T, V] or [B, V], any strides as
    long as a row's logits are next to each other. targets: int32 or int64 CUDA tensor
    [B, T] or [B] (negative: the row is not scored), or None; lengths: host int array
    [B] or None. Returns a TokenLogprobs (logp, entropy, stats, top_id, top_logp, status) of
    device tensors; logp is None without targets, entropy where it is not asked for, top_id and
    top_logp where top_k is 0. `out`: a TokenLogprobs of an earlier call of the same shapes, to
    write into. Enqueues on `stream` (default: torch's current stream)."""
    import torch
    code, B, T, V, stride_b, stride_t, lens, target_bytes = _logit_rows(logits, targets, lengths)
    dev = logits.device
    rows = tuple(logits.shape[:-1])
    top_k = int(top_k)
    context, raw = _on_stream(dev, stream)
    lib = load_library()
    mine = out is None
    with context:
        if mine:
            f32, i32 = torch.float32, torch.int32
            if not 0 <= top_k <= MAX_TOP:
                raise ValueError("top_k outside [0, MAX_TOP]")
            out = TokenLogprobs(
                None if targets is None else torch.empty(rows, dtype=f32, device=dev),
                torch.empty(rows, dtype=f32, device=dev) if entropy else None,
                torch.empty(rows + (2,), dtype=f32, device=dev),
                torch.empty(rows + (top_k,), dtype=i32, device=dev) if top_k else None,
                torch.empty(rows + (top_k,), dtype=f32, device=dev) if top_k else None,
                torch.empty(rows, dtype=i32, device=dev))
        else:
            for t, wanted, shape, dt in (
                    (out.logp, targets is not None, rows, torch.float32),
                    (out.entropy, entropy, rows, torch.float32),
                    (out.stats, True, rows + (2,), torch.float32),
                    (out.top_id, top_k > 0, rows + (top_k,), torch.int32),
                    (out.top_logp, top_k > 0, rows + (top_k,), torch.float32),
                    (out.status, True, rows, torch.int32)):
                if (t is not None) != bool(wanted) or wanted and (
                        tuple(t.shape) != shape or t.dtype != dt or not t.is_contiguous() or t.device != dev):
                    raise ValueError("output tensor has the wrong shape, dtype, layout or device")
        need = ctypes.c_int64(0)
        _check(lib.lfmmi_token_logprobs_workspace(code, B, T, V, top_k, ctypes.byref(need)))
        ws = torch.empty(need.value, dtype=torch.uint8, device=dev) if need.value else None
        _check(lib.lfmmi_token_logprobs(
            logits.data_ptr(), code, B, T, V, stride_b, stride_t, None if lens is None else _hp(lens),
            _ptr(targets), target_bytes, scale, top_k, _ptr(out.logp), _ptr(out.entropy),
            _ptr(out.stats), _ptr(out.top_id), _ptr(out.top_logp), _ptr(out.status), _ptr(ws),
            need.value, raw))
    if not mine:
        _written([t for t in out if t is not None])
    return out


def lfmmi_token_logprobs_backward(logits, targets, stats, entropy, grad_logp=None,
                                  grad_entropy=None, lengths=None, scale=1.0, grad=None,
                                  stream=None):
    """Gradient with respect to `logits` of a loss whose gradients with respect to the log
    probabilities and entropies of lfmmi_token_logprobs are grad_logp and grad_entropy
    (float32 [B, T] or [B]; None: zero). stats and entropy: what that call returned. `grad`: a
    contiguous tensor like logits to write into, the logits themselves if they are contiguous.
    Returns the gradient."""
    import torch
    code, B, T, V, stride_b, stride_t, lens, target_bytes = _logit_rows(logits, targets, lengths)
    dev = logits.device
    rows = tuple(logits.shape[:-1])
    for t, shape in ((stats, rows + (2,)), (entropy, rows), (grad_logp, rows), (grad_entropy, rows)):
        if t is not None and (tuple(t.shape) != shape or t.dtype != torch.float32 or
                              not t.is_contiguous() or t.device != dev):
            raise ValueError("stats, entropy or a gradient has the wrong shape, dtype, layout or device")
    context, raw = _on_stream(dev, stream)
    mine = grad is None
    with context:
        if mine:
            grad = torch.empty(logits.shape, dtype=logits.dtype, device=dev)
        elif grad.shape != logits.shape or grad.dtype != logits.dtype or not grad.is_contiguous() \
                or grad.device != dev:
            raise ValueError("output tensor has the wrong shape, dtype, layout or device")
        _check(load_library().lfmmi_token_logprobs_backward(
            logits.data_ptr(), code, B, T, V, stride_b, stride_t, None if lens is None else _hp(lens),
            _ptr(targets), target_bytes, scale, _ptr(stats), _ptr(entropy), _ptr(grad_logp),
            _ptr(grad_entropy), grad.data_ptr(), raw))
    if not mine:
        _written(grad)
    return grad


def _dense(t):
    """Whether the values of `t` fill a stretch of memory, each once (in any order)."""
    if t.is_contiguous():
        return True
    step = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != step:
            return False
        step *= size
    return True


def _alike(a, b):
    """Whether the values of two tensors of as many lie in the same order."""
    if a.is_contiguous() and b.is_contiguous():
        return True
    return a.shape == b.shape and all(p == q for p, q, n in zip(a.stride(), b.stride(), a.shape) if n != 1)


def _described(tensors):
    """(devices, dtypes, numbers of values, whether all are contiguous) of tensors: an attribute at a
    time, which takes half the time of a tensor at a time."""
    return ([t.get_device() for t in tensors], [t.dtype for t in tensors], [t.numel() for t in tensors],
            all([t.is_contiguous() for t in tensors]))


def _grad_arrays(grads, out):
    """Checked host arrays (pointers, output pointers or None, counts, dtype codes) of gradient
    tensors of one device and tensors laid out as they are."""
    devices, dtypes, counts, plain = _described(grads)
    codes = list(map(_dtype_codes().get, dtypes))
    if devices[0] < 0 or None in codes or devices.count(devices[0]) != len(grads):
        raise ValueError("gradients must be float32, bfloat16 or float16 tensors on one CUDA device")
    if not plain and not all([_dense(g) for g in grads]):
        raise ValueError("gradients must fill their memory: contiguous, or a permutation of that")
    outs = None
    if out is not None:
        if len(out) != len(grads):
            raise ValueError("out must have one tensor for each gradient")
        out_devices, out_dtypes, out_counts, out_plain = _described(out)
        # (of contiguous ones the number of values says it all)
        if out_devices != devices or out_dtypes != dtypes or out_counts != counts or \
                not (plain and out_plain) and not all([_alike(o, g) for o, g in zip(out, grads)]):
            raise ValueError("output tensor has the wrong shape, dtype, layout or device")
        outs = array.array("Q", [o.data_ptr() for o in out])
    return (array.array("Q", [g.data_ptr() for g in grads]), outs, array.array("q", counts),
            array.array("i", codes))


def _at(values):
    return values.buffer_info()[0]


def _grad_workspace(n, dev):
    import torch
    size = 16384 + 32 * (n + 1)   # LFMMI_GRAD_WORKSPACE_BYTES(n)
    return torch.empty(size, dtype=torch.uint8, device=dev), size


def lfmmi_grad_norm(grads, norm=None, stream=None):
    """Norm of the gradient tensors `grads` (a list, of float32, bfloat16 and float16 CUDA
    tensors of one device) taken together: a float32 device tensor of no dimensions."""
    return _grads_call(grads, None, None, norm, stream)


def lfmmi_clip_grads(grads, max_norm, out=None, norm=None, stream=None):
    """Scales the gradient tensors `grads` so that their norm, taken together, is at most
    max_norm: in place, or into the tensors `out` (of the same sizes, layouts and dtypes).
    Gradients whose norm is not finite become 0. Returns the norm they had, a float32 device
    tensor of no dimensions."""
    return _grads_call(grads, float(max_norm), out, norm, stream)


def _grads_call(grads, max_norm, out, norm, stream):
    import torch
    grads = list(grads)
    if not grads:
        raise ValueError("no gradients")
    if out is not None:
        out = list(out)
    n = len(grads)
    pointers, outs, counts, codes = _grad_arrays(grads, out)
    dev = grads[0].device
    if norm is not None and (norm.numel() != 1 or norm.dtype != torch.float32 or norm.device != dev):
        raise ValueError("output tensor has the wrong shape, dtype, layout or device")
    context, raw = _on_stream(dev, stream)
    lib = load_library()
    written = [] if norm is None else [norm]
    with context:
        if norm is None:
            norm = torch.empty((), dtype=torch.float32, device=dev)
        ws, size = _grad_workspace(n, dev)
        if max_norm is None:
            _check(lib.lfmmi_grad_norm(n, _at(pointers), _at(counts), _at(codes), norm.data_ptr(),
                                       ws.data_ptr(), size, raw))
        else:
            _check(lib.lfmmi_clip_grads(n, _at(pointers), None if outs is None else _at(outs), _at(counts),
                                        _at(codes), max_norm, norm.data_ptr(), ws.data_ptr(), size, raw))
            written += grads if out is None else out
    if written:
        _written(written)
    return norm
