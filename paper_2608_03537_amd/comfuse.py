"""Thin Python binding of libcomfuse (ctypes).

Argument marshalling only: every step of every operator runs in the HIP
kernels of ``libcomfuse.so``.  torch supplies device memory and streams.
If the library is missing, every call raises — there is no fallback path.

The raw entry points keep the C names (``cf_gemm_postnorm`` ...) and take the
ctypes structures below; the ``gemm_postnorm`` / ``gemm_subgraph`` / ``b2b_*``
/ ``gemm`` / ``rowop`` helpers build those structures from torch tensors and
allocate the outputs.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
import threading

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcomfuse.so")

# ---------------------------------------------------------------- enums
CF_F32, CF_BF16, CF_FP8_E4M3, CF_I8, CF_I4, CF_FP4_E2M1 = 0, 1, 2, 3, 4, 5
CF_LAYOUT_KN, CF_LAYOUT_NK = 0, 1
(CF_N_SCALE, CF_N_BIAS, CF_N_RESIDUAL, CF_N_LAYERNORM, CF_N_RMSNORM, CF_N_GELU,
 CF_N_GELU_TANH, CF_N_RELU, CF_N_STORE, CF_N_ROWAMAX_QUANT, CF_N_SOFTMAX, CF_N_SOFTCAP) = range(12)
CF_MID_GELU_BIAS, CF_MID_SOFTMAX, CF_MID_RELU_BIAS = 0, 1, 2
CF_OUT_STORE, CF_OUT_BIAS_RESIDUAL_LN, CF_OUT_BIAS_RELU = 0, 1, 2
CF_ACT_NONE, CF_ACT_GELU, CF_ACT_GELU_TANH, CF_ACT_RELU = 0, 1, 2, 3
CF_PAIRS_HALVES, CF_PAIRS_NEIGHBOURS = 0, 1
PATH_AUTO, PATH_WHOLE_ROW, PATH_CLUSTER, PATH_SPLIT = 0, 1, 2, 3
CF_WS_HEADER_BYTES = 8916992       # zero-filled start of a row workspace
CF_WS_OPTIONAL_BYTES = 8917008     # a workspace query's answer where the workspace may be left out
CF_PREFIX_WS_HEADER_BYTES = 1 << 18   # arrival counters at the start of attention_prefix's workspace
CF_PAGED_WS_HEADER_BYTES = 1 << 18    # ... of attention_paged's
CF_B2B_WS_HEADER_BYTES = 1 << 20   # split-MLP arrival counters at the start of its workspace
STATUS = {0: "CF_OK", 1: "CF_ERR_NULL", 2: "CF_ERR_SHAPE", 3: "CF_ERR_LD", 4: "CF_ERR_ALIGN",
          5: "CF_ERR_DTYPE", 6: "CF_ERR_WORKSPACE", 7: "CF_ERR_UNSUPPORTED", 8: "CF_ERR_ALIAS",
          9: "CF_ERR_HIP", 10: "CF_ERR_STRUCT", 11: "CF_ERR_PEER_TIMEOUT"}

vp, i64, f32p = C.c_void_p, C.c_int64, C.POINTER(C.c_float)


class PostnormArgs(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("M", i64), ("N", i64), ("K", i64),
                ("in_dtype", C.c_int), ("out_dtype", C.c_int),
                ("X", vp), ("ldx", i64), ("W", vp), ("ldw", i64), ("w_layout", C.c_int),
                ("bias", vp), ("R", vp), ("ldr", i64), ("gamma", vp), ("beta", vp),
                ("alpha", C.c_float), ("eps", C.c_float), ("Y", vp), ("ldy", i64), ("path", C.c_int)]


class Node(C.Structure):
    _fields_ = [("kind", C.c_int), ("inp", vp), ("out", vp), ("out2", vp), ("ld", i64),
                ("dtype", C.c_int), ("v0", vp), ("v1", vp), ("f0", C.c_float)]


class SubgraphArgs(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("M", i64), ("N", i64), ("K", i64), ("in_dtype", C.c_int),
                ("X", vp), ("ldx", i64), ("W", vp), ("ldw", i64), ("w_layout", C.c_int),
                ("nodes", C.POINTER(Node)), ("n_nodes", C.c_int), ("path", C.c_int)]


class B2BArgs(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("batch", i64), ("M", i64), ("K", i64), ("N1", i64), ("N2", i64),
                ("dtype", C.c_int),
                ("X", vp), ("ldx", i64), ("sx", i64),
                ("W1", vp), ("ldw1", i64), ("sw1", i64), ("w1_layout", C.c_int), ("b1", vp),
                ("mid", C.c_int), ("mid_scale", C.c_float),
                ("W2", vp), ("ldw2", i64), ("sw2", i64), ("w2_layout", C.c_int),
                ("out", C.c_int), ("b2", vp), ("R", vp), ("ldr", i64), ("sr", i64),
                ("gamma", vp), ("beta", vp), ("eps", C.c_float),
                ("O", vp), ("ldo", i64), ("so", i64)]


class RmsnormQuantArgs(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("M", i64), ("N", i64), ("dtype", C.c_int), ("X", vp), ("ldx", i64),
                ("R", vp), ("ldr", i64), ("H", vp), ("ldh", i64), ("gamma", vp), ("norm", C.c_int),
                ("eps", C.c_float), ("code_dtype", C.c_int), ("Q", vp), ("ldq", i64), ("s", vp)]


class GemmI8Args(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("M", i64), ("N", i64), ("K", i64), ("A", vp), ("lda", i64),
                ("B", vp), ("ldb", i64), ("sa", vp), ("sb", vp), ("bias", vp), ("act", C.c_int),
                ("out_dtype", C.c_int), ("C", vp), ("ldc", i64)]


class AttentionPrefixArgs(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("batch", i64), ("H", i64), ("Hk", i64), ("Lq", i64), ("P", i64),
                ("S", i64), ("d", i64), ("dtype", C.c_int),
                ("Q", vp), ("q_b", i64), ("q_h", i64), ("q_l", i64),
                ("Kp", vp), ("kp_h", i64), ("kp_l", i64), ("Vp", vp), ("vp_h", i64), ("vp_l", i64),
                ("Ks", vp), ("ks_b", i64), ("ks_h", i64), ("ks_l", i64),
                ("Vs", vp), ("vs_b", i64), ("vs_h", i64), ("vs_l", i64),
                ("lens", vp), ("causal", C.c_int), ("scale", C.c_float),
                ("O", vp), ("o_b", i64), ("o_h", i64), ("o_l", i64)]


class W4QuantArgs(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("N", i64), ("K", i64), ("group", i64), ("dtype", C.c_int), ("W", vp),
                ("ldw", i64), ("w_dtype", C.c_int), ("tiles", vp), ("s_dtype", C.c_int), ("s", vp), ("lds", i64)]


class GemmW4Args(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("M", i64), ("N", i64), ("K", i64), ("group", i64), ("A", vp), ("lda", i64),
                ("w_dtype", C.c_int), ("W", vp), ("s_dtype", C.c_int), ("s", vp), ("lds", i64), ("bias", vp),
                ("act", C.c_int), ("out_dtype", C.c_int), ("C", vp), ("ldc", i64)]


# cf_cache, a member of the structures below
_CACHE_FIELDS = [("code_dtype", C.c_int), ("n_pages", i64), ("page", i64),
                 ("cK", vp), ("ck_p", i64), ("ck_h", i64), ("ck_l", i64), ("cV", vp), ("cv_p", i64), ("cv_h", i64),
                 ("cv_l", i64), ("cKs", vp), ("cks_p", i64), ("cks_h", i64), ("cVs", vp), ("cvs_p", i64), ("cvs_h", i64)]


class CacheWriteArgs(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("T", i64), ("H", i64), ("Hk", i64), ("d", i64),
                ("Q", vp), ("q_t", i64), ("q_h", i64), ("Qo", vp), ("qo_t", i64), ("qo_h", i64),
                ("K", vp), ("k_t", i64), ("k_h", i64), ("V", vp), ("v_t", i64), ("v_h", i64), ("slots", vp),
                ("rot", i64), ("pairs", C.c_int), ("pos", vp), ("ldpos", i64), ("freq", vp), ("n_axes", i64),
                ("section0", i64), ("section1", i64), ("section2", i64), ("section3", i64)] + _CACHE_FIELDS


class CacheReadArgs(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("batch", i64), ("Hk", i64), ("S", i64), ("d", i64)] + _CACHE_FIELDS + [
                ("table", vp), ("ldt", i64), ("pages", i64), ("lens", vp),
                ("K", vp), ("k_b", i64), ("k_h", i64), ("k_l", i64), ("V", vp), ("v_b", i64), ("v_h", i64), ("v_l", i64)]


class AttentionPagedArgs(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("batch", i64), ("H", i64), ("Hk", i64), ("Lq", i64), ("d", i64),
                ("Q", vp), ("q_b", i64), ("q_h", i64), ("q_l", i64)] + _CACHE_FIELDS + [
                ("table", vp), ("ldt", i64), ("pages", i64), ("lens", vp), ("causal", C.c_int), ("scale", C.c_float),
                ("softcap", C.c_float), ("O", vp), ("o_b", i64), ("o_h", i64), ("o_l", i64)]


class CfError(RuntimeError):
    def __init__(self, status, detail):
        self.status = status
        super().__init__(f"{STATUS.get(status, status)}: {detail}")


_lib = None
_lib_lock = threading.Lock()


def lib():
    """Load libcomfuse.so from the package directory (raises if missing)."""
    global _lib
    if _lib is None:
        with _lib_lock:
            if _lib is None:
                if not os.path.exists(LIB_PATH):
                    raise RuntimeError(f"libcomfuse.so not built ({LIB_PATH}); run paper_2608_03537_amd/build.py")
                L = C.CDLL(LIB_PATH)
                L.cf_version.restype = C.c_int
                L.cf_last_error.restype = C.c_char_p
                L.cf_status_string.restype = C.c_char_p
                L.cf_status_string.argtypes = [C.c_int]
                for name, argt in [("cf_gemm_postnorm", C.POINTER(PostnormArgs)),
                                   ("cf_gemm_subgraph", C.POINTER(SubgraphArgs)),
                                   ("cf_b2bgemm", C.POINTER(B2BArgs))]:
                    f = getattr(L, name)
                    f.restype = C.c_int
                    f.argtypes = [argt, vp, C.c_size_t, vp]
                    w = getattr(L, name.replace("cf_b2bgemm", "cf_b2bgemm") + "_workspace")
                    w.restype = C.c_size_t
                    w.argtypes = [argt]
                L.cf_gemm.restype = C.c_int
                L.cf_gemm.argtypes = [i64, i64, i64, i64, C.c_int, C.c_int, vp, i64, i64, vp, i64, i64,
                                      C.c_int, vp, C.c_float, vp, i64, i64, vp]
                L.cf_rowop.restype = C.c_int
                L.cf_rowop.argtypes = [i64, i64, i64, C.c_int, vp, i64, i64, C.POINTER(Node), C.c_int, vp]
                L.cf_gemm_subgraph_noalloc.restype = C.c_int
                L.cf_gemm_subgraph_noalloc.argtypes = [C.POINTER(SubgraphArgs), vp]
                for name, ws in [("cf_rmsnorm_quant", False), ("cf_gemm_i8", False), ("cf_attention_prefix", True),
                                 ("cf_w4_quant", False), ("cf_gemm_w4", False), ("cf_cache_write", False),
                                 ("cf_cache_read", False), ("cf_attention_paged", True)]:
                    f = getattr(L, name)
                    f.restype = C.c_int
                    f.argtypes = [vp, vp, C.c_size_t, vp] if ws else [vp, vp]   # arguments: byref or packed bytes
                L.cf_w4_pack.restype = C.c_int
                L.cf_w4_pack.argtypes = [i64, i64, vp, i64, vp, vp]
                for name in ("cf_gemm_i8_form", "cf_attention_prefix_form", "cf_gemm_w4_form", "cf_attention_paged_form"):
                    getattr(L, name).restype = C.c_char_p
                    getattr(L, name).argtypes = [vp]
                for name in ("cf_attention_prefix_workspace", "cf_attention_paged_workspace"):
                    getattr(L, name).restype = C.c_size_t
                    getattr(L, name).argtypes = [vp]
                L.cf_workspace_check.restype = C.c_int
                L.cf_workspace_check.argtypes = [vp, C.c_size_t, vp]
                _lib = L
    return _lib


def _check(status):
    if status != 0:
        raise CfError(status, lib().cf_last_error().decode())


# ---------------------------------------------------------------- raw C names
def cf_version():
    return lib().cf_version()


def cf_gemm_postnorm(args, workspace, ws_bytes, stream):
    return lib().cf_gemm_postnorm(C.byref(args), workspace, ws_bytes, stream)


def cf_gemm_postnorm_workspace(args):
    return lib().cf_gemm_postnorm_workspace(C.byref(args))


def cf_gemm_subgraph(args, workspace, ws_bytes, stream):
    return lib().cf_gemm_subgraph(C.byref(args), workspace, ws_bytes, stream)


def cf_gemm_subgraph_workspace(args):
    return lib().cf_gemm_subgraph_workspace(C.byref(args))


def cf_gemm_subgraph_noalloc(args, stream):
    return lib().cf_gemm_subgraph_noalloc(C.byref(args), stream)


def cf_b2bgemm(args, workspace, ws_bytes, stream):
    return lib().cf_b2bgemm(C.byref(args), workspace, ws_bytes, stream)


def cf_b2bgemm_workspace(args):
    return lib().cf_b2bgemm_workspace(C.byref(args))


def cf_gemm(*args):
    return lib().cf_gemm(*args)


def cf_rowop(batch, M, N, dtype, P, ldp, sp, nodes, n_nodes, stream):
    return lib().cf_rowop(batch, M, N, dtype, P, ldp, sp, nodes, n_nodes, stream)


def cf_rmsnorm_quant(args, stream):
    return lib().cf_rmsnorm_quant(C.byref(args), stream)


def cf_gemm_i8(args, stream):
    return lib().cf_gemm_i8(C.byref(args), stream)


def cf_gemm_i8_form(args):
    return lib().cf_gemm_i8_form(C.byref(args)).decode()


def cf_attention_prefix(args, workspace, ws_bytes, stream):
    return lib().cf_attention_prefix(C.byref(args), workspace, ws_bytes, stream)


def cf_attention_prefix_workspace(args):
    return lib().cf_attention_prefix_workspace(C.byref(args))


def cf_attention_prefix_form(args):
    return lib().cf_attention_prefix_form(C.byref(args)).decode()


def cf_w4_quant(args, stream):
    return lib().cf_w4_quant(C.byref(args), stream)


def cf_w4_pack(*args):
    return lib().cf_w4_pack(*args)


def cf_gemm_w4(args, stream):
    return lib().cf_gemm_w4(C.byref(args), stream)


def cf_gemm_w4_form(args):
    return lib().cf_gemm_w4_form(C.byref(args)).decode()


def cf_cache_write(args, stream):
    return lib().cf_cache_write(C.byref(args), stream)


def cf_cache_read(args, stream):
    return lib().cf_cache_read(C.byref(args), stream)


def cf_attention_paged(args, workspace, ws_bytes, stream):
    return lib().cf_attention_paged(C.byref(args), workspace, ws_bytes, stream)


def cf_attention_paged_workspace(args):
    return lib().cf_attention_paged_workspace(C.byref(args))


def cf_attention_paged_form(args):
    return lib().cf_attention_paged_form(C.byref(args)).decode()


def cf_workspace_check(workspace, ws_bytes, stream):
    return lib().cf_workspace_check(workspace, ws_bytes, stream)


def cf_status_string(s):
    return lib().cf_status_string(s).decode()


def cf_last_error():
    return lib().cf_last_error().decode()


# ---------------------------------------------------------------- torch helpers
def _torch():
    import torch
    return torch


def _dt(t):
    torch = _torch()
    if t.dtype == torch.float32:
        return CF_F32
    if t.dtype == torch.bfloat16:
        return CF_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _ld(t):
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("expected a 2-D tensor with unit column stride")
    return t.stride(0)


def _stream(stream):
    torch = _torch()
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


_ws_cache: dict = {}   # (device, stream, kind) -> workspace of eager calls
_ws_graph: dict = {}   # the same -> (capture, workspace) of the last capture


def _capturing():
    return _torch().cuda.is_current_stream_capturing()


def _capture_id(stream):
    """Number of the graph capture that ``stream`` takes part in, or None."""
    status, number = C.c_int(), C.c_ulonglong()
    e = lib().hipStreamGetCaptureInfo(C.c_void_p(_stream(stream)), C.byref(status), C.byref(number))
    return number.value if e == 0 and status.value == 1 else None


def _graph_workspace(nbytes, key, device, stream):
    """The workspace of the capture in progress: allocated in it, so that the
    graph owns the memory, and its header zero-filled by the graph's first
    node that uses it, so that no replay depends on what ran before."""
    torch = _torch()
    capture = _capture_id(stream)
    have = _ws_graph.get(key)
    if have is None or capture is None or have[0] != capture or have[1].numel() < nbytes:
        header = {"rows": CF_WS_HEADER_BYTES, "b2b": CF_B2B_WS_HEADER_BYTES, "prefix": CF_PREFIX_WS_HEADER_BYTES,
                  "paged": CF_PAGED_WS_HEADER_BYTES}[key[2]]
        with torch.cuda.stream(stream):
            ws = torch.empty(max(nbytes, header), dtype=torch.uint8, device=device)
            ws[:header].view(torch.int32).zero_()
        have = _ws_graph[key] = (capture, ws)
    return have[1]


def workspace(nbytes, device, stream=None, kind="rows"):
    """A zero-initialised workspace of at least nbytes on ``device``, cached per
    (device, stream, kind): calls on one stream run in order, so they may
    share it; calls on different streams get different workspaces (the
    row-cluster round counters live in it).  kind "b2b" is that of the split
    MLP and of attention with split keys (their arrival counters must not meet
    another entry point's data), "prefix" that of attention_prefix and "paged" that of
    attention_paged, for the same reason.  Calls captured into a graph share one of the
    capture's own, never an eager one: a graph outlives what the cache holds,
    and its replays may overlap eager calls or another graph."""
    torch = _torch()
    if nbytes == 0:
        return None
    key = (str(device), _stream(stream), kind)
    if _capturing():
        return _graph_workspace(nbytes, key, device, stream)
    ws = _ws_cache.get(key)
    if ws is None or ws.numel() < nbytes:
        # made on the stream that will use it, so the zero-fill runs before the call
        with torch.cuda.stream(stream):
            ws = torch.zeros(max(nbytes, 1 << 20), dtype=torch.uint8, device=device)
        _ws_cache[key] = ws
    return ws


def check_workspace(ws, stream=None):
    """Raise CfError(CF_ERR_PEER_TIMEOUT) if a row-cluster wait gave up since
    the last check of ``ws`` (synchronises the stream; clears the word)."""
    if ws is not None:
        _check(cf_workspace_check(_ptr(ws), ws.numel(), _stream(stream)))


def _row_workspace(ws, need, device, stream, check):
    """The workspace to pass for a row call whose query answered ``need``.  An
    optional one is left out where using it would make the call synchronise
    (``check``), and in a graph capture unless the caller gives it: the graph
    outlives what the cache holds (a larger call replaces it)."""
    if need == CF_WS_OPTIONAL_BYTES and (check or (ws is None and _capturing())):
        return None
    return workspace(need, device, stream) if ws is None else ws


def _after_call(ws, need, stream, check):
    # The error word exists only when the plan used a workspace; checking
    # synchronises, so it is skipped while a graph is being captured (the
    # caller then checks after replaying, with check_workspace).
    if check and need > 0 and need != CF_WS_OPTIONAL_BYTES and not _capturing():
        check_workspace(ws, stream)


def postnorm_args(X, W, bias=None, R=None, gamma=None, beta=None, Y=None, *, w_layout=CF_LAYOUT_NK,
                  alpha=1.0, eps=1e-5, path=PATH_AUTO):
    M, K = X.shape
    N = W.shape[0] if w_layout == CF_LAYOUT_NK else W.shape[1]
    a = PostnormArgs()
    a.struct_size = C.sizeof(PostnormArgs)
    a.M, a.N, a.K = M, N, K
    a.in_dtype = _dt(X)
    a.out_dtype = _dt(Y)
    a.X, a.ldx = _ptr(X), _ld(X)
    a.W, a.ldw, a.w_layout = _ptr(W), _ld(W), w_layout
    a.bias, a.gamma, a.beta = _ptr(bias), _ptr(gamma), _ptr(beta)
    a.R, a.ldr = _ptr(R), (_ld(R) if R is not None else 0)
    a.alpha, a.eps = alpha, eps
    a.Y, a.ldy = _ptr(Y), _ld(Y)
    a.path = path
    return a


def gemm_postnorm(X, W, bias=None, R=None, gamma=None, beta=None, *, w_layout=CF_LAYOUT_NK, alpha=1.0,
                  eps=1e-5, out_dtype=None, path=PATH_AUTO, out=None, ws=None, stream=None, check=True):
    """Y = LayerNorm(alpha * X.W + bias + R) * gamma + beta, fused.

    check=True reads the workspace's error word after the call (a stream
    synchronisation) and raises if a row-cluster wait gave up; pass
    check=False to keep the call asynchronous and use check_workspace later.
    Where the workspace is optional (a query answers CF_WS_OPTIONAL_BYTES:
    narrow rows), check=True runs on whole rows, without the synchronisation
    and without a workspace, also if one is given; only check=False takes the
    row clusters (128 x 256 x 256 in fp32 14.9 us against 6.8).
    """
    torch = _torch()
    M = X.shape[0]
    N = W.shape[0] if w_layout == CF_LAYOUT_NK else W.shape[1]
    Y = out if out is not None else torch.empty((M, N), dtype=out_dtype or X.dtype, device=X.device)
    a = postnorm_args(X, W, bias, R, gamma, beta, Y, w_layout=w_layout, alpha=alpha, eps=eps, path=path)
    need = cf_gemm_postnorm_workspace(a)
    ws = _row_workspace(ws, need, X.device, stream, check)
    _check(cf_gemm_postnorm(a, _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)))
    _after_call(ws, need, stream, check)
    return Y


def make_nodes(spec):
    """spec: list of dicts {kind, in, out, out2, ld, dtype, v0, v1, f0} (tensors allowed)."""
    arr = (Node * len(spec))()
    for i, d in enumerate(spec):
        n = arr[i]
        n.kind = d["kind"]
        for src, dst in (("in", "inp"), ("out", "out"), ("out2", "out2"), ("v0", "v0"), ("v1", "v1")):
            v = d.get(src)
            setattr(n, dst, v.data_ptr() if hasattr(v, "data_ptr") else v)
        n.ld = d.get("ld", 0)
        n.dtype = d.get("dtype", CF_F32)
        n.f0 = d.get("f0", 0.0)
    return arr


def subgraph_args(X, W, nodes, *, w_layout=CF_LAYOUT_NK, path=PATH_AUTO):
    M, K = X.shape
    N = W.shape[0] if w_layout == CF_LAYOUT_NK else W.shape[1]
    a = SubgraphArgs()
    a.struct_size = C.sizeof(SubgraphArgs)
    a.M, a.N, a.K = M, N, K
    a.in_dtype = _dt(X)
    a.X, a.ldx = _ptr(X), _ld(X)
    a.W, a.ldw, a.w_layout = _ptr(W), _ld(W), w_layout
    a.nodes, a.n_nodes = nodes, len(nodes)
    a.path = path
    return a


def gemm_subgraph(X, W, spec, *, w_layout=CF_LAYOUT_NK, path=PATH_AUTO, ws=None, stream=None, check=True):
    """Run X.W followed by the node list ``spec`` (outputs are given in spec).
    ``check`` as in gemm_postnorm."""
    nodes = make_nodes(spec)
    a = subgraph_args(X, W, nodes, w_layout=w_layout, path=path)
    need = cf_gemm_subgraph_workspace(a)
    ws = _row_workspace(ws, need, X.device, stream, check)
    _check(cf_gemm_subgraph(a, _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)))
    _after_call(ws, need, stream, check)


def gemm_subgraph_noalloc(X, W, spec, *, w_layout=CF_LAYOUT_NK, path=PATH_AUTO, stream=None):
    """gemm_subgraph without a workspace: the library's own per-GPU scratch
    array serves the split path (no allocation anywhere; calls on one GPU
    must not overlap)."""
    nodes = make_nodes(spec)
    a = subgraph_args(X, W, nodes, w_layout=w_layout, path=path)
    _check(cf_gemm_subgraph_noalloc(a, _stream(stream)))


def ln_gelu_amax(X, W, bias=None, R=None, *, eps=1e-5, qmax=448.0, z_dtype=None, quant_codes=True,
                 w_layout=CF_LAYOUT_NK, path=PATH_AUTO, ws=None, stream=None, gelu=CF_N_GELU, check=True):
    """Z = GELU(LN(X.W + b + R)); s = rowmax|Z| / qmax; Q = e4m3(Z / s).  Returns (Z, s, Q)."""
    torch = _torch()
    M = X.shape[0]
    N = W.shape[0] if w_layout == CF_LAYOUT_NK else W.shape[1]
    Z = torch.empty((M, N), dtype=z_dtype or X.dtype, device=X.device)
    s = torch.empty((M,), dtype=torch.float32, device=X.device)
    Q = torch.empty((M, N), dtype=torch.uint8, device=X.device) if quant_codes else None
    spec = []
    if bias is not None:
        spec.append(dict(kind=CF_N_BIAS, v0=bias))
    if R is not None:
        spec.append(dict(kind=CF_N_RESIDUAL, **{"in": R}, ld=_ld(R), dtype=_dt(R)))
    spec += [dict(kind=CF_N_LAYERNORM, f0=eps), dict(kind=gelu),
             dict(kind=CF_N_STORE, out=Z, ld=_ld(Z), dtype=_dt(Z)),
             dict(kind=CF_N_ROWAMAX_QUANT, out=s, out2=Q, ld=(N if Q is None else _ld(Q)), f0=qmax)]
    gemm_subgraph(X, W, spec, w_layout=w_layout, path=path, ws=ws, stream=stream, check=check)
    return Z, s, Q


def gemm(A, B, *, b_layout=CF_LAYOUT_NK, bias=None, alpha=1.0, out_dtype=None, out=None, stream=None):
    """C = alpha * A.B (+ bias).  A: [M,K] or [b,M,K]; B: [N,K] (NK) or [K,N] (KN), optionally batched."""
    torch = _torch()
    batched = A.dim() == 3
    A3 = A if batched else A.unsqueeze(0)
    B3 = B if B.dim() == 3 else B.unsqueeze(0)
    nb, M, K = A3.shape
    N = B3.shape[1] if b_layout == CF_LAYOUT_NK else B3.shape[2]
    Cm = out if out is not None else torch.empty((nb, M, N), dtype=out_dtype or A.dtype, device=A.device)
    C3 = Cm if Cm.dim() == 3 else Cm.unsqueeze(0)
    sb = B3.stride(0) if B3.shape[0] > 1 else 0
    _check(cf_gemm(nb, M, N, K, _dt(A3), _dt(C3), _ptr(A3), A3.stride(1), A3.stride(0), _ptr(B3), B3.stride(1), sb,
                   b_layout, _ptr(bias), alpha, _ptr(C3), C3.stride(1), C3.stride(0), _stream(stream)))
    return Cm if (batched or out is not None) else Cm[0]


def rowop(P, spec, stream=None):
    """Run a node list over the rows of a materialised matrix P (unfused).

    P is [M, N] or a batch [b, M, N] (any batch stride, unit column stride);
    the node list's matrices then hold the b * M rows one after another."""
    nodes = make_nodes(spec)
    if P.dim() == 3:
        nb, M, N = P.shape
        if P.stride(2) != 1:
            raise ValueError("expected a unit column stride")
        ldp, sp = P.stride(1), P.stride(0)
    else:
        nb, (M, N) = 1, P.shape
        ldp, sp = _ld(P), 0
    _check(cf_rowop(nb, M, N, _dt(P), _ptr(P), ldp, sp, nodes, len(nodes), _stream(stream)))


def _stack(t, batch=None):
    """(batch, rows, cols, ld, batch stride) of a [rows, cols] or [batch, rows,
    cols] operand with unit column stride.  A 2-D operand beside batched ones
    is shared by every batch entry (stride 0)."""
    if t.dim() == 2:
        return (batch or 1), t.shape[0], t.shape[1], _ld(t), 0
    if t.dim() != 3 or t.stride(2) != 1:
        raise ValueError("expected a 2-D or 3-D tensor with unit column stride")
    if batch is not None and t.shape[0] != batch:
        raise ValueError(f"batch {t.shape[0]} != {batch}")
    return t.shape[0], t.shape[1], t.shape[2], t.stride(1), t.stride(0)


def _b2b_args(**kw):
    a = B2BArgs()
    a.struct_size = C.sizeof(B2BArgs)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def b2b_ffn(X, W1t, b1, W2t, b2=None, R=None, gamma=None, beta=None, *, eps=1e-5, layernorm=True, out=None,
            stream=None):
    """Fused FFN block O = LN(GELU(X W1 + b1) W2 + b2 + R) * gamma + beta.

    X [M, K] bf16; W1t = W1^T [N1, K]; W2t = W2^T [N2, N1]; R [M, N2] (pass X
    for the residual FFN block).  With layernorm=False, O = S W2 (+ b2 + R).
    Batched: X [B, M, K] (and R, out [B, M, N2]); a 3-D weight holds one
    matrix per batch entry, a 2-D one is shared; vectors are shared.
    """
    torch = _torch()
    B, M, K, ldx, sx = _stack(X)
    B = B if X.dim() == 3 else None
    _, N1, _, ldw1, sw1 = _stack(W1t, B)
    _, N2, _, ldw2, sw2 = _stack(W2t, B)
    shape = (M, N2) if B is None else (B, M, N2)
    O = out if out is not None else torch.empty(shape, dtype=torch.bfloat16, device=X.device)
    _, _, _, ldo, so = _stack(O, B)
    ldr, sr = _stack(R, B)[3:] if R is not None else (0, 0)
    a = _b2b_args(batch=B or 1, M=M, K=K, N1=N1, N2=N2, dtype=CF_BF16,
                  X=_ptr(X), ldx=ldx, sx=sx, W1=_ptr(W1t), ldw1=ldw1, sw1=sw1, w1_layout=CF_LAYOUT_NK,
                  b1=_ptr(b1), mid=CF_MID_GELU_BIAS, mid_scale=1.0,
                  W2=_ptr(W2t), ldw2=ldw2, sw2=sw2, w2_layout=CF_LAYOUT_NK,
                  out=CF_OUT_BIAS_RESIDUAL_LN if layernorm else CF_OUT_STORE, b2=_ptr(b2),
                  R=_ptr(R), ldr=ldr, sr=sr,
                  gamma=_ptr(gamma), beta=_ptr(beta), eps=eps, O=_ptr(O), ldo=ldo, so=so)
    _check(cf_b2bgemm(a, None, 0, _stream(stream)))
    return O


def b2b_mlp(X, W1t, b1, W2t, b2=None, *, out_relu=False, out=None, ws=None, stream=None):
    """Fused MLP block O = ReLU(X W1 + b1) W2 + b2 (ReLU(O) with out_relu), the
    DLRM bottom-MLP pattern.  X [M, K] bf16; W1t = W1^T [N1, K]; W2t = W2^T
    [N2, N1]; hidden units in chunks of 256, which may be split over workgroups
    and summed through the workspace while the grid of 128-row blocks and chunks
    fits 256 workgroups, else all run by one workgroup per 128-row block.  Batched as b2b_ffn: X, out [B, M, .],
    weights 3-D (per entry) or 2-D (shared)."""
    torch = _torch()
    B, M, K, ldx, sx = _stack(X)
    B = B if X.dim() == 3 else None
    _, N1, _, ldw1, sw1 = _stack(W1t, B)
    _, N2, _, ldw2, sw2 = _stack(W2t, B)
    shape = (M, N2) if B is None else (B, M, N2)
    O = out if out is not None else torch.empty(shape, dtype=torch.bfloat16, device=X.device)
    _, _, _, ldo, so = _stack(O, B)
    a = _b2b_args(batch=B or 1, M=M, K=K, N1=N1, N2=N2, dtype=CF_BF16,
                  X=_ptr(X), ldx=ldx, sx=sx, W1=_ptr(W1t), ldw1=ldw1, sw1=sw1, w1_layout=CF_LAYOUT_NK,
                  b1=_ptr(b1), mid=CF_MID_RELU_BIAS, mid_scale=1.0,
                  W2=_ptr(W2t), ldw2=ldw2, sw2=sw2, w2_layout=CF_LAYOUT_NK,
                  out=CF_OUT_BIAS_RELU if out_relu else CF_OUT_STORE, b2=_ptr(b2),
                  R=None, ldr=0, sr=0, gamma=None, beta=None, eps=0.0, O=_ptr(O), ldo=ldo, so=so)
    need = cf_b2bgemm_workspace(a)
    if ws is None:
        ws = workspace(need, X.device, stream, kind="b2b")
    _check(cf_b2bgemm(a, _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)))
    return O


def _attention_workspace(a, device, stream):
    """The workspace of a call with few queries (it lets several workgroups
    share a query block's keys), or None: the call then runs without it, as it
    does in a graph capture (the graph outlives what the cache holds: a larger
    call replaces it)."""
    if a.batch * ((a.M + 31) // 32) >= 256:
        return None
    need = cf_b2bgemm_workspace(a)
    if need == 0 or _capturing():
        return None
    return workspace(need, device, stream, kind="b2b")


def b2b_attention(Q, K, V, scale=None, out=None, stream=None, ws=None):
    """O = softmax(scale * Q K^T) V for Q [B, H, Lq, d], K, V [B, H, Lk, d] (bf16, contiguous).

    ws: a workspace of the caller's own, its first CF_B2B_WS_HEADER_BYTES zero,
    for a call with few queries.  Without it an eager call takes a cached one
    and a captured call keeps a query block's keys in one workgroup."""
    torch = _torch()
    B, H, Lq, d = Q.shape
    Lk = K.shape[2]
    if scale is None:
        scale = d ** -0.5
    for t in (Q, K, V):
        if not t.is_contiguous():
            raise ValueError("attention operands must be contiguous [B, H, L, d]")
    O = out if out is not None else torch.empty((B, H, Lq, d), dtype=torch.bfloat16, device=Q.device)
    a = _b2b_args(batch=B * H, M=Lq, K=d, N1=Lk, N2=d, dtype=CF_BF16,
                  X=_ptr(Q), ldx=d, sx=Lq * d, W1=_ptr(K), ldw1=d, sw1=Lk * d, w1_layout=CF_LAYOUT_NK,
                  b1=None, mid=CF_MID_SOFTMAX, mid_scale=scale,
                  W2=_ptr(V), ldw2=d, sw2=Lk * d, w2_layout=CF_LAYOUT_KN,
                  out=CF_OUT_STORE, b2=None, R=None, ldr=0, sr=0, gamma=None, beta=None, eps=0.0,
                  O=_ptr(O), ldo=d, so=Lq * d)
    if ws is None:
        ws = _attention_workspace(a, Q.device, stream)
    _check(cf_b2bgemm(a, _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream)))
    return O


# ---------------------------------------------------------------- 8-bit serving path
# These helpers run on the operands' device, whichever is current, and their new
# tensors belong to the stream that the call uses.  A decoding step makes many
# small calls, so they ask torch for the raw device and stream numbers (a
# torch.cuda.Stream object costs 2.7 us a call) and pack the argument block into
# bytes (0.4 us for attention's 34 fields; a ctypes structure takes 1.4).
def _elsewhere(call, X, stream, *args, **kw):
    """The call with `stream` current (given: of X's device), or with X's device current."""
    torch = _torch()
    if not X.is_cuda:
        raise ValueError(f"expected operands on a GPU, got {X.device}")
    if stream is not None and stream.device != X.device:
        raise ValueError(f"operands on {X.device}, stream of {stream.device}")
    with torch.cuda.stream(stream) if stream is not None else torch.cuda.device(X.device):
        return call(X, *args, **kw)


def _here(X, stream):
    """(library, torch, device index, raw stream) where the call can run on the current device and stream, else None."""
    torch = _torch()
    device = X.get_device()       # -1 on the host
    if stream is not None or device < 0 or device != torch._C._cuda_getDevice():
        return None
    return _lib or lib(), torch, device, torch._C._cuda_getCurrentRawStream(device)


def _rows(torch, M, N, dtype, device, size):
    """A new [M, N] tensor whose rows start every multiple of 16 bytes (`size`: bytes of an element), and its
    leading dimension."""
    if N * size % 16 == 0:
        return torch.empty(M, N, dtype=dtype, device=device), N
    ld = -(-N * size // 16) * 16 // size
    return torch.empty_strided((M, N), (ld, 1), dtype=dtype, device=device), ld


def _row_ld(t, M, N, size):
    """Leading dimension of an [M, N] tensor with unit column stride; a single row's
    is free, and taken as the row rounded up to 16 bytes."""
    s = t.stride()
    if s[1] != 1 and N != 1:
        raise ValueError("expected a 2-D tensor with unit column stride")
    return s[0] if M > 1 else -(-N * size // 16) * 16 // size


def _vector(t, n, f32, device, name):
    """The address of n contiguous fp32 values on `device`."""
    if t.dtype is not f32 or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{name}: expected {n} contiguous fp32 values beside the other operands")
    return t.data_ptr()


def _like(t, shape, dtype, device, name):
    """t, checked to be of a shape and type on `device`."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device:
        raise ValueError(f"{name}: expected {tuple(shape)} of {dtype} beside the other operands, got {tuple(t.shape)} of "
                         f"{t.dtype} on {t.device}")
    return t


def _choice(table, key, name):
    if key not in table:
        raise ValueError(f"{name}: expected one of {', '.join(table)}, got {key!r}")
    return table[key]


_CODES = {"int8": CF_I8, "e4m3": CF_FP8_E4M3}
_FORMATS = {C.c_size_t: "N", i64: "q", C.c_int: "i", C.c_float: "f", vp: "P"}
_RMSNORM_QUANT, _GEMM_I8, _PREFIX = (struct.Struct("@" + "".join(_FORMATS[f] for _, f in t._fields_))
                                     for t in (RmsnormQuantArgs, GemmI8Args, AttentionPrefixArgs))
_RMSNORM_QUANT_SIZE, _GEMM_I8_SIZE, _PREFIX_SIZE = _RMSNORM_QUANT.size, _GEMM_I8.size, _PREFIX.size


def rmsnorm_quant(X, R=None, gamma=None, *, eps=1e-5, norm=True, code="int8", residual=None, out=None, scale=None,
                  stream=None):
    """(Q, s, H): 8-bit codes and row scales of RMSNorm(X + R) * gamma, and H = X + R.

    X, R [M, N] bf16 or fp32, gamma fp32 [N].  Q is int8 [M, N], or uint8 holding
    E4M3 codes (code="e4m3"); s fp32 [M]; Q * s stands for the normed row.
    norm=False quantises the rows as they are.  H is None without R; `residual`
    names the tensor it goes to, which may be R (in place).  `out` and `scale`
    take Q and s.  Q of int8 is what gemm_i8 takes as its tokens, s as sa; E4M3
    codes are for a product of the caller's own.

    Rows start every multiple of 16 bytes, here and in gemm_i8: a width of whole
    16 bytes, or rows that are padded to it (views of wider tensors).  Other
    tensors are refused (CF_ERR_ALIGN), also as outputs.  New outputs of other
    widths are views of padded rows, which these helpers take as they are and
    which are not contiguous: .contiguous() packs them.
    """
    here = _here(X, stream)
    if here is None:
        return _elsewhere(rmsnorm_quant, X, stream, R, gamma, eps=eps, norm=norm, code=code, residual=residual, out=out,
                          scale=scale)
    L, torch, device, raw = here
    shape, dtype, dev, f32 = X.shape, X.dtype, X.device, torch.float32
    M, N = shape
    dt, size = (CF_BF16, 2) if dtype is torch.bfloat16 else (_dt(X), 4)
    cdt, qdt = (CF_I8, torch.int8) if code == "int8" else (_choice(_CODES, code, "code"), torch.uint8)
    whole = N * size % 16 == 0    # rows of whole 16 bytes: a contiguous tensor's leading dimension is N
    plain = whole and X.is_contiguous()
    ldx = N if plain else _row_ld(X, M, N, size)
    rp = hp = ldr = ldh = 0
    H = residual
    if R is not None:
        if R.dtype is not dtype or R.shape != shape or R.get_device() != device:
            _like(R, shape, dtype, device, "R")
        rp, ldr = R.data_ptr(), N if whole and R.is_contiguous() else _row_ld(R, M, N, size)
        if H is None:
            H, ldh = (torch.empty_like(X), N) if plain else _rows(torch, M, N, dtype, dev, size)
            hp = H.data_ptr()
    if residual is not None:
        _like(H, shape, dtype, device, "residual")
        hp, ldh = H.data_ptr(), _row_ld(H, M, N, size)
    if out is None:
        Q, ldq = _rows(torch, M, N, qdt, dev, 1)
    else:
        Q = _like(out, shape, qdt, device, "out")
        ldq = _row_ld(Q, M, N, 1)
    s = torch.empty(M, dtype=f32, device=dev) if scale is None else scale
    a = _RMSNORM_QUANT.pack(_RMSNORM_QUANT_SIZE, M, N, dt, X.data_ptr(), ldx, rp, ldr, hp, ldh,
                            0 if gamma is None else _vector(gamma, N, f32, device, "gamma"), 1 if norm else 0, eps, cdt,
                            Q.data_ptr(), ldq, s.data_ptr() if scale is None else _vector(s, M, f32, device, "scale"))
    status = L.cf_rmsnorm_quant(a, raw)
    if status:
        _check(status)
    return Q, s, H


_ACTS = {"none": CF_ACT_NONE, "gelu": CF_ACT_GELU, "gelu_tanh": CF_ACT_GELU_TANH, "relu": CF_ACT_RELU}


def gemm_i8(A, B, sa=None, sb=None, *, bias=None, act="none", out_dtype=None, out=None, stream=None):
    """C = act((A . B^T) * sa[:, None] * sb + bias) of int8 A [M, K] and B [N, K].

    sa fp32 [M] or [M, 1] (a scale per token), sb fp32 [N] (per channel), bias fp32 [N];
    act "none", "gelu", "gelu_tanh" or "relu"; C bf16 (or fp32) [M, N], its rows padded to whole
    16 bytes where N is not (as rmsnorm_quant's outputs).  K is a multiple of 16.
    """
    here = _here(A, stream)
    if here is None:
        return _elsewhere(gemm_i8, A, stream, B, sa, sb, bias=bias, act=act, out_dtype=out_dtype, out=out)
    L, torch, device, raw = here
    i8, f32 = torch.int8, torch.float32
    M, K = A.shape
    N = B.size(0)
    if A.dtype is not i8 or B.dtype is not i8:
        raise TypeError(f"expected int8 operands, got {A.dtype} and {B.dtype}")
    _like(B, (N, K), i8, device, "B")
    if out is None:
        dt = CF_F32 if out_dtype is f32 else CF_BF16
        if dt == CF_BF16 and out_dtype not in (None, torch.bfloat16):
            raise TypeError(f"unsupported dtype {out_dtype}")
        Cm, ldc = _rows(torch, M, N, f32 if dt == CF_F32 else torch.bfloat16, A.device, 4 if dt == CF_F32 else 2)
    else:
        dt, Cm = _dt(out), _like(out, (M, N), out_dtype or out.dtype, device, "out")
        ldc = _row_ld(Cm, M, N, 4 if dt == CF_F32 else 2)
    whole = K % 16 == 0
    a = _GEMM_I8.pack(_GEMM_I8_SIZE, M, N, K,
                      A.data_ptr(), K if whole and A.is_contiguous() else _row_ld(A, M, K, 1),
                      B.data_ptr(), K if whole and B.is_contiguous() else _row_ld(B, N, K, 1),
                      0 if sa is None else _vector(sa, M, f32, device, "sa"),
                      0 if sb is None else _vector(sb, N, f32, device, "sb"),
                      0 if bias is None else _vector(bias, N, f32, device, "bias"),
                      CF_ACT_NONE if act == "none" else _choice(_ACTS, act, "act"), dt, Cm.data_ptr(), ldc)
    status = L.cf_gemm_i8(a, raw)
    if status:
        _check(status)
    return Cm


_CF_ERR_WORKSPACE = 6
_prefix_lock = threading.Lock()   # threads that share a stream share its workspace: a call's launches stay together


def _prefix_workspace(torch, need, device, key):
    """workspace(need, device, kind=key[2]) at less cost: cached per device and stream while nothing is captured.
    A new one is half as large again as the last, so that a batch that grows step by step seldom needs it, and only
    its counters are cleared."""
    if torch._C._cuda_isCurrentStreamCapturing():
        return workspace(need, device, None, kind=key[2])
    ws = _ws_cache.get(key)
    if ws is None or ws.numel() < need:
        size = max(need, 1 << 20 if ws is None else ws.numel() * 3 // 2)
        ws = torch.empty(size, dtype=torch.uint8, device=device)
        ws[:CF_PREFIX_WS_HEADER_BYTES].view(torch.int32).zero_()   # attention_paged's counters are as many
        _ws_cache[key] = ws
    return ws


def attention_prefix(Q, Kp, Vp, Ks=None, Vs=None, lens=None, *, causal=False, scale=None, out=None, ws=None,
                     stream=None):
    """O = softmax(scale * Q [Kp; Ks]^T) [Vp; Vs] for sequences that share the prefix Kp, Vp.

    Q [B, H, Lq, d]; Kp, Vp [Hk, P, d], one copy for the batch; Ks, Vs
    [B, Hk, S, d], of which sequence b uses the first lens[b] (int32 [B] on the
    device; None: all S); bf16, d 64 or 128, H a multiple of Hk, any strides that
    are multiples of 8 elements with unit innermost stride (caches stored
    token-major are passed as transposed views).  causal: query i sees the own
    keys j < lens[b] - (Lq - 1 - i).  A query that sees no key gets 0.  ws: a
    workspace of the caller's own (uint8, cf_attention_prefix_workspace bytes, its first
    CF_PREFIX_WS_HEADER_BYTES zero before its first use).
    """
    here = _here(Q, stream)
    if here is None:
        return _elsewhere(attention_prefix, Q, stream, Kp, Vp, Ks, Vs, lens, causal=causal, scale=scale, out=out, ws=ws)
    L, torch, device, raw = here
    bf16 = torch.bfloat16
    shape = Q.shape
    B, H, Lq, d = shape
    Hk, P = Kp.size(0), Kp.size(1)
    if (Ks is None) != (Vs is None):
        raise ValueError("Ks and Vs come together")
    S = 0 if Ks is None else Ks.size(2)
    # one condition where all is well; else _like names the operand
    pshape, ks, vs = (Hk, P, d), (0, 0, 0, 1), (0, 0, 0, 1)
    if not (Q.dtype is Kp.dtype is Vp.dtype is bf16 and Kp.shape == pshape and Vp.shape == pshape and
            Kp.get_device() == Vp.get_device() == device):
        for t, want, name in ((Q, shape, "Q"), (Kp, pshape, "Kp"), (Vp, pshape, "Vp")):
            _like(t, want, bf16, device, name)
    if Ks is not None:
        oshape = (B, Hk, S, d)
        if not (Ks.dtype is Vs.dtype is bf16 and Ks.shape == oshape and Vs.shape == oshape and
                Ks.get_device() == Vs.get_device() == device):
            _like(Ks, oshape, bf16, device, "Ks")
            _like(Vs, oshape, bf16, device, "Vs")
        ks, vs = Ks.stride(), Vs.stride()
    O = torch.empty_like(Q) if out is None else _like(out, shape, bf16, device, "out")
    q, o, kp, vpr = Q.stride(), O.stride(), Kp.stride(), Vp.stride()
    if not q[3] == o[3] == kp[2] == vpr[2] == ks[3] == vs[3] == 1:
        raise ValueError("expected unit innermost strides")
    if lens is not None:
        _like(lens, (B,), torch.int32, device, "lens")
        if not lens.is_contiguous():
            raise ValueError("lens: expected a contiguous vector")
    a = _PREFIX.pack(_PREFIX_SIZE, B, H, Hk, Lq, P, S, d, CF_BF16, Q.data_ptr(), q[0], q[1], q[2],
                     Kp.data_ptr(), kp[0], kp[1], Vp.data_ptr(), vpr[0], vpr[1],
                     0 if Ks is None else Ks.data_ptr(), ks[0], ks[1], ks[2],
                     0 if Vs is None else Vs.data_ptr(), vs[0], vs[1], vs[2],
                     0 if lens is None else lens.data_ptr(), 1 if causal else 0,
                     d ** -0.5 if scale is None else scale, O.data_ptr(), o[0], o[1], o[2])
    need = 0 if ws is not None else L.cf_attention_prefix_workspace(a)
    if need:
        with _prefix_lock:
            ws = _prefix_workspace(torch, need, Q.device, (device, raw, "prefix"))
            status = L.cf_attention_prefix(a, ws.data_ptr(), ws.numel(), raw)
    elif ws is None:
        status = L.cf_attention_prefix(a, None, 0, raw)
    else:
        if ws.dtype is not torch.uint8 or not ws.is_contiguous() or ws.get_device() != device:
            raise ValueError("ws: expected a contiguous uint8 tensor beside the other operands")
        status = L.cf_attention_prefix(a, ws.data_ptr(), ws.numel(), raw)
    if status:
        _check(status)
    return O


# ---------------------------------------------------------------- 4-bit weights
_CODES4 = {"int4": CF_I4, "e2m1": CF_FP4_E2M1}
_W4_QUANT, _GEMM_W4, _CACHE_WRITE, _CACHE_READ, _PAGED = (
    struct.Struct("@" + "".join(_FORMATS[f] for _, f in t._fields_))
    for t in (W4QuantArgs, GemmW4Args, CacheWriteArgs, CacheReadArgs, AttentionPagedArgs))
_GEMM_W4_SIZE, _CACHE_WRITE_SIZE, _CACHE_READ_SIZE, _PAGED_SIZE = (s.size for s in (_GEMM_W4, _CACHE_WRITE, _CACHE_READ, _PAGED))


def _tiles(N, K):
    return -(-N // 32), -(-K // 64), 1024


def w4_quant(W, group=128, *, code="int4", scales=None, stream=None):
    """(tiles, s): W [N, K] (bf16 or fp32) as 4-bit codes with a scale per channel and `group` k.

    code "int4" (s = max / 7) or "e2m1" (OCP 4-bit floating point, s = max / 6); `group` is a multiple
    of 32 that divides K.  s [K / group, N] is fp32, or of the type `scales`
    (torch.bfloat16: the codes are taken by the rounded scale).  tiles: uint8
    [ceil(N / 32), ceil(K / 64), 1024], as gemm_w4 takes them.  Done once for a weight.
    """
    here = _here(W, stream)
    if here is None:
        return _elsewhere(w4_quant, W, stream, group, code=code, scales=scales)
    L, torch, device, raw = here
    N, K = W.shape
    size = W.element_size()
    sdt = torch.float32 if scales is None else scales
    if sdt not in (torch.float32, torch.bfloat16):
        raise TypeError(f"unsupported dtype {sdt}")
    if group <= 0 or K % group:
        raise ValueError(f"group: expected a divisor of {K}, got {group}")
    w = torch.empty(_tiles(N, K), dtype=torch.uint8, device=W.device)
    s = torch.empty(K // group, N, dtype=sdt, device=W.device)
    a = _W4_QUANT.pack(_W4_QUANT.size, N, K, group, _dt(W), W.data_ptr(), _row_ld(W, N, K, size),
                       _choice(_CODES4, code, "code"), w.data_ptr(), _dt(s), s.data_ptr(), N)
    _check(L.cf_w4_quant(a, raw))
    return w, s


def w4_pack(codes, stream=None):
    """Tiles, as gemm_w4 takes them, of 4-bit codes [N, K / 2] (uint8: k in the low four bits, k + 1 in the
    high ones); K is a multiple of 32.  Done once for a weight."""
    here = _here(codes, stream)
    if here is None:
        return _elsewhere(w4_pack, codes, stream)
    L, torch, device, raw = here
    if codes.dtype is not torch.uint8:
        raise TypeError(f"expected uint8 codes, got {codes.dtype}")
    N, K = codes.size(0), 2 * codes.size(1)
    if codes.stride(1) != 1:
        raise ValueError("expected a 2-D tensor with unit column stride")
    w = torch.empty(_tiles(N, K), dtype=torch.uint8, device=codes.device)
    _check(L.cf_w4_pack(N, K, codes.data_ptr(), codes.stride(0), w.data_ptr(), raw))
    return w


def gemm_w4(A, W, s, *, code="int4", bias=None, act="none", out_dtype=None, out=None, stream=None):
    """C = act(A . w^T + bias) with 4-bit weights w[n, k] = s[k / group, n] * value(code[n, k]).

    A [M, K] bf16; W the tiles of w4_quant or w4_pack; s [K / group, N] bf16 or fp32,
    its rows any distance apart; code "int4" or "e2m1"; bias fp32 [N]; act "none", "gelu",
    "gelu_tanh" or "relu"; C bf16 (or fp32) [M, N], its rows padded to whole 16 bytes where N is not
    (as rmsnorm_quant's outputs).
    """
    here = _here(A, stream)
    if here is None:
        return _elsewhere(gemm_w4, A, stream, W, s, code=code, bias=bias, act=act, out_dtype=out_dtype, out=out)
    L, torch, device, raw = here
    bf16, f32 = torch.bfloat16, torch.float32
    M, K = A.shape
    ng, N = s.shape
    if A.dtype is not bf16:
        raise TypeError(f"expected bf16 tokens, got {A.dtype}")
    if ng == 0 or K % ng:
        raise ValueError(f"s: expected [K / group, N], got {tuple(s.shape)} for K = {K}")
    if W.shape != (-(-N // 32), -(-K // 64), 1024) or W.dtype is not torch.uint8 or W.get_device() != device or not W.is_contiguous():
        _like(W, _tiles(N, K), torch.uint8, device, "W")
        raise ValueError("W: expected contiguous tiles")
    if s.get_device() != device or (s.stride(1) != 1 and N > 1):
        raise ValueError("s: expected rows of unit stride beside the other operands")
    if out is None:
        dt = CF_F32 if out_dtype is f32 else CF_BF16
        if dt == CF_BF16 and out_dtype not in (None, bf16):
            raise TypeError(f"unsupported dtype {out_dtype}")
        Cm, ldc = _rows(torch, M, N, f32 if dt == CF_F32 else bf16, A.device, 4 if dt == CF_F32 else 2)
    else:
        dt, Cm = _dt(out), _like(out, (M, N), out_dtype or out.dtype, device, "out")
        ldc = _row_ld(Cm, M, N, 4 if dt == CF_F32 else 2)
    a = _GEMM_W4.pack(_GEMM_W4_SIZE, M, N, K, K // ng, A.data_ptr(),
                      K if K % 8 == 0 and A.is_contiguous() else _row_ld(A, M, K, 2),
                      _choice(_CODES4, code, "code"), W.data_ptr(), CF_BF16 if s.dtype is bf16 else _dt(s), s.data_ptr(),
                      s.stride(0), 0 if bias is None else _vector(bias, N, f32, device, "bias"),
                      CF_ACT_NONE if act == "none" else _choice(_ACTS, act, "act"), dt, Cm.data_ptr(), ldc)
    status = L.cf_gemm_w4(a, raw)
    if status:
        _check(status)
    return Cm


# ---------------------------------------------------------------- cache of pages
# Kc, Vc [n_pages, Hk, page, d]: bf16, or int8 or E4M3 codes (uint8 or torch.float8_e4m3fn) with fp32 scales Ks,
# Vs [n_pages, Hk, page]; pages of a power of two of 16 to 1024 tokens, d 64 or 128.  Any strides that are multiples of 16
# bytes with unit innermost stride (pages stored token-major are passed as transposed views); the scales of a page's
# tokens lie beside each other.  Slot t is row t % page of page t // page.
def cache_pages(n_pages, Hk, page, d, code="bf16", device="cuda"):
    """(Kc, Vc, Ks, Vs) for a new cache, zero; code "bf16" (Ks, Vs None), "int8" or "e4m3"."""
    torch = _torch()
    dtypes = {"bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.uint8}
    dtype = _choice(dtypes, code, "code")
    rows = [torch.zeros(n_pages, Hk, page, d, dtype=dtype, device=device) for _ in range(2)]
    if code == "bf16":
        return (*rows, None, None)
    return (*rows, *(torch.zeros(n_pages, Hk, page, dtype=torch.float32, device=device) for _ in range(2)))


def _cache(torch, Kc, Vc, Ks, Vs, Hk, d, device):
    """The fields of cf_cache."""
    dtype, shape = Kc.dtype, Kc.shape
    dt = (CF_BF16 if dtype is torch.bfloat16 else CF_I8 if dtype is torch.int8 else
          CF_FP8_E4M3 if dtype in (torch.uint8, torch.float8_e4m3fn) else None)
    if dt is None:
        raise TypeError(f"Kc: expected bf16, int8 or E4M3 pages, got {dtype}")
    if len(shape) != 4 or shape[1] != Hk or shape[3] != d:
        raise ValueError(f"Kc: expected [n_pages, {Hk}, page, {d}], got {tuple(shape)}")
    if Vc.dtype is not dtype or Vc.shape != shape or Kc.get_device() != device or Vc.get_device() != device:
        _like(Kc, shape, dtype, device, "Kc")
        _like(Vc, shape, dtype, device, "Vc")
    k, v = Kc.stride(), Vc.stride()
    if not k[3] == v[3] == 1:
        raise ValueError("expected unit innermost strides")
    if dt == CF_BF16:
        if Ks is not None or Vs is not None:
            raise ValueError("bf16 pages have no scales")
        return dt, shape[0], shape[2], Kc.data_ptr(), k[0], k[1], k[2], Vc.data_ptr(), v[0], v[1], v[2], 0, 0, 0, 0, 0, 0
    if Ks is None or Vs is None:
        raise ValueError("8-bit pages come with the scales Ks and Vs")
    f32 = torch.float32
    if not (Ks.dtype is Vs.dtype is f32 and Ks.shape == Vs.shape == shape[:3] and Ks.get_device() == Vs.get_device() == device):
        _like(Ks, shape[:3], f32, device, "Ks")
        _like(Vs, shape[:3], f32, device, "Vs")
    ks, vs = Ks.stride(), Vs.stride()
    if not ks[2] == vs[2] == 1:
        raise ValueError("expected unit innermost strides")
    return (dt, shape[0], shape[2], Kc.data_ptr(), k[0], k[1], k[2], Vc.data_ptr(), v[0], v[1], v[2],
            Ks.data_ptr(), ks[0], ks[1], Vs.data_ptr(), vs[0], vs[1])


def _ints(t, shape, i32, device, name):
    """The address of int32 values of a shape with unit innermost stride on `device`."""
    if t.dtype is not i32 or t.shape != shape or t.get_device() != device or t.stride(-1) != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: expected int32 {tuple(shape)} with unit innermost stride beside the other operands, got "
                         f"{tuple(t.shape)} of {t.dtype} on {t.device}")
    return t.data_ptr()


_PAIRS = {"halves": CF_PAIRS_HALVES, "neighbours": CF_PAIRS_NEIGHBOURS}


def cache_write(K, V, slots, Kc, Vc, Ks=None, Vs=None, *, q=None, pos=None, freq=None, sections=None, pairs="halves",
                out=None, stream=None):
    """Write the rows K, V [T, Hk, d] of T new tokens (bf16) to slots [T] (int32) of the cache, after rotary
    positions; returns the queries q [T, H, d], rotated as the keys are (None without q).

    A slot outside the cache is padding, and not written; the slots of a call differ.  pos int32
    [T], or [axes, T] where a pair takes its angle from one of up to four axes (time, height, width): the
    first sections[0] pairs from axis 0, the next sections[1] from axis 1.  Pair i turns by pos * freq[i];
    freq fp32 [rot / 2], rot <= d a multiple of 16, elements from rot on stay as they are.  pairs "halves":
    elements i and i + rot / 2; "neighbours": 2 i and 2 i + 1.  Without pos nothing is rotated.
    `out` takes the queries, and may be q (in place).  8-bit codes: see rmsnorm_quant; each row has its scale.
    """
    here = _here(K, stream)
    if here is None:
        return _elsewhere(cache_write, K, stream, V, slots, Kc, Vc, Ks, Vs, q=q, pos=pos, freq=freq, sections=sections,
                          pairs=pairs, out=out)
    L, torch, device, raw = here
    bf16, i32, shape = torch.bfloat16, torch.int32, K.shape
    T, Hk, d = shape
    if not (K.dtype is V.dtype is bf16 and V.shape == shape and V.get_device() == slots.get_device() == device and
            slots.dtype is i32 and slots.shape == (T,) and slots.is_contiguous()):
        _like(K, shape, bf16, device, "K")
        _like(V, shape, bf16, device, "V")
        _ints(slots, (T,), i32, device, "slots")
        if T > 1 and slots.stride(0) != 1:
            raise ValueError("slots: expected a contiguous vector")
    k, v = K.stride(), V.stride()
    H, Q, qp, op, qs, os_ = 0, None, 0, 0, (0, 0, 1), (0, 0, 1)
    if q is not None:
        H = q.size(1)
        if q.dtype is not bf16 or q.get_device() != device or q.shape != (T, H, d):
            _like(q, (T, H, d), bf16, device, "q")
        Q = torch.empty_like(q) if out is None else _like(out, (T, H, d), bf16, device, "out")
        qp, op, qs, os_ = q.data_ptr(), Q.data_ptr(), q.stride(), Q.stride()
    elif out is not None:
        raise ValueError("out comes with q")
    if not k[2] == v[2] == qs[2] == os_[2] == 1:
        raise ValueError("expected unit innermost strides")
    rot = n_axes = ldpos = pp = fp = s0 = s1 = s2 = s3 = 0
    if (pos is None) != (freq is None):
        raise ValueError("pos and freq come together")
    if pos is not None:
        half = freq.numel()
        rot, fp = 2 * half, _vector(freq, half, torch.float32, device, "freq")
        if pos.dim() == 1:
            n_axes, ldpos, s0 = 1, T, half
            pp = _ints(pos, (T,), i32, device, "pos")
        else:
            n_axes, ldpos = pos.size(0), pos.stride(0)
            pp = _ints(pos, (n_axes, T), i32, device, "pos")
        if sections is not None or n_axes > 1:
            if sections is None or len(sections) != n_axes or n_axes > 4:
                raise ValueError(f"sections: expected one for each of up to 4 axes, got {sections}")
            s0, s1, s2, s3 = (*sections, 0, 0, 0)[:4]
        elif n_axes == 1:
            s0 = half
    a = _CACHE_WRITE.pack(_CACHE_WRITE_SIZE, T, H, Hk, d, qp, qs[0], qs[1], op, os_[0], os_[1], K.data_ptr(), k[0], k[1],
                          V.data_ptr(), v[0], v[1], slots.data_ptr(), rot,
                          CF_PAIRS_HALVES if pairs == "halves" else _choice(_PAIRS, pairs, "pairs"), pp, ldpos, fp, n_axes,
                          s0, s1, s2, s3, *_cache(torch, Kc, Vc, Ks, Vs, Hk, d, device))
    status = L.cf_cache_write(a, raw)
    if status:
        _check(status)
    return Q


def cache_read(Kc, Vc, table, lens, Ks=None, Vs=None, *, S=None, out=None, stream=None):
    """(K, V) [B, Hk, S, d] bf16: the first lens[b] rows of each sequence, row j from page table[b, j // page].

    table int32 [B, pages], lens int32 [B].  S: by default what the table's pages hold.  Rows behind lens[b] (and
    of pages that the cache has not) are left as they are in `out`, a pair of tensors, and hold anything in new ones;
    attention_prefix takes K, V and lens as a batch's own keys.
    """
    here = _here(Kc, stream)
    if here is None:
        return _elsewhere(cache_read, Kc, stream, Vc, table, lens, Ks, Vs, S=S, out=out)
    L, torch, device, raw = here
    bf16, i32 = torch.bfloat16, torch.int32
    _, Hk, page, d = Kc.shape
    B, pages = table.shape
    if out is None:
        S = pages * page if S is None else S
        K, V = (torch.empty((B, Hk, S, d), dtype=bf16, device=Kc.device) for _ in range(2))
    else:
        K, V = out
        S = K.size(2) if S is None else S
        shape = (B, Hk, S, d)
        if not (K.dtype is V.dtype is bf16 and K.shape == shape and V.shape == shape and K.get_device() == V.get_device() == device):
            _like(K, shape, bf16, device, "out")
            _like(V, shape, bf16, device, "out")
    k, v = K.stride(), V.stride()
    if not k[3] == v[3] == 1:
        raise ValueError("expected unit innermost strides")
    a = _CACHE_READ.pack(_CACHE_READ_SIZE, B, Hk, S, d, *_cache(torch, Kc, Vc, Ks, Vs, Hk, d, device),
                         _ints(table, (B, pages), i32, device, "table"), table.stride(0), pages, _ints(lens, (B,), i32, device, "lens"),
                         K.data_ptr(), k[0], k[1], k[2], V.data_ptr(), v[0], v[1], v[2])
    status = L.cf_cache_read(a, raw)
    if status:
        _check(status)
    return K, V


def attention_paged(Q, Kc, Vc, table, lens, Ks=None, Vs=None, *, causal=False, scale=None, softcap=0.0, out=None, ws=None,
                    stream=None):
    """O = softmax(cap(scale * Q K^T)) V over the first lens[b] keys of each sequence's pages; cap(x) = softcap *
    tanh(x / softcap), or x where softcap is 0.

    Q [B, H, Lq, d] bf16, Lq up to 64, H a multiple of Hk; table int32 [B, pages], lens int32 [B] (the new tokens
    among them: cache_write comes first).  causal: query i sees the keys j < lens[b] - (Lq - 1 - i).  A
    query that sees no key gets 0; keys of a page that the cache has not are not seen.  ws: a
    workspace of the caller's own (uint8, cf_attention_paged_workspace bytes, its first CF_PAGED_WS_HEADER_BYTES
    zero before its first use).
    """
    here = _here(Q, stream)
    if here is None:
        return _elsewhere(attention_paged, Q, stream, Kc, Vc, table, lens, Ks, Vs, causal=causal, scale=scale,
                          softcap=softcap, out=out, ws=ws)
    L, torch, device, raw = here
    bf16, i32 = torch.bfloat16, torch.int32
    shape = Q.shape
    B, H, Lq, d = shape
    if Q.dtype is not bf16:
        _like(Q, shape, bf16, device, "Q")
    O = torch.empty_like(Q) if out is None else _like(out, shape, bf16, device, "out")
    q, o = Q.stride(), O.stride()
    if not q[3] == o[3] == 1:
        raise ValueError("expected unit innermost strides")
    pages = table.size(1)
    Hk = Kc.size(1)
    a = _PAGED.pack(_PAGED_SIZE, B, H, Hk, Lq, d, Q.data_ptr(), q[0], q[1], q[2],
                    *_cache(torch, Kc, Vc, Ks, Vs, Hk, d, device), _ints(table, (B, pages), i32, device, "table"), table.stride(0), pages,
                    _ints(lens, (B,), i32, device, "lens"), 1 if causal else 0, d ** -0.5 if scale is None else scale, softcap,
                    O.data_ptr(), o[0], o[1], o[2])
    if ws is not None:
        if ws.dtype is not torch.uint8 or not ws.is_contiguous() or ws.get_device() != device:
            raise ValueError("ws: expected a contiguous uint8 tensor beside the other operands")
        status = L.cf_attention_paged(a, ws.data_ptr(), ws.numel(), raw)
    else:
        key = (device, raw, "paged")
        with _prefix_lock:
            # the cached workspace as it is: a call that wants a larger one says so, and has done nothing
            ws = None if torch._C._cuda_isCurrentStreamCapturing() else _ws_cache.get(key)
            status = L.cf_attention_paged(a, None, 0, raw) if ws is None else L.cf_attention_paged(a, ws.data_ptr(), ws.numel(), raw)
            if status == _CF_ERR_WORKSPACE:
                ws = _prefix_workspace(torch, L.cf_attention_paged_workspace(a), Q.device, key)
                status = L.cf_attention_paged(a, ws.data_ptr(), ws.numel(), raw)
    if status:
        _check(status)
    return O
