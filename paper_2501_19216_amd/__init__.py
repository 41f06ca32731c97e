"""Python binding of libe2f, the MI355X Wigner-6j convolution (E2Former,
arXiv 2501.19216).

Argument marshalling only: every step of the layer runs in the HIP kernels
of ``libe2f.so`` through its C ABI (``include/e2f.h``); torch tensors are
used for device memory and the current stream.  The functions carry the
names of the C entry points.  If the library is not built, importing this
package raises: there is no fallback.
"""
from __future__ import annotations

import array
import bisect
import ctypes
import operator
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libe2f.so")

E2F_OK, E2F_EINVAL, E2F_ECAPACITY, E2F_ENOMEM, E2F_EDEVICE, E2F_EUNSUPPORTED = range(6)
E2F_F32, E2F_BF16 = 0, 1
E2F_FORM_AUTO, E2F_FORM_SPLIT, E2F_FORM_FUSED = 0, 1, 2
_FORMS = {"auto": E2F_FORM_AUTO, "split": E2F_FORM_SPLIT, "fused": E2F_FORM_FUSED}
_STATUS = {0: "E2F_OK", 1: "E2F_EINVAL", 2: "E2F_ECAPACITY", 3: "E2F_ENOMEM", 4: "E2F_EDEVICE", 5: "E2F_EUNSUPPORTED"}

# every function declared in include/e2f.h
EXPORTED = ["e2f_create", "e2f_destroy", "e2f_last_error", "e2f_node_tp_dim", "e2f_real_cg", "e2f_knn_graph",
            "e2f_attention_weights", "e2f_recoupling_weight", "e2f_neighbor_list", "e2f_solid_harmonics",
            "e2f_node_tp", "e2f_aggregate_workspace_size", "e2f_aggregate", "e2f_wigner6j_workspace_size", "e2f_wigner6j_workspace_min", "e2f_wigner6j_prepare",
            "e2f_wigner6j_conv_forward", "e2f_wigner6j_conv_forward_noalloc", "e2f_validate_graph", "e2f_wigner6j_conv_forward_dense",
            "e2f_wigner6j_conv_forward_global", "e2f_wigner6j_conv_backward", "e2f_edge_tp_conv_forward",
            "e2f_transpose_graph_workspace_size", "e2f_transpose_graph", "e2f_attention_forward",
            "e2f_attention_backward_workspace_size", "e2f_attention_backward", "e2f_block_norm_forward",
            "e2f_block_norm_workspace_size", "e2f_block_norm_backward", "e2f_grad_norm_workspace_size",
            "e2f_grad_norm", "e2f_grad_clip", "e2f_embedding_forward", "e2f_embedding_backward_workspace_size",
            "e2f_embedding_backward", "e2f_layer_norm_forward", "e2f_layer_norm_workspace_size",
            "e2f_layer_norm_backward", "e2f_orthogonalize_workspace_size", "e2f_orthogonalize", "e2f_profile", "e2f_profile_read", "e2f_last_slices"]


class E2FError(RuntimeError):
    def __init__(self, status: int, where: str, msg: str):
        super().__init__("%s: %s (%s)" % (where, _STATUS.get(status, status), msg))
        self.status = status


class ConvParams(ctypes.Structure):
    _fields_ = [("lmax", ctypes.c_int), ("channels", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("cutoff", ctypes.c_float), ("path_w", ctypes.c_void_p), ("mix_w", ctypes.c_void_p),
                ("mix_dtype", ctypes.c_int), ("tile_side", ctypes.c_float), ("y_norm", ctypes.c_int32),
                ("form", ctypes.c_int32)]


class AttentionParams(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int32), ("k_heads", ctypes.c_int32), ("dk", ctypes.c_int32),
                ("n_rbf", ctypes.c_int32), ("cutoff", ctypes.c_float), ("scale", ctypes.c_float),
                ("cap", ctypes.c_float), ("dtype", ctypes.c_int), ("ldq", ctypes.c_int64), ("ldk", ctypes.c_int64)]


class NormParams(ctypes.Structure):
    _fields_ = [("lmax", ctypes.c_int), ("channels", ctypes.c_int32), ("gates", ctypes.c_int32),
                ("eps", ctypes.c_float), ("dtype", ctypes.c_int), ("post_w", ctypes.c_void_p),
                ("res_scale", ctypes.c_void_p), ("pre_w", ctypes.c_void_p)]


class EmbeddingParams(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_int32), ("channels", ctypes.c_int32), ("lmax", ctypes.c_int),
                ("scale", ctypes.c_float), ("table_dtype", ctypes.c_int), ("dtype", ctypes.c_int),
                ("index_bytes", ctypes.c_int32), ("ld", ctypes.c_int64)]


class LayerNormParams(ctypes.Structure):
    _fields_ = [("lmax", ctypes.c_int), ("channels", ctypes.c_int32), ("eps", ctypes.c_float),
                ("silu", ctypes.c_int32), ("dtype", ctypes.c_int), ("weight", ctypes.c_void_p),
                ("bias", ctypes.c_void_p), ("ldx", ctypes.c_int64)]


class OrthogonalizeParams(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("steps", ctypes.c_int32),
                ("coefs", ctypes.c_void_p), ("eps", ctypes.c_float), ("momentum", ctypes.c_float),
                ("nesterov", ctypes.c_int32), ("scale", ctypes.c_float), ("decay", ctypes.c_float),
                ("grad_dtype", ctypes.c_int), ("dtype", ctypes.c_int)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError("libe2f.so is not built; run `python paper_2501_19216_amd/build_lib.py` "
                          "(or __graft_entry__.build())")
    L = ctypes.CDLL(LIB_PATH)
    i, i32, i64, p, f = ctypes.c_int, ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
    L.e2f_create.argtypes = [i, i, ctypes.POINTER(p)]
    L.e2f_create.restype = i
    L.e2f_destroy.argtypes = [p]
    L.e2f_destroy.restype = None
    L.e2f_last_error.argtypes = []
    L.e2f_last_error.restype = ctypes.c_char_p
    L.e2f_node_tp_dim.argtypes = [i]
    L.e2f_node_tp_dim.restype = i64
    L.e2f_real_cg.argtypes = [i, i, i, p]
    L.e2f_real_cg.restype = i
    L.e2f_recoupling_weight.argtypes = [i, i, i, i, i]
    L.e2f_recoupling_weight.restype = ctypes.c_double
    L.e2f_neighbor_list.argtypes = [p, p, p, i32, f, p, p, i64, ctypes.POINTER(i64), p]
    L.e2f_neighbor_list.restype = i
    L.e2f_knn_graph.argtypes = [p, p, p, i32, i32, p, p, i64, ctypes.POINTER(i64), p]
    L.e2f_knn_graph.restype = i
    L.e2f_attention_weights.argtypes = [p, p, p, p, i32, i32, i32, p, i32, f, p, p, i64, p, p]
    L.e2f_attention_weights.restype = i
    L.e2f_solid_harmonics.argtypes = [p, p, p, p, i32, i, p, p]
    L.e2f_solid_harmonics.restype = i
    L.e2f_node_tp.argtypes = [p, p, p, p, p, i32, i32, i, p, p]
    L.e2f_node_tp.restype = i
    L.e2f_aggregate_workspace_size.argtypes = [p, i32, i64, i32, ctypes.POINTER(ctypes.c_size_t)]
    L.e2f_aggregate_workspace_size.restype = i
    L.e2f_aggregate.argtypes = [p, p, i32, i32, i32, i32, p, p, i64, p, p, p, p, ctypes.c_size_t, p]
    L.e2f_aggregate.restype = i
    L.e2f_last_slices.argtypes = [p, ctypes.POINTER(i64)]
    L.e2f_last_slices.restype = i
    for name in ("e2f_wigner6j_workspace_size", "e2f_wigner6j_workspace_min"):
        fn = getattr(L, name)
        fn.argtypes = [p, ctypes.POINTER(ConvParams), i32, i64, ctypes.POINTER(ctypes.c_size_t)]
        fn.restype = i
    L.e2f_wigner6j_prepare.argtypes = [p, ctypes.POINTER(ConvParams)]
    L.e2f_wigner6j_prepare.restype = i
    L.e2f_validate_graph.argtypes = [p, i32, p, p, i64, ctypes.POINTER(i32), p]
    L.e2f_validate_graph.restype = i
    L.e2f_profile.argtypes = [p, i]
    L.e2f_profile.restype = i
    L.e2f_profile_read.argtypes = [p, ctypes.c_char_p, ctypes.c_size_t]
    L.e2f_profile_read.restype = i
    L.e2f_wigner6j_conv_forward.argtypes = [p, ctypes.POINTER(ConvParams), p, p, p, i32, p, p, i64, p, p, p,
                                            ctypes.c_size_t, p]
    L.e2f_wigner6j_conv_forward.restype = i
    L.e2f_wigner6j_conv_forward_noalloc.argtypes = [p, ctypes.POINTER(ConvParams), p, p, p, i32, p, p, i64, p, p,
                                                    p]
    L.e2f_wigner6j_conv_forward_noalloc.restype = i
    L.e2f_edge_tp_conv_forward.argtypes = [p, ctypes.POINTER(ConvParams), p, p, p, i32, p, p, i64, p, p, p]
    L.e2f_edge_tp_conv_forward.restype = i
    L.e2f_wigner6j_conv_forward_dense.argtypes = [p, ctypes.POINTER(ConvParams), p, p, i32, p, p, p]
    L.e2f_wigner6j_conv_forward_dense.restype = i
    L.e2f_wigner6j_conv_forward_global.argtypes = [p, ctypes.POINTER(ConvParams), p, p, i32, p, p]
    L.e2f_wigner6j_conv_forward_global.restype = i
    L.e2f_wigner6j_conv_backward.argtypes = [p, ctypes.POINTER(ConvParams), p, p, p, p, i32, p, p, i64, p, p, p, p, p]
    L.e2f_wigner6j_conv_backward.restype = i
    sz, psz = ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)
    pa, pn = ctypes.POINTER(AttentionParams), ctypes.POINTER(NormParams)
    pe, pl, po = (ctypes.POINTER(t) for t in (EmbeddingParams, LayerNormParams, OrthogonalizeParams))
    for name, args in (("e2f_transpose_graph_workspace_size", [p, i32, i64, psz]),
                       ("e2f_transpose_graph", [p, i32, p, p, i64, p, p, p, p, sz, p]),
                       ("e2f_attention_forward", [p, pa, p, p, p, p, i32, p, p, p, i64, p, p, p]),
                       ("e2f_attention_backward_workspace_size", [p, pa, i32, i64, psz]),
                       ("e2f_attention_backward", [p, pa, p, p, p, p, i32, p, p, p, i64] + [p] * 11 + [sz, p]),
                       ("e2f_block_norm_forward", [p, pn, p, p, p, i32, p, p, p, p]),
                       ("e2f_block_norm_workspace_size", [p, pn, i32, psz]),
                       ("e2f_block_norm_backward", [p, pn, p, p, p, p, i32] + [p] * 9 + [sz, p]),
                       ("e2f_grad_norm_workspace_size", [p, i32, p, psz]),
                       ("e2f_grad_norm", [p, i32, p, p, p, p, p, p, sz, p]),
                       ("e2f_grad_clip", [p, i32, p, p, p, p, p, f, p]),
                       ("e2f_embedding_forward", [p, pe, p, p, i32, p, p]),
                       ("e2f_embedding_backward_workspace_size", [p, pe, i32, psz]),
                       ("e2f_embedding_backward", [p, pe, p, i32, p, p, p, sz, p]),
                       ("e2f_layer_norm_forward", [p, pl, p, i32, p, p]),
                       ("e2f_layer_norm_workspace_size", [p, pl, i32, psz]),
                       ("e2f_layer_norm_backward", [p, pl, p, i32, p, p, p, p, p, sz, p]),
                       ("e2f_orthogonalize_workspace_size", [p, po, i32, psz]),
                       ("e2f_orthogonalize", [p, po, i32, p, p, p, p, p, p, sz, p])):
        getattr(L, name).argtypes = args
        getattr(L, name).restype = i
    return L


lib = _load()


def _check(st: int, where: str, allow=()):
    if st != E2F_OK and st not in allow:
        raise E2FError(st, where, lib.e2f_last_error().decode())
    return st


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(device=None):
    """The handle of a device's current stream (without a stream object: 0.1 us instead of 2)."""
    if device is not None and not isinstance(device, torch.device):
        device = torch.device(device)
    index = None if device is None else device.index
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if index is None else index))


def _dev(t, dtype, name):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.dtype != dtype or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor" % (name, dtype))
    return t


class Context:
    """Owns an e2f_ctx (coefficient tables) on one device, and the device
    workspace tensor the binding passes to the Wigner-6j forward."""

    def __init__(self, lmax_max: int = 6, device: int | None = 0):
        h = ctypes.c_void_p()
        dev = -1 if device is None else int(device)
        _check(lib.e2f_create(lmax_max, dev, ctypes.byref(h)), "e2f_create")
        self.handle = h
        self.device = dev
        self.lmax_max = lmax_max
        self.workspace = None
        self.stream_workspaces = {}

    def workspace_for(self, nbytes: int, device) -> torch.Tensor:
        """A device buffer of at least nbytes, kept for later calls."""
        if self.workspace is None or self.workspace.numel() < nbytes:
            self.workspace = None
            self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        return self.workspace

    def close(self):
        if self.handle:
            self.workspace = None
            self.stream_workspaces = {}
            lib.e2f_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def e2f_create(lmax_max: int = 6, device: int | None = 0) -> Context:
    return Context(lmax_max, device)


def e2f_destroy(ctx: Context) -> None:
    ctx.close()


def e2f_node_tp_dim(lmax: int) -> int:
    return int(lib.e2f_node_tp_dim(lmax))


def e2f_real_cg(l1: int, l2: int, l3: int):
    import numpy as np
    out = np.zeros((2 * l1 + 1, 2 * l2 + 1, 2 * l3 + 1))
    _check(lib.e2f_real_cg(l1, l2, l3, out.ctypes.data_as(ctypes.c_void_p)), "e2f_real_cg")
    return out


def e2f_recoupling_weight(a: int, b: int, u: int, o: int, d: int) -> float:
    return float(lib.e2f_recoupling_weight(a, b, u, o, d))


def e2f_neighbor_list(ctx: Context, pos: torch.Tensor, cutoff: float, graph_id: torch.Tensor | None = None,
                      row_ptr: torch.Tensor | None = None, col_idx: torch.Tensor | None = None):
    """Radius graph as device CSR (row_ptr int64 [N+1], col_idx int32 [E]).

    With preallocated row_ptr/col_idx large enough, one library call; else a
    size query first."""
    _dev(pos, torch.float32, "pos")
    _dev(graph_id, torch.int32, "graph_id")
    n = pos.shape[0]
    E = ctypes.c_int64(0)
    if row_ptr is not None and col_idx is not None:
        _dev(row_ptr, torch.int64, "row_ptr")
        _dev(col_idx, torch.int32, "col_idx")
        st = _check(lib.e2f_neighbor_list(ctx.handle, _ptr(pos), _ptr(graph_id), n, cutoff, _ptr(row_ptr),
                                          _ptr(col_idx), col_idx.numel(), ctypes.byref(E), _stream(pos.device)),
                    "e2f_neighbor_list", allow=(E2F_ECAPACITY,))
        if st == E2F_OK:
            return row_ptr, col_idx[:E.value]
    row_ptr = torch.empty(n + 1, dtype=torch.int64, device=pos.device)
    _check(lib.e2f_neighbor_list(ctx.handle, _ptr(pos), _ptr(graph_id), n, cutoff, _ptr(row_ptr), None, 0,
                                 ctypes.byref(E), _stream(pos.device)), "e2f_neighbor_list", allow=(E2F_ECAPACITY,))
    col = torch.empty(max(E.value, 1), dtype=torch.int32, device=pos.device)
    _check(lib.e2f_neighbor_list(ctx.handle, _ptr(pos), _ptr(graph_id), n, cutoff, _ptr(row_ptr), _ptr(col),
                                 col.numel(), ctypes.byref(E), _stream(pos.device)), "e2f_neighbor_list")
    return row_ptr, col[:E.value]


def e2f_knn_graph(ctx: Context, pos: torch.Tensor, k: int, graph_id: torch.Tensor | None = None):
    """k-nearest-neighbour graph as device CSR (row_ptr int64 [N+1], col_idx int32 [E])."""
    _dev(pos, torch.float32, "pos")
    _dev(graph_id, torch.int32, "graph_id")
    n = pos.shape[0]
    E = ctypes.c_int64(0)
    row_ptr = torch.empty(n + 1, dtype=torch.int64, device=pos.device)
    _check(lib.e2f_knn_graph(ctx.handle, _ptr(pos), _ptr(graph_id), n, k, _ptr(row_ptr), None, 0, ctypes.byref(E),
                             _stream(pos.device)), "e2f_knn_graph", allow=(E2F_ECAPACITY,))
    col = torch.empty(max(E.value, 1), dtype=torch.int32, device=pos.device)
    _check(lib.e2f_knn_graph(ctx.handle, _ptr(pos), _ptr(graph_id), n, k, _ptr(row_ptr), _ptr(col), col.numel(),
                             ctypes.byref(E), _stream(pos.device)), "e2f_knn_graph")
    return row_ptr, col[:E.value]


def e2f_attention_weights(ctx: Context, pos, row_ptr, col_idx, cutoff: float, q=None, k=None, rbf_w=None,
                          heads: int | None = None, out=None):
    """Attention weights [E, heads] float32: q, k [N, heads, dk] (or None),
    rbf_w [heads, R] (or None)."""
    for t, name in ((pos, "pos"), (q, "q"), (k, "k"), (rbf_w, "rbf_w")):
        _dev(t, torch.float32, name)
    _dev(row_ptr, torch.int64, "row_ptr")
    _dev(col_idx, torch.int32, "col_idx")
    n = pos.shape[0]
    H = heads if heads is not None else (q.shape[1] if q is not None else rbf_w.shape[0])
    dk = 0 if q is None else q.shape[2]
    R = 0 if rbf_w is None else rbf_w.shape[1]
    E = col_idx.numel()
    if out is None:
        out = torch.empty(E, H, dtype=torch.float32, device=pos.device)
    _dev(out, torch.float32, "out")
    _check(lib.e2f_attention_weights(ctx.handle, _ptr(pos), _ptr(q), _ptr(k), n, H, dk, _ptr(rbf_w), R, cutoff,
                                     _ptr(row_ptr), _ptr(col_idx), E, _ptr(out), _stream(pos.device)),
           "e2f_attention_weights")
    return out


def _arg(ctx, t, dtype, shape, name):
    """The address of a contiguous tensor of this type and shape on the context's device (None: NULL)."""
    if t is None:
        return None
    if t.dtype != dtype or t.get_device() != ctx.device or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor on the context's device" % (name, dtype))
    if t.shape != shape:
        raise ValueError("%s must have shape %s" % (name, tuple(shape)))
    return t.data_ptr()


def _fits(*sizes):
    """The C interface's sizes are 32-bit: ctypes would take larger ones modulo 2^32."""
    if max(sizes) > 0x7fffffff:
        raise ValueError("atoms, heads, features and channels must be below 2^31")


def _capturing(device):
    """Whether this device's current stream is (torch asks the current device's)."""
    if torch.cuda.current_device() == device:
        return torch.cuda.is_current_stream_capturing()
    with torch.cuda.device(device):
        return torch.cuda.is_current_stream_capturing()


def _workspace(ctx, workspace, nbytes, device, stream):
    """The caller's workspace, or the context's own for the (current) stream, grown to nbytes."""
    if workspace is None:
        if _capturing(ctx.device):
            raise ValueError("under graph capture the workspace must be given")
        kept = ctx.stream_workspaces.get(stream.value)
        if kept is None or kept.numel() < nbytes:
            ctx.stream_workspaces[stream.value] = kept = None  # (its memory may become the larger one's)
            ctx.stream_workspaces[stream.value] = kept = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        return kept
    if workspace.get_device() != ctx.device or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the context's device")
    return workspace


_DTYPES = {torch.float32: E2F_F32, torch.bfloat16: E2F_BF16}
_SHAPE, _DTYPE = operator.attrgetter("shape"), operator.attrgetter("dtype")


def e2f_transpose_graph(ctx, n, row_ptr, col_idx, workspace=None):
    """The graph by senders: (rowT_ptr int64 [n+1], colT int32 [E], the
    receivers, perm int32 [E], the edges in the graph's own order).  Here and
    below, workspace: a uint8 device tensor, or None: the context's own for the
    current stream, which grows on demand (code under graph capture gives one
    of its own)."""
    E, dev = col_idx.numel(), col_idx.device
    _fits(n)
    rp, ci = _arg(ctx, row_ptr, torch.int64, (n + 1,), "row_ptr"), _arg(ctx, col_idx, torch.int32, (E,), "col_idx")
    b = ctypes.c_size_t(0)
    _check(lib.e2f_transpose_graph_workspace_size(ctx.handle, n, E, ctypes.byref(b)),
           "e2f_transpose_graph_workspace_size")
    stream = _stream(dev)
    workspace = _workspace(ctx, workspace, b.value, dev, stream)
    row_t = torch.empty(n + 1, dtype=torch.int64, device=dev)
    col_t, perm = (torch.empty(E, dtype=torch.int32, device=dev) for _ in range(2))
    _check(lib.e2f_transpose_graph(ctx.handle, n, rp, ci, E, row_t.data_ptr(), col_t.data_ptr(), perm.data_ptr(),
                                   workspace.data_ptr(), workspace.numel(), stream), "e2f_transpose_graph")
    return row_t, col_t, perm


def _features(ctx, t, n, name):
    """dtype, heads, features and elements between atoms of q or k [n, heads, dk] (heads and features packed)."""
    if t.get_device() != ctx.device or t.dtype not in _DTYPES:
        raise ValueError("%s must be a float32 or bfloat16 tensor on the context's device" % name)
    if t.dim() != 3 or t.shape[0] != n:
        raise ValueError("%s must be [n, heads, dk]" % name)
    _, h, d = t.shape
    s0, s1, s2 = t.stride()
    if (d > 1 and s2 != 1) or (h > 1 and s1 != d) or (n > 1 and s0 < h * d):
        raise ValueError("%s must be packed within an atom, with at least heads * dk elements between atoms" % name)
    return _DTYPES[t.dtype], h, d, s0 if n > 1 else 0


def _attention_args(ctx, pos, row_ptr, col_idx, cutoff, q, k, rbf_w, heads, scale, cap, graph_id):
    """The parameters, and the addresses of what both directions read."""
    n, E = pos.shape[0], col_idx.numel()
    if (q is None) != (k is None):
        raise ValueError("q and k go together")
    dt, H, dk, ldq, Hk, ldk = E2F_F32, heads, 0, 0, heads, 0
    if q is not None:
        dt, H, dk, ldq = _features(ctx, q, n, "q")
        dt2, Hk, dk2, ldk = _features(ctx, k, n, "k")
        if dt2 != dt or dk2 != dk:
            raise ValueError("q and k must agree in type and features")
        if heads is not None and heads != H:
            raise ValueError("q must have `heads` heads")
    elif rbf_w is not None:
        H = rbf_w.shape[0] if H is None else H
    if H is None:
        raise ValueError("heads must be given without q and rbf_w")
    R = 0 if rbf_w is None else rbf_w.shape[-1]
    _fits(n, H, 0 if Hk is None else Hk, dk, R)
    prm = AttentionParams(H, H if Hk is None else Hk, dk, R, cutoff, scale, cap, dt, ldq, ldk)
    return prm, (_arg(ctx, pos, torch.float32, (n, 3), "pos"), _arg(ctx, graph_id, torch.int32, (n,), "graph_id"),
                 None if q is None else q.data_ptr(), None if k is None else k.data_ptr(), n,
                 _arg(ctx, rbf_w, torch.float32, (H, R), "rbf_w"),
                 _arg(ctx, row_ptr, torch.int64, (n + 1,), "row_ptr"),
                 _arg(ctx, col_idx, torch.int32, (E,), "col_idx"), E)


def e2f_attention_forward(ctx, pos, row_ptr, col_idx, cutoff, q=None, k=None, rbf_w=None, heads=None, scale=1.0,
                          cap=0.0, graph_id=None, alpha=None, lse=None):
    """Attention weights from capped scores under a mask by graph: (alpha
    [E, heads], lse [n, heads]) float32.  q [n, heads, dk], k [n, k_heads, dk]
    float32 or bfloat16, packed within an atom (columns of one projection are
    fine); rbf_w [heads, R] or None; cap 0: none."""
    prm, args = _attention_args(ctx, pos, row_ptr, col_idx, cutoff, q, k, rbf_w, heads, scale, cap, graph_id)
    n, E, H, dev = pos.shape[0], col_idx.numel(), prm.heads, pos.device
    if alpha is None:
        alpha = torch.empty(E, H, dtype=torch.float32, device=dev)
    if lse is None:
        lse = torch.empty(n, H, dtype=torch.float32, device=dev)
    _check(lib.e2f_attention_forward(ctx.handle, ctypes.byref(prm), *args,
                                     _arg(ctx, alpha, torch.float32, (E, H), "alpha"),
                                     _arg(ctx, lse, torch.float32, (n, H), "lse"), _stream(dev)),
           "e2f_attention_forward")
    return alpha, lse


def e2f_attention_backward(ctx, pos, row_ptr, col_idx, cutoff, alpha, lse, grad_alpha, row_t=None, col_t=None,
                           perm=None, q=None, k=None, rbf_w=None, heads=None, scale=1.0, cap=0.0, graph_id=None,
                           want_qk=True, want_rbf=True, want_pos=True, workspace=None):
    """Vector-Jacobian products of e2f_attention_forward: (grad_q [n, heads,
    dk], grad_k [n, k_heads, dk], grad_rbf_w [heads, R], grad_pos [n, 3]), each
    None unless requested and there.  row_t, col_t, perm: e2f_transpose_graph's
    (not needed for grad_rbf_w alone)."""
    prm, args = _attention_args(ctx, pos, row_ptr, col_idx, cutoff, q, k, rbf_w, heads, scale, cap, graph_id)
    n, E, H, dev = pos.shape[0], col_idx.numel(), prm.heads, pos.device
    read = (_arg(ctx, row_t, torch.int64, (n + 1,), "row_t"), _arg(ctx, col_t, torch.int32, (E,), "col_t"),
            _arg(ctx, perm, torch.int32, (E,), "perm"), _arg(ctx, alpha, torch.float32, (E, H), "alpha"),
            _arg(ctx, lse, torch.float32, (n, H), "lse"), _arg(ctx, grad_alpha, torch.float32, (E, H), "grad_alpha"))
    gq = torch.empty(q.shape, dtype=q.dtype, device=dev) if want_qk and prm.dk else None
    gk = torch.empty(k.shape, dtype=k.dtype, device=dev) if want_qk and prm.dk else None
    gw = torch.empty_like(rbf_w) if want_rbf and prm.n_rbf else None
    gp = torch.empty_like(pos) if want_pos else None
    b = ctypes.c_size_t(0)
    _check(lib.e2f_attention_backward_workspace_size(ctx.handle, ctypes.byref(prm), n, E, ctypes.byref(b)),
           "e2f_attention_backward_workspace_size")
    stream = _stream(dev)
    workspace = _workspace(ctx, workspace, b.value, dev, stream)
    _check(lib.e2f_attention_backward(ctx.handle, ctypes.byref(prm), *args, *read,
                                      *(None if t is None else t.data_ptr() for t in (gq, gk, gw, gp)),
                                      workspace.data_ptr(), workspace.numel(), stream),
           "e2f_attention_backward")
    return gq, gk, gw, gp


def _norm_args(ctx, x, lmax, block, gate, post_w, res_scale, pre_w, eps):
    """The parameters, and the addresses of what both directions read."""
    dt, shape = x.dtype, x.shape
    if dt not in _DTYPES:
        raise ValueError("x must be float32 or bfloat16")
    n, C = shape[0], shape[-1]
    if shape != (n, (lmax + 1) ** 2, C) and (lmax or shape != (n, C)):
        raise ValueError("x must be [n, (lmax+1)^2, C]")
    G = 0
    if gate is not None:
        G = 1 if gate.dim() == 2 else gate.shape[1]
    _fits(n, C, G)
    w = [_arg(ctx, t, torch.float32, (lmax + 1, C), name)
         for t, name in ((post_w, "post_w"), (res_scale, "res_scale"), (pre_w, "pre_w"))]
    return NormParams(lmax, C, G, eps, _DTYPES[dt], *w), (
        _arg(ctx, x, dt, shape, "x"), _arg(ctx, block, dt, shape, "block"),
        _arg(ctx, gate, dt, (n, C) if gate is not None and gate.dim() == 2 else (n, G, C), "gate"))


def e2f_block_norm_forward(ctx, x, lmax, block=None, gate=None, post_w=None, res_scale=None, pre_w=None, eps=1e-5,
                           out=None, normed=None):
    """The norm of a block's output, its gate, scale and residual sum, and the
    norm before the next block: (out like x, or x itself without a block;
    normed like x, or None without pre_w; rstd [n, 2] float32 for the backward).
    x, block [n, (lmax+1)^2, C] (lmax = 0: also [n, C]) float32 or bfloat16; gate
    [n, 1 or lmax+1, C] of x's type; post_w, res_scale, pre_w [lmax+1, C] float32."""
    prm, args = _norm_args(ctx, x, lmax, block, gate, post_w, res_scale, pre_w, eps)
    n = x.shape[0]
    if block is not None and out is None:
        out = torch.empty_like(x)
    if pre_w is not None and normed is None:
        normed = torch.empty_like(x)
    rstd = torch.empty(n, 2, dtype=torch.float32, device=x.device)
    _check(lib.e2f_block_norm_forward(ctx.handle, ctypes.byref(prm), *args, n,
                                      _arg(ctx, out, x.dtype, x.shape, "out"),
                                      _arg(ctx, normed, x.dtype, x.shape, "normed"), rstd.data_ptr(),
                                      _stream(x.device)), "e2f_block_norm_forward")
    return x if block is None else out, normed, rstd


def e2f_block_norm_backward(ctx, x, rstd, lmax, block=None, gate=None, post_w=None, res_scale=None, pre_w=None,
                            eps=1e-5, grad_out=None, grad_normed=None, want_weights=True, workspace=None):
    """Vector-Jacobian products of e2f_block_norm_forward: (grad_x, grad_block,
    grad_gate, grad_post_w, grad_res_scale, grad_pre_w), each None where the
    input is; the last three also without want_weights."""
    prm, args = _norm_args(ctx, x, lmax, block, gate, post_w, res_scale, pre_w, eps)
    n = x.shape[0]
    read = (_arg(ctx, rstd, torch.float32, (n, 2), "rstd"), n, _arg(ctx, grad_out, x.dtype, x.shape, "grad_out"),
            _arg(ctx, grad_normed, x.dtype, x.shape, "grad_normed"))
    grads = [None if t is None else torch.empty_like(t) for t in (x, block, gate)]
    grads += [None if t is None or not want_weights else torch.empty_like(t) for t in (post_w, res_scale, pre_w)]
    space, stream = (None, 0), _stream(x.device)
    if any(t is not None for t in grads[3:]):
        b = ctypes.c_size_t(0)
        _check(lib.e2f_block_norm_workspace_size(ctx.handle, ctypes.byref(prm), n, ctypes.byref(b)),
               "e2f_block_norm_workspace_size")
        workspace = _workspace(ctx, workspace, b.value, x.device, stream)
        space = (workspace.data_ptr(), workspace.numel())
    _check(lib.e2f_block_norm_backward(ctx.handle, ctypes.byref(prm), *args, *read,
                                       *(None if t is None else t.data_ptr() for t in grads), *space,
                                       stream), "e2f_block_norm_backward")
    return tuple(grads)


class _TensorList:
    """Host arrays of the addresses, sizes and types of device tensors (contiguous, on the context's device)."""

    def __init__(self, ctx, tensors, name):
        dtypes = array.array("i", [_DTYPES.get(t.dtype, -1) for t in tensors])
        if (-1 in dtypes or not all(map(torch.Tensor.is_contiguous, tensors)) or
                not {ctx.device}.issuperset(map(torch.Tensor.get_device, tensors))):
            raise ValueError("%s must be contiguous float32 or bfloat16 tensors on the context's device" % name)
        self.count = len(tensors)
        self.keep = (array.array("Q", map(torch.Tensor.data_ptr, tensors)),
                     array.array("q", map(torch.Tensor.numel, tensors)), dtypes)
        self.ptrs, self.sizes, self.dtypes = (a.buffer_info()[0] for a in self.keep)


def _grad_norm(ctx, t, device, workspace, stream):
    b = ctypes.c_size_t(0)
    _check(lib.e2f_grad_norm_workspace_size(ctx.handle, t.count, t.sizes, ctypes.byref(b)),
           "e2f_grad_norm_workspace_size")
    workspace = _workspace(ctx, workspace, b.value, device, stream)
    sumsq, norm = (torch.empty((), dtype=d, device=device) for d in (torch.float64, torch.float32))
    _check(lib.e2f_grad_norm(ctx.handle, t.count, t.ptrs, t.sizes, t.dtypes, _ptr(sumsq), _ptr(norm),
                             _ptr(workspace), workspace.numel(), stream), "e2f_grad_norm")
    return sumsq, norm


def _grad_clip(ctx, t, outs, sumsq, max_norm, stream):
    to = t if outs is None else _TensorList(ctx, outs, "outs")
    if to.keep[1:] != t.keep[1:]:
        raise ValueError("outs must have the tensors' sizes and types")
    _check(lib.e2f_grad_clip(ctx.handle, t.count, t.ptrs, to.ptrs, t.sizes, t.dtypes, _ptr(sumsq), float(max_norm),
                             stream), "e2f_grad_clip")


def e2f_grad_norm(ctx, tensors, workspace=None):
    """The norm over all values of the tensors: (sumsq float64, norm float32),
    device tensors without dimensions.  Ranks that hold parts add sumsq."""
    device = torch.device("cuda", ctx.device)
    return _grad_norm(ctx, _TensorList(ctx, tensors, "tensors"), device, workspace, _stream(device))


def e2f_grad_clip(ctx, tensors, sumsq, max_norm, outs=None):
    """outs[t] = tensors[t] * min(1, max_norm / (sqrt(sumsq) + 1e-6)), in place
    without outs; sumsq: e2f_grad_norm's (or the sum of several ranks')."""
    _arg(ctx, sumsq, torch.float64, (), "sumsq")
    _grad_clip(ctx, _TensorList(ctx, tensors, "tensors"), outs, sumsq, max_norm, _stream(sumsq.device))
    return tensors if outs is None else outs


def e2f_clip_grad_norm(ctx, tensors, max_norm, outs=None, workspace=None):
    """e2f_grad_norm and e2f_grad_clip of the same tensors; returns the norm
    before clipping (float32, a device tensor without dimensions)."""
    device = torch.device("cuda", ctx.device)
    t = _TensorList(ctx, tensors, "tensors")
    stream = _stream(device)
    sumsq, norm = _grad_norm(ctx, t, device, workspace, stream)
    _grad_clip(ctx, t, outs, sumsq, max_norm, stream)
    return norm


def _rows(ctx, t, n, lmax, C, dtype, name):
    """Elements between rows of t [n, (lmax+1)^2, C] (lmax = 0: also [n, C]), packed within a row; 0: packed."""
    if t.dtype != dtype or t.get_device() != ctx.device:
        raise ValueError("%s must be a %s tensor on the context's device" % (name, dtype))
    K = (lmax + 1) ** 2
    shape, stride = t.shape, t.stride()
    if shape != (n, K, C) and (lmax or shape != (n, C)):
        raise ValueError("%s must be [%d, %d, %d]" % (name, n, K, C))
    if (C > 1 and stride[-1] != 1) or (K > 1 and stride[1] != C) or (n > 1 and stride[0] < K * C):
        raise ValueError("%s must be packed within a row, with at least (lmax+1)^2 C elements between rows" % name)
    return stride[0] if n > 1 else 0


def _embedding_args(ctx, index, vocab, C, lmax, scale, table_dtype, dtype, ld):
    """The parameters and the index's address."""
    if index.dtype not in (torch.int32, torch.int64) or index.dim() != 1:
        raise ValueError("index must be [n] of int32 or int64")
    if table_dtype not in _DTYPES or dtype not in _DTYPES:
        raise ValueError("the table and the rows must be float32 or bfloat16")
    _fits(index.shape[0], vocab, C)
    return (EmbeddingParams(vocab, C, lmax, scale, _DTYPES[table_dtype], _DTYPES[dtype],
                            4 if index.dtype == torch.int32 else 8, ld),
            _arg(ctx, index, index.dtype, index.shape, "index"))


def e2f_embedding_forward(ctx, table, index, lmax=0, scale=1.0, dtype=None, out=None):
    """Rows of the table [V, C] (float32 or bfloat16) by their types, as the
    scalars of irrep features: out [n, (lmax+1)^2, C] (lmax = 0: [n, C]) of
    `dtype` (the table's where None), the other components 0.  index [n] int32 or
    int64; those outside [0, V) give zeros.  out may have rows further apart."""
    if table.dim() != 2:
        raise ValueError("table must be [V, C]")
    n, (V, C) = index.shape[0], table.shape
    if out is None:
        dtype = table.dtype if dtype is None else dtype
        out = torch.empty((n, (lmax + 1) ** 2, C) if lmax else (n, C), dtype=dtype, device=table.device)
        ld = 0
    else:
        dtype = out.dtype if dtype is None else dtype
        ld = _rows(ctx, out, n, lmax, C, dtype, "out")
    prm, at = _embedding_args(ctx, index, V, C, lmax, scale, table.dtype, dtype, ld)
    _check(lib.e2f_embedding_forward(ctx.handle, ctypes.byref(prm), _arg(ctx, table, table.dtype, (V, C), "table"), at,
                                     n, out.data_ptr(), _stream(table.device)), "e2f_embedding_forward")
    return out


def e2f_embedding_backward(ctx, index, grad_out, vocab, lmax=0, scale=1.0, dtype=None, grad_table=None,
                           workspace=None):
    """The gradient of e2f_embedding_forward's table, [vocab, C] of `dtype`
    (grad_out's where None), zeros for types without rows.  grad_out [n,
    (lmax+1)^2, C] (lmax = 0: also [n, C]) may have rows further apart."""
    n, C, dev = index.shape[0], grad_out.shape[-1], grad_out.device
    ld = _rows(ctx, grad_out, n, lmax, C, grad_out.dtype, "grad_out")
    if grad_table is None:
        grad_table = torch.empty(vocab, C, dtype=grad_out.dtype if dtype is None else dtype, device=dev)
    elif dtype is not None and grad_table.dtype != dtype:
        raise ValueError("grad_table must be of `dtype`")
    prm, at = _embedding_args(ctx, index, vocab, C, lmax, scale, grad_table.dtype, grad_out.dtype, ld)
    b = ctypes.c_size_t(0)
    _check(lib.e2f_embedding_backward_workspace_size(ctx.handle, ctypes.byref(prm), n, ctypes.byref(b)),
           "e2f_embedding_backward_workspace_size")
    stream = _stream(dev)
    workspace = _workspace(ctx, workspace, b.value, dev, stream)
    _check(lib.e2f_embedding_backward(ctx.handle, ctypes.byref(prm), at, n, grad_out.data_ptr(),
                                      _arg(ctx, grad_table, grad_table.dtype, (vocab, C), "grad_table"),
                                      workspace.data_ptr(), workspace.numel(), stream), "e2f_embedding_backward")
    return grad_table


def _layer_args(ctx, x, lmax, weight, bias, eps, silu):
    """The parameters, the rows and a row's channels."""
    if x.dtype not in _DTYPES:
        raise ValueError("x must be float32 or bfloat16")
    n, C = x.shape[0], x.shape[-1]
    _fits(n, C)
    if weight is not None and not lmax and weight.dim() == 1:
        weight = weight[None]
    return n, C, LayerNormParams(lmax, C, eps, int(bool(silu)), _DTYPES[x.dtype],
                                 _arg(ctx, weight, torch.float32, (lmax + 1, C), "weight"),
                                 _arg(ctx, bias, torch.float32, (C,), "bias"),
                                 _rows(ctx, x, n, lmax, C, x.dtype, "x"))


def e2f_layer_norm_forward(ctx, x, lmax=0, weight=None, bias=None, eps=1e-5, silu=False, out=None):
    """Layer norm of irrep features x [n, (lmax+1)^2, C] (scalars by mean and
    variance, higher degrees by one root mean square), or of rows [n, C] with lmax
    = 0, there with silu also its activation: out like x, packed.  x float32 or
    bfloat16, whose rows may be further apart; weight [lmax+1, C] (lmax = 0: also
    [C]), bias [C] float32."""
    n, C, prm = _layer_args(ctx, x, lmax, weight, bias, eps, silu)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _check(lib.e2f_layer_norm_forward(ctx.handle, ctypes.byref(prm), x.data_ptr(), n,
                                      _arg(ctx, out, x.dtype, x.shape, "out"), _stream(x.device)),
           "e2f_layer_norm_forward")
    return out


def e2f_layer_norm_backward(ctx, x, grad_out, lmax=0, weight=None, bias=None, eps=1e-5, silu=False, want_x=True,
                            want_weights=True, workspace=None):
    """Vector-Jacobian products of e2f_layer_norm_forward: (grad_x like x,
    packed; grad_weight [lmax+1, C]; grad_bias [C]), None unless wanted."""
    n, C, prm = _layer_args(ctx, x, lmax, weight, bias, eps, silu)
    dev = x.device
    gx = torch.empty(x.shape, dtype=x.dtype, device=dev) if want_x else None
    gw = gb = None
    space, stream = (None, 0), _stream(dev)
    if want_weights:
        gw = torch.empty(lmax + 1, C, dtype=torch.float32, device=dev)
        gb = torch.empty(C, dtype=torch.float32, device=dev)
        if weight is not None and weight.dim() == 1:
            gw = gw[0]
        b = ctypes.c_size_t(0)
        _check(lib.e2f_layer_norm_workspace_size(ctx.handle, ctypes.byref(prm), n, ctypes.byref(b)),
               "e2f_layer_norm_workspace_size")
        workspace = _workspace(ctx, workspace, b.value, dev, stream)
        space = (workspace.data_ptr(), workspace.numel())
    _check(lib.e2f_layer_norm_backward(ctx.handle, ctypes.byref(prm), x.data_ptr(), n,
                                       _arg(ctx, grad_out, x.dtype, x.shape, "grad_out"),
                                       *(None if t is None else t.data_ptr() for t in (gx, gw, gb)), *space, stream),
           "e2f_layer_norm_backward")
    return gx, gw, gb


def _matrices(ctx, tensors, name, dtype, shapes):
    """Checks matrices [rows, cols] or stacks of them [batch, rows, cols] of these shapes (contiguous, of one type)."""
    if list(map(_SHAPE, tensors)) != shapes:
        raise ValueError("%s must have the gradients' shapes" % name)
    if (not {dtype}.issuperset(map(_DTYPE, tensors)) or not all(map(torch.Tensor.is_contiguous, tensors)) or
            not {ctx.device}.issuperset(map(torch.Tensor.get_device, tensors))):
        raise ValueError("%s must be contiguous tensors of one type on the context's device" % name)


def _addresses(tensors, many, step):
    """Host array of the addresses of the tensors' matrices: many[k] of them in tensor k, `step` bytes each."""
    first = list(map(torch.Tensor.data_ptr, tensors))
    if step and len(set(many)) == 1:
        offsets = range(0, many[0] * step, step)
        return array.array("Q", [a + i for a in first for i in offsets])
    return array.array("Q", [a + i * step for a, n in zip(first, many) for i in range(n)])


def _disjoint(outputs, inputs):
    """Refuses lists of tensors in which an output lies over another tensor, but over the one of its own number that it
    replaces.  inputs: lists, or None; outputs: (a list, which of the inputs' lists it replaces, -1: none)."""
    span = lambda t: (t.data_ptr(), t.data_ptr() + t.numel() * t.element_size())  # noqa: E731
    outs = sorted((*span(t), which, i) for ts, which in outputs for i, t in enumerate(ts) if t.numel())
    if any(b[0] < a[1] for a, b in zip(outs, outs[1:])):
        raise ValueError("two outputs overlap")
    for which, ts in enumerate(inputs):
        for i, t in enumerate(ts or ()):
            lo, hi = span(t)
            # (the outputs are disjoint: the last that begins before the input's end is the one that ends last)
            k = bisect.bisect_left(outs, (hi,)) - 1
            if lo < hi and k >= 0 and outs[k][1] > lo and outs[k] != (lo, hi, which, i):
                raise ValueError("an output overlaps another tensor")


def e2f_orthogonalize(ctx, grads, outs=None, weights=None, moments=None, new_moments=None, momentum=0.95,
                      nesterov=True, steps=5, coefs=None, scale=1.0, decay=0.0, eps=1e-7, workspace=None):
    """Orthogonalised updates of matrices (the step of the Muon optimiser):
    outs[t] = decay weights[t] + scale X, X from grads[t] through its momentum by
    `steps` Newton-Schulz steps with coefs (a, b, c), or one such triple for
    each step (None: 3.4445, -4.7750, 2.0315).  Tensors are matrices [rows, cols]
    or stacks [batch, rows, cols] of any sizes; grads of one type, weights and outs of one
    (float32 or bfloat16), moments float32.  Without moments the gradients
    themselves are orthogonalised.  None: new tensors like weights (or grads) for outs, and
    moments themselves for new_moments; outs may be weights; apart from these no output may lie over another tensor.  A call that is
    refused has changed nothing.  Under graph capture a workspace must be given, as for every operator with one, also
    where no matrix needs it.  Returns outs."""
    if not grads:
        return [] if outs is None else outs
    gt, shapes = grads[0].dtype, list(map(_SHAPE, grads))
    if not {2, 3}.issuperset(map(len, shapes)):
        raise ValueError("grads must be [rows, cols] or [batch, rows, cols]")
    _matrices(ctx, grads, "grads", gt, shapes)
    if outs is None:
        outs = [torch.empty_like(t) for t in (grads if weights is None else weights)]
    wt = outs[0].dtype if outs else None
    if gt not in _DTYPES or wt not in _DTYPES:
        raise ValueError("grads and outs must be float32 or bfloat16")
    _matrices(ctx, outs, "outs", wt, shapes)
    if weights is not None and weights is not outs:
        _matrices(ctx, weights, "weights", wt, shapes)
    if new_moments is None:
        new_moments = moments
    elif moments is None:
        raise ValueError("new_moments without moments")
    if moments is not None:
        _matrices(ctx, moments, "moments", torch.float32, shapes)
        if new_moments is not moments:
            _matrices(ctx, new_moments, "new_moments", torch.float32, shapes)
    flat = None
    if coefs is not None:
        flat = [float(c) for row in (coefs if len(coefs) and hasattr(coefs[0], "__len__") else [coefs] * steps)
                for c in row]
        if len(flat) != 3 * steps:
            raise ValueError("coefs must be three numbers, or three for each step")
        flat = array.array("f", flat)
    by_size = {}
    for k, shape in enumerate(shapes):
        by_size.setdefault(shape[-2:], []).append(k)
    device = grads[0].device
    stream = _stream(device)
    # every size is checked before the first is launched: a call that is refused has changed nothing
    calls, need = [], 0
    for (rows, cols), which in by_size.items():
        _fits(rows, cols)
        many = [1 if len(shapes[k]) == 2 else shapes[k][0] for k in which]
        lists = []
        for tensors in (grads, moments, new_moments, weights, outs):
            if tensors is None:
                lists.append(None)
                continue
            mine = tensors if len(by_size) == 1 else [tensors[k] for k in which]
            lists.append(_addresses(mine, many, rows * cols * mine[0].element_size()))
        prm = OrthogonalizeParams(rows, cols, steps, None if flat is None else flat.buffer_info()[0], eps, momentum,
                                  int(bool(nesterov)), scale, decay, _DTYPES[gt], _DTYPES[wt])
        b = ctypes.c_size_t(0)
        _check(lib.e2f_orthogonalize_workspace_size(ctx.handle, ctypes.byref(prm), len(lists[0]), ctypes.byref(b)),
               "e2f_orthogonalize_workspace_size")
        calls.append((prm, lists))
        need = max(need, b.value)
    space = _workspace(ctx, workspace, need, device, stream)
    if len(calls) > 1:  # (the library sees the matrices of one size at a time)
        if space.numel() < need:
            raise E2FError(E2F_ECAPACITY, "e2f_orthogonalize", "workspace of %d bytes is required" % need)
        if need and space.data_ptr() % 256:
            raise E2FError(E2F_EINVAL, "e2f_orthogonalize", "workspace must be 256-byte aligned")
        _disjoint([(outs, 2), ([space[:need]], -1)] + ([] if new_moments is None else [(new_moments, 1)]),
                  [grads, moments, None if decay == 0 else weights])
    for prm, lists in calls:
        _check(lib.e2f_orthogonalize(ctx.handle, ctypes.byref(prm), len(lists[0]),
                                     *(None if a is None else a.buffer_info()[0] for a in lists), space.data_ptr(),
                                     space.numel(), stream), "e2f_orthogonalize")
    return outs


def e2f_solid_harmonics(ctx: Context, pos: torch.Tensor, lmax: int, origins: torch.Tensor | None = None,
                        origin_id: torch.Tensor | None = None) -> torch.Tensor:
    _dev(pos, torch.float32, "pos")
    _dev(origins, torch.float32, "origins")
    _dev(origin_id, torch.int32, "origin_id")
    out = torch.empty(pos.shape[0], (lmax + 1) ** 2, dtype=torch.float32, device=pos.device)
    _check(lib.e2f_solid_harmonics(ctx.handle, _ptr(pos), _ptr(origins), _ptr(origin_id), pos.shape[0], lmax,
                                   _ptr(out), _stream(pos.device)), "e2f_solid_harmonics")
    return out


def e2f_node_tp(ctx: Context, pos: torch.Tensor, feat: torch.Tensor, lmax: int, origins: torch.Tensor | None = None,
                origin_id: torch.Tensor | None = None) -> torch.Tensor:
    _dev(pos, torch.float32, "pos")
    _dev(feat, torch.float32, "feat")
    _dev(origins, torch.float32, "origins")
    _dev(origin_id, torch.int32, "origin_id")
    n, nk, C = feat.shape
    out = torch.empty(n, e2f_node_tp_dim(lmax), C, dtype=torch.float32, device=feat.device)
    _check(lib.e2f_node_tp(ctx.handle, _ptr(pos), _ptr(origins), _ptr(origin_id), _ptr(feat), n, C, lmax, _ptr(out),
                           _stream(feat.device)), "e2f_node_tp")
    return out


def e2f_aggregate(ctx: Context, T: torch.Tensor, row_ptr: torch.Tensor, col_idx: torch.Tensor,
                  alpha: torch.Tensor | None, out: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None, order: torch.Tensor | None = None) -> torch.Tensor:
    """The aggregation alone: S[i][h] = sum over row i's edges e = (i, j) of
    alpha[e][h] T[j][h] for T [n, heads, rows, C/heads] float32 (head-major);
    alpha [E, heads] or None (ones); order: int32 [n], the permutation whose
    consecutive receivers form the blocks (None: index order).  Returns S of
    T's shape.  (sync)"""
    _dev(T, torch.float32, "T")
    _dev(row_ptr, torch.int64, "row_ptr")
    _dev(col_idx, torch.int32, "col_idx")
    _dev(alpha, torch.float32, "alpha")
    _dev(order, torch.int32, "order")
    if T.dim() != 4:
        raise ValueError("T must be [n, heads, rows, C/heads]")
    n, H, K, dh = T.shape
    E = col_idx.numel()
    if out is None:
        out = torch.empty_like(T)
    _dev(out, torch.float32, "out")
    if workspace is None:
        b = ctypes.c_size_t(0)
        _check(lib.e2f_aggregate_workspace_size(ctx.handle, n, E, H, ctypes.byref(b)), "e2f_aggregate_workspace_size")
        workspace = ctx.workspace_for(b.value, T.device)
    elif not workspace.is_cuda or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 device tensor")
    _check(lib.e2f_aggregate(ctx.handle, _ptr(T), n, K, H * dh, H, _ptr(row_ptr), _ptr(col_idx), E, _ptr(alpha),
                             _ptr(order), _ptr(out), _ptr(workspace), workspace.numel(), _stream(T.device)),
           "e2f_aggregate")
    return out


def _params(lmax, channels, heads, cutoff, path_w, mix_w, tile_side, y_norm=False, form="auto"):
    import numpy as np
    keep = None
    pw = None
    if path_w is not None:
        keep = np.ascontiguousarray(path_w, dtype=np.float64)
        if keep.size != (lmax + 1) ** 3:
            raise ValueError("path_w must have (lmax+1)^3 entries")
        pw = keep.ctypes.data_as(ctypes.c_void_p)
    mix_dtype = E2F_F32
    if mix_w is not None:
        if mix_w.dtype == torch.bfloat16:
            mix_dtype = E2F_BF16
        else:
            _dev(mix_w, torch.float32, "mix_w")
        if not mix_w.is_cuda or not mix_w.is_contiguous():
            raise ValueError("mix_w must be a contiguous device tensor")
    prm = ConvParams(lmax, channels, heads, cutoff, pw, None if mix_w is None else mix_w.data_ptr(), mix_dtype,
                     float(tile_side), int(bool(y_norm)), _FORMS[form] if isinstance(form, str) else int(form))
    return prm, keep


def _conv_args(pos, feat, row_ptr, col_idx, alpha, graph_id, out):
    _dev(pos, torch.float32, "pos")
    _dev(feat, torch.float32, "feat")
    _dev(row_ptr, torch.int64, "row_ptr")
    _dev(col_idx, torch.int32, "col_idx")
    _dev(alpha, torch.float32, "alpha")
    _dev(graph_id, torch.int32, "graph_id")
    if out is None:
        out = torch.empty_like(feat)
    _dev(out, torch.float32, "out")
    return out


def e2f_wigner6j_workspace_size(ctx, n, n_edges, lmax, channels, heads, cutoff, path_w=None, mix_w=None,
                                tile_side=0.0, y_norm=False, minimum=False, form="auto") -> int:
    """Workspace bytes of the forward (the one-pass size, or with minimum=True
    the smallest size it accepts)."""
    prm, keep = _params(lmax, channels, heads, cutoff, path_w, mix_w, tile_side, y_norm, form)
    b = ctypes.c_size_t(0)
    fn = lib.e2f_wigner6j_workspace_min if minimum else lib.e2f_wigner6j_workspace_size
    _check(fn(ctx.handle, ctypes.byref(prm), n, n_edges, ctypes.byref(b)),
           "e2f_wigner6j_workspace_min" if minimum else "e2f_wigner6j_workspace_size")
    del keep
    return b.value


def e2f_wigner6j_prepare(ctx, lmax, channels, heads, cutoff, path_w=None, mix_w=None, tile_side=0.0,
                         y_norm=False, form="auto") -> None:
    """Upload the coefficient set and coupling schedule these parameters use."""
    prm, keep = _params(lmax, channels, heads, cutoff, path_w, mix_w, tile_side, y_norm, form)
    _check(lib.e2f_wigner6j_prepare(ctx.handle, ctypes.byref(prm)), "e2f_wigner6j_prepare")
    del keep


def e2f_wigner6j_conv_forward(ctx, pos, feat, row_ptr, col_idx, alpha, lmax, heads, cutoff, path_w=None, mix_w=None,
                              graph_id=None, tile_side=0.0, out=None, y_norm=False, workspace=None,
                              form="auto"):
    """Wigner-6j convolution forward; returns out [N,(L+1)^2,C] float32.
    y_norm: attention weights alpha / |r_i - r_j|^f per filter degree f.
    workspace: a uint8 device tensor (any size from the minimum up); None
    uses the context's own, grown to the one-pass size.
    form: "auto", "split" (S written, then recoupled by a second kernel) or
    "fused" (the aggregation applies the recouple itself where it can)."""
    out = _conv_args(pos, feat, row_ptr, col_idx, alpha, graph_id, out)
    n, nk, C = feat.shape
    E = col_idx.numel()
    prm, keep = _params(lmax, C, heads, cutoff, path_w, mix_w, tile_side, y_norm, form)
    if workspace is None:
        b = ctypes.c_size_t(0)
        _check(lib.e2f_wigner6j_workspace_size(ctx.handle, ctypes.byref(prm), n, E, ctypes.byref(b)),
               "e2f_wigner6j_workspace_size")
        workspace = ctx.workspace_for(b.value, feat.device)
    elif not workspace.is_cuda or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 device tensor")
    st = lib.e2f_wigner6j_conv_forward(ctx.handle, ctypes.byref(prm), _ptr(pos), _ptr(graph_id), _ptr(feat), n,
                                       _ptr(row_ptr), _ptr(col_idx), E, _ptr(alpha), _ptr(out), _ptr(workspace),
                                       workspace.numel(), _stream(feat.device))
    del keep
    _check(st, "e2f_wigner6j_conv_forward")
    return out


def e2f_wigner6j_conv_forward_noalloc(ctx, pos, feat, row_ptr, col_idx, alpha, lmax, heads, cutoff, path_w=None,
                                      mix_w=None, graph_id=None, tile_side=0.0, out=None, y_norm=False,
                                      form="auto"):
    """The forward in the library's per-GPU scratch memory (no allocation;
    the parameters must have been prepared).  out must be given by callers
    that cannot allocate: with out=None the binding allocates it."""
    out = _conv_args(pos, feat, row_ptr, col_idx, alpha, graph_id, out)
    n, nk, C = feat.shape
    prm, keep = _params(lmax, C, heads, cutoff, path_w, mix_w, tile_side, y_norm, form)
    st = lib.e2f_wigner6j_conv_forward_noalloc(ctx.handle, ctypes.byref(prm), _ptr(pos), _ptr(graph_id), _ptr(feat),
                                               n, _ptr(row_ptr), _ptr(col_idx), col_idx.numel(), _ptr(alpha),
                                               _ptr(out), _stream(feat.device))
    del keep
    _check(st, "e2f_wigner6j_conv_forward_noalloc")
    return out


def e2f_edge_tp_conv_forward(ctx, pos, feat, row_ptr, col_idx, alpha, lmax, heads, cutoff, path_w=None, mix_w=None,
                             graph_id=None, tile_side=0.0, out=None, y_norm=False):
    """Per-edge SO(3) convolution baseline; same output as the 6j forward."""
    out = _conv_args(pos, feat, row_ptr, col_idx, alpha, graph_id, out)
    n, nk, C = feat.shape
    prm, keep = _params(lmax, C, heads, cutoff, path_w, mix_w, tile_side, y_norm)
    st = lib.e2f_edge_tp_conv_forward(ctx.handle, ctypes.byref(prm), _ptr(pos), _ptr(graph_id), _ptr(feat), n,
                                      _ptr(row_ptr), _ptr(col_idx), col_idx.numel(), _ptr(alpha), _ptr(out),
                                      _stream(feat.device))
    del keep
    _check(st, "e2f_edge_tp_conv_forward")
    return out


def e2f_validate_graph(ctx, n, row_ptr, col_idx) -> int:
    """0 if the device CSR is well formed, else the error bits of e2f.h."""
    _dev(row_ptr, torch.int64, "row_ptr")
    _dev(col_idx, torch.int32, "col_idx")
    bad = ctypes.c_int32(0)
    _check(lib.e2f_validate_graph(ctx.handle, n, _ptr(row_ptr), _ptr(col_idx), col_idx.numel(), ctypes.byref(bad),
                                  _stream(row_ptr.device)), "e2f_validate_graph")
    return bad.value


def e2f_wigner6j_conv_forward_dense(ctx, pos, feat, alpha, lmax, heads, cutoff, path_w=None, mix_w=None, out=None):
    """Dense-graph forward (every atom attends to every other): alpha [N,N,H]
    float32 (receiver, sender, head) or None; returns out [N,(L+1)^2,C]."""
    _dev(pos, torch.float32, "pos")
    _dev(feat, torch.float32, "feat")
    _dev(alpha, torch.float32, "alpha")
    n, nk, C = feat.shape
    if alpha is not None and tuple(alpha.shape) != (n, n, heads):
        raise ValueError("alpha must be [N, N, heads]")
    if out is None:
        out = torch.empty_like(feat)
    _dev(out, torch.float32, "out")
    prm, keep = _params(lmax, C, heads, cutoff, path_w, mix_w, 0.0)
    st = lib.e2f_wigner6j_conv_forward_dense(ctx.handle, ctypes.byref(prm), _ptr(pos), _ptr(feat), n, _ptr(alpha),
                                             _ptr(out), _stream(feat.device))
    del keep
    _check(st, "e2f_wigner6j_conv_forward_dense")
    return out


def e2f_wigner6j_conv_forward_global(ctx, pos, feat, lmax, heads, cutoff, path_w=None, mix_w=None, out=None):
    """Uniform attention over the whole graph (alpha = 1 for every pair, self
    included), in O(N) through the global moments; returns out [N,(L+1)^2,C]."""
    _dev(pos, torch.float32, "pos")
    _dev(feat, torch.float32, "feat")
    n, nk, C = feat.shape
    if out is None:
        out = torch.empty_like(feat)
    _dev(out, torch.float32, "out")
    prm, keep = _params(lmax, C, heads, cutoff, path_w, mix_w, 0.0)
    st = lib.e2f_wigner6j_conv_forward_global(ctx.handle, ctypes.byref(prm), _ptr(pos), _ptr(feat), n, _ptr(out),
                                              _stream(feat.device))
    del keep
    _check(st, "e2f_wigner6j_conv_forward_global")
    return out


def e2f_wigner6j_conv_backward(ctx, pos, feat, grad_out, row_ptr, col_idx, alpha, lmax, heads, cutoff, path_w=None,
                               mix_w=None, graph_id=None, tile_side=0.0, want_feat=True, want_alpha=True,
                               want_pos=False):
    """Vector-Jacobian products of the forward: (grad_feat [N,(L+1)^2,C],
    grad_alpha [E,H], grad_pos [N,3]), each None unless requested."""
    for t, name in ((pos, "pos"), (feat, "feat"), (grad_out, "grad_out"), (alpha, "alpha")):
        _dev(t, torch.float32, name)
    _dev(row_ptr, torch.int64, "row_ptr")
    _dev(col_idx, torch.int32, "col_idx")
    _dev(graph_id, torch.int32, "graph_id")
    n, nk, C = grad_out.shape
    E = col_idx.numel()
    gf = torch.empty_like(grad_out) if want_feat else None
    ga = torch.empty(E, heads, dtype=torch.float32, device=grad_out.device) if want_alpha else None
    gp = torch.empty(n, 3, dtype=torch.float32, device=grad_out.device) if want_pos else None
    prm, keep = _params(lmax, C, heads, cutoff, path_w, mix_w, tile_side)
    st = lib.e2f_wigner6j_conv_backward(ctx.handle, ctypes.byref(prm), _ptr(pos), _ptr(graph_id), _ptr(feat),
                                        _ptr(grad_out), n, _ptr(row_ptr), _ptr(col_idx), E, _ptr(alpha), _ptr(gf),
                                        _ptr(ga), _ptr(gp), _stream(grad_out.device))
    del keep
    _check(st, "e2f_wigner6j_conv_backward")
    return gf, ga, gp


def e2f_profile(ctx: Context, enable: bool) -> None:
    """Start (clearing earlier records) or stop event timing of every launch group."""
    _check(lib.e2f_profile(ctx.handle, 1 if enable else 0), "e2f_profile")


def e2f_profile_read(ctx: Context) -> dict:
    """{step name: (launch groups, total ms)} recorded since e2f_profile(ctx, True)."""
    buf = ctypes.create_string_buffer(1 << 16)
    _check(lib.e2f_profile_read(ctx.handle, buf, len(buf)), "e2f_profile_read")
    out = {}
    for line in buf.value.decode().splitlines():
        name, cnt, ms = line.split()
        out[name] = (int(cnt), float(ms))
    return out


def e2f_last_slices(ctx: Context) -> int:
    """Receiver slices of the last factorised forward on this context."""
    v = ctypes.c_int64(0)
    _check(lib.e2f_last_slices(ctx.handle, ctypes.byref(v)), "e2f_last_slices")
    return v.value
