"""Python binding of libdynahead (ctypes).

Argument marshalling only: every step of the draft head runs in the HIP
kernels of libdynahead.so.  PyTorch supplies device memory and streams.  The
binding fails loudly when the library is missing; there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdynahead.so")

OK, ERR_INVALID_ARG, ERR_CAPACITY, ERR_WORKSPACE, ERR_UNSUPPORTED, ERR_HIP, ERR_DEVICE_DATA = range(7)
F32, BF16 = 0, 1
ACT = {"none": 0, "relu": 1, "silu": 2}
SEL_ARGMAX, SEL_TOPK, SEL_SAMPLE, SEL_UNION = 1, 2, 4, 8
OPT_LOGITS_PATH, OPT_ROUTER_PATH, OPT_KERNEL_TIMING, OPT_GEMV_ROWS, OPT_FUSED_B1, OPT_MFMA_UNROLL = 1, 2, 3, 4, 5, 6
OPT_GATHER_CFG, OPT_GREEDY_GRID, OPT_UNION_CFG, OPT_KMEANS_CFG, OPT_WAIT_BOUND_US = 7, 8, 9, 10, 11
MAX_KT = 64
MAX_STEPS, MAX_NODES, MAX_TEACHER = 32, 1024, 1024


class DynaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{message} (status {status})")
        self.status = status


class _Layout(ctypes.Structure):
    _fields_ = [("V", ctypes.c_int32), ("d", ctypes.c_int32), ("M", ctypes.c_int32),
                ("wdtype", ctypes.c_int32), ("W_perm", ctypes.c_void_p),
                ("perm", ctypes.c_void_p), ("offsets", ctypes.c_void_p),
                ("cap_by_k", ctypes.c_void_p), ("max_cluster", ctypes.c_int32)]


class _Router(ctypes.Structure):
    _fields_ = [("d_r", ctypes.c_int32), ("H", ctypes.c_int32), ("M", ctypes.c_int32),
                ("wdtype", ctypes.c_int32), ("act", ctypes.c_int32), ("W1", ctypes.c_void_p),
                ("b1", ctypes.c_void_p), ("W2", ctypes.c_void_p), ("b2", ctypes.c_void_p)]


class _DraftStep(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_void_p), ("logprobs", ctypes.c_void_p), ("logits", ctypes.c_void_p),
                ("clusters", ctypes.c_void_p), ("k", ctypes.c_int32), ("cap", ctypes.c_int32),
                ("shared", ctypes.c_int32), ("temperature", ctypes.c_float), ("tail_beta", ctypes.c_float)]


class _Quant(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("d", ctypes.c_int32), ("data", ctypes.c_void_p)]


class _ShortlistRows(ctypes.Structure):
    _fields_ = [("L", ctypes.c_void_p), ("token_rows", ctypes.c_void_p), ("sel_sorted", ctypes.c_void_p),
                ("sel_rowoff", ctypes.c_void_p), ("row_len", ctypes.c_void_p), ("k", ctypes.c_int32),
                ("shared", ctypes.c_int32)]


_lib = None
ABI_VERSION = 2  # DYNA_ABI_VERSION of include/dynahead.h

_P = ctypes.c_void_p
_I = ctypes.c_int32
_F = ctypes.c_float
_Z = ctypes.c_size_t
_L = ctypes.c_int64

_SIGNATURES = {
    "dyna_abi_version": (_I, []),
    "dyna_status_string": (ctypes.c_char_p, [_I]),
    "dyna_last_error": (ctypes.c_char_p, []),
    "dyna_set_option": (_I, [_I, _I]),
    "dyna_kernel_timing": (_I, [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64), _I]),
    "dyna_layout_workspace_bytes": (_Z, [_I, _I]),
    "dyna_build_layout": (_I, [_P, _I, _I, _P, _I, _I, _P, _P, _P, _P, _P, _P, _Z, _P]),
    "dyna_workspace_bytes": (_Z, [_P, _P, _I, _I, _I]),
    "dyna_route": (_I, [_P, _P, _I, _I, _I, _P, _P, _P, _P, _Z, _P]),
    "dyna_shortlist": (_I, [_P, _P, _I, _I, _P, _P, _P, _P, _I, _P]),
    "dyna_shortlist_logits": (_I, [_P, _P, _I, _I, _I, _P, _P, _P, _P, _I, _P, _Z, _P]),
    "dyna_draft_select": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _F, _F, _P, _P, _P, _P, _P,
                               _P, _Z, _P]),
    "dyna_draft_head": (_I, [_P, _P, _P, _P, _I, _I, _I, _I, _I, _F, _F, _P, _P, _P, _P, _P, _P, _P,
                             _I, _P, _Z, _P, _P, _P]),
    "dyna_draft_head_noalloc": (_I, [_P, _P, _P, _P, _I, _I, _I, _I, _I, _F, _F, _P, _P, _P, _P, _P, _P, _P,
                                     _I, _P]),
    "dyna_dense_workspace_bytes": (_Z, [_I, _I]),
    "dyna_cluster_budget": (_I, [_I, _I, _I, _I, _I]),
    "dyna_beam_expand": (_I, [_P, _P, _P, _I, _I, _I, _P, _P, _P, _P]),
    "dyna_kmeans_workspace_bytes": (ctypes.c_size_t, [_I, _I, _I]),
    "dyna_kmeans_assign": (_I, [_P, _I, _I, _I, _P, _I, _P, _P, _P, ctypes.c_size_t, _P]),
    "dyna_kmeans_update": (_I, [_P, _I, _I, _I, _P, _I, _P, _P, ctypes.c_size_t, _P]),
    "dyna_kmeans": (_I, [_P, _I, _I, _I, _I, _P, _I, _P, _P, _P, ctypes.c_size_t, _P]),
    "dyna_static_budget": (_I, [_I, _I]),
    "dyna_token_rows": (_I, [_P, _P, _P]),
    "dyna_verify_workspace_bytes": (_Z, [_I, _I, _I, _I]),
    "dyna_verify_chain": (_I, [_P, _I, _I, _L, _L, _I, _I, _P, _P, _F, _P, _P, _P, _P, _P, _P, _P, _Z, _P]),
    "dyna_verify_tree": (_I, [_P, _I, _I, _L, _L, _I, _I, _P, _P, _I, _F, _P, _P, _P, _P, _P, _P, _Z, _P]),
    "dyna_distill_workspace_bytes": (_Z, [_I, _I]),
    "dyna_distill": (_I, [_P, _I, _I, _L, _I, _P, _P, _I, _I, _I, _F, _P, _P, _P, _P, _L, _P, _Z, _P]),
    "dyna_distill_grad": (_I, [_P, _I, _I, _L, _I, _P, _P, _I, _I, _I, _F, _P, _P, _P, _L, _P]),
    "dyna_router_loss": (_I, [_P, _I, _I, _L, _I, _P, _I, _P, _I, _F, _P, _P, _P, _L, _P]),
    "dyna_quant_bytes": (_Z, [_I, _I]),
    "dyna_quantize_rows": (_I, [_P, _I, _I, _I, _L, _P, _P]),
    "dyna_dequantize_rows": (_I, [_P, _P, _I, _L, _P]),
    "dyna_quant_product_workspace_bytes": (_Z, [_I, _I]),
    "dyna_quant_product": (_I, [_P, _I, _P, _I, _L, _P, _I, _P, _I, _L, _P, _Z, _P]),
    "dyna_quant_shortlist_logits": (_I, [_P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _I, _P, _Z, _P]),
    "dyna_token_logprobs_workspace_bytes": (_Z, [_I, _I, _I, _I]),
    "dyna_token_logprobs": (_I, [_P, _I, _I, _L, _I, _P, _P, _I, _F, _I, _P, _P, _P, _P, _P, _P, _Z, _P]),
    "dyna_token_logprobs_grad": (_I, [_P, _I, _I, _L, _I, _P, _P, _I, _F, _P, _P, _P, _P, _L, _P]),
    "dyna_dense_head": (_I, [_P, _I, _I, _I, _P, _I, _I, _I, _I, _F, _P, _P, _P, _P, _P, _P, _P,
                             _Z, _P]),
}
EXPORTED = tuple(_SIGNATURES)


def lib():
    """Load libdynahead.so (built in-tree).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2510_13847_amd.build` (hipcc, gfx950)")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        if L.dyna_abi_version() != ABI_VERSION:
            raise RuntimeError("libdynahead ABI version mismatch")
        _lib = L
    return _lib


def _check(status: int):
    if status != OK:
        raise DynaError(status, lib().dyna_last_error().decode())


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _stream(stream) -> int:
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _need(t, name, device=True, contiguous=True):
    if t is None:
        raise ValueError(f"{name} is required")
    if device and not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def set_option(option: int, value: int):
    _check(lib().dyna_set_option(option, value))


def kernel_timing(reset=True):
    """(total_ms, launches) of the gathered-head kernel launches timed so far."""
    ms = ctypes.c_double(0.0)
    n = ctypes.c_int64(0)
    _check(lib().dyna_kernel_timing(ctypes.byref(ms), ctypes.byref(n), 1 if reset else 0))
    return ms.value, n.value


# --------------------------------------------------------------------------
@dataclass
class Layout:
    """Device layout from build_layout (tensors are kept alive here).  W_perm None: a head whose rows are kept in
    four bits alone, for the calls that do not read them."""
    V: int
    d: int
    M: int
    W_perm: object
    perm: object
    offsets: object
    cap_by_k: np.ndarray   # host int32 [M + 1]
    max_cluster: int

    def __post_init__(self):
        dtype = BF16 if self.W_perm is None else _dtype_code(self.W_perm)
        self._c = _Layout(self.V, self.d, self.M, dtype, _ptr(self.W_perm), _ptr(self.perm), _ptr(self.offsets),
                          self.cap_by_k.ctypes.data_as(ctypes.c_void_p).value, self.max_cluster)

    def with_weights(self, W_perm) -> "Layout":
        """The same layout over another copy of the permuted head (replicas), or without one (None)."""
        return Layout(self.V, self.d, self.M, W_perm, self.perm, self.offsets, self.cap_by_k,
                      self.max_cluster)

    @property
    def c(self):
        return ctypes.byref(self._c)

    def cap(self, k: int) -> int:
        return int(self.cap_by_k[k])


@dataclass
class Router:
    W1: object
    W2: Optional[object] = None
    b1: Optional[object] = None
    b2: Optional[object] = None
    act: str = "silu"

    def __post_init__(self):
        H = 0 if self.W2 is None else self.W1.shape[0]
        M = self.W1.shape[0] if self.W2 is None else self.W2.shape[0]
        self.d_r, self.H, self.M = self.W1.shape[1], H, M
        self._c = _Router(self.d_r, H, M, _dtype_code(self.W1), ACT[self.act], _ptr(self.W1),
                          _ptr(self.b1), _ptr(self.W2), _ptr(self.b2))

    @property
    def c(self):
        return ctypes.byref(self._c)


# --------------------------------------------------------------------------
def layout_workspace_bytes(V: int, M: int) -> int:
    return int(lib().dyna_layout_workspace_bytes(V, M))


def build_layout(cluster_of, W_lm, M: int, stream=None) -> Layout:
    """dyna_build_layout: cluster-contiguous copy of W_lm [V, d] (synchronous)."""
    import torch
    _need(cluster_of, "cluster_of")
    _need(W_lm, "W_lm")
    V, d = W_lm.shape
    dev = W_lm.device
    W_perm = torch.empty_like(W_lm)
    perm = torch.empty(V, dtype=torch.int32, device=dev)
    offsets = torch.empty(M + 1, dtype=torch.int32, device=dev)
    cap = np.zeros(M + 1, dtype=np.int32)
    mx = ctypes.c_int32(0)
    wsb = layout_workspace_bytes(V, M)
    ws = torch.empty(max(wsb, 1), dtype=torch.uint8, device=dev)
    _check(lib().dyna_build_layout(_ptr(cluster_of), V, M, _ptr(W_lm), _dtype_code(W_lm), d,
                                   _ptr(W_perm), _ptr(perm), _ptr(offsets),
                                   cap.ctypes.data_as(ctypes.c_void_p), ctypes.byref(mx),
                                   _ptr(ws), wsb, _stream(stream)))
    return Layout(V, d, M, W_perm, perm, offsets, cap, int(mx.value))


def workspace_bytes(layout: Optional[Layout], router: Optional[Router], B: int, k: int, cap: int) -> int:
    return int(lib().dyna_workspace_bytes(layout.c if layout else None, router.c if router else None,
                                          B, k, cap))


def workspace(layout, router, B, k, cap, device="cuda"):
    """Zero-filled workspace (the one-context kernels' counters start at zero)."""
    import torch
    n = workspace_bytes(layout, router, B, k, cap)
    return torch.zeros(max(n, 1), dtype=torch.uint8, device=device)


def route(router: Router, x, k: int, ws=None, want_scores=False, stream=None):
    """dyna_route -> (topk_ids [B, k] int32, topk_scores [B, k], scores [B, M] or None)."""
    import torch
    _need(x, "x")
    B = x.shape[0]
    dev = x.device
    ids = torch.empty((B, k), dtype=torch.int32, device=dev)
    sc = torch.empty((B, k), dtype=torch.float32, device=dev)
    scores = torch.empty((B, router.M), dtype=torch.float32, device=dev) if want_scores else None
    if ws is None:
        ws = workspace(None, router, B, k, 0, dev)
    _check(lib().dyna_route(router.c, _ptr(x), _dtype_code(x), B, k, _ptr(ids), _ptr(sc),
                            _ptr(scores), _ptr(ws), ws.numel(), _stream(stream)))
    return ids, sc, scores


def shortlist(layout: Layout, topk_ids, with_ids=True, stream=None):
    """dyna_shortlist -> (sel_sorted, sel_rowoff, row_len, shortlist_ids or None)."""
    import torch
    _need(topk_ids, "topk_ids")
    B, k = topk_ids.shape
    dev = topk_ids.device
    cap = layout.cap(k)
    sel = torch.empty((B, k), dtype=torch.int32, device=dev)
    rowoff = torch.empty((B, k + 1), dtype=torch.int32, device=dev)
    row_len = torch.empty(B, dtype=torch.int32, device=dev)
    ids = torch.full((B, max(cap, 1)), -1, dtype=torch.int32, device=dev) if with_ids else None
    _check(lib().dyna_shortlist(layout.c, _ptr(topk_ids), B, k, _ptr(sel), _ptr(rowoff),
                                _ptr(row_len), _ptr(ids), cap, _stream(stream)))
    return sel, rowoff, row_len, ids


def shortlist_logits(layout: Layout, h, sel_sorted, sel_rowoff, row_len, cap=None, ws=None,
                     out=None, stream=None):
    """dyna_shortlist_logits -> logits [B, cap] fp32 (slots past row_len untouched)."""
    import torch
    _need(h, "h")
    B, k = sel_sorted.shape
    cap = layout.cap(k) if cap is None else cap
    dev = h.device
    if out is None:
        out = torch.full((B, cap), float("nan"), dtype=torch.float32, device=dev)
    if ws is None:
        ws = workspace(layout, None, B, k, cap, dev)
    _check(lib().dyna_shortlist_logits(layout.c, _ptr(h), _dtype_code(h), B, k, _ptr(sel_sorted),
                                       _ptr(sel_rowoff), _ptr(row_len), _ptr(out), cap, _ptr(ws),
                                       ws.numel(), _stream(stream)))
    return out


def _select_outputs(B, k_t, mode, dev):
    import torch
    want_ids = bool(mode & (SEL_ARGMAX | SEL_TOPK))
    kt = k_t if mode & SEL_TOPK else 1
    ids = torch.empty((B, kt), dtype=torch.int32, device=dev) if want_ids else None
    lps = torch.empty((B, kt), dtype=torch.float32, device=dev) if want_ids else None
    smp = torch.empty(B, dtype=torch.int32, device=dev) if mode & SEL_SAMPLE else None
    slp = torch.empty(B, dtype=torch.float32, device=dev) if mode & SEL_SAMPLE else None
    return ids, lps, smp, slp


def draft_select(layout: Layout, logits, sel_sorted, sel_rowoff, row_len, mode=SEL_TOPK, k_t=1,
                 temperature=1.0, uniforms=None, cap=None, ws=None, stream=None, tail_beta=0.0):
    """dyna_draft_select -> dict(ids, logprobs, sample, sample_logprob)."""
    B, k = sel_sorted.shape
    cap = logits.shape[1] if cap is None else cap
    dev = logits.device
    ids, lps, smp, slp = _select_outputs(B, k_t, mode, dev)
    if ws is None:
        ws = workspace(layout, None, B, k, cap, dev)
    _check(lib().dyna_draft_select(layout.c, _ptr(logits), _ptr(sel_sorted), _ptr(sel_rowoff),
                                   _ptr(row_len), B, k, cap, mode, k_t, temperature, tail_beta,
                                   _ptr(uniforms), _ptr(ids), _ptr(lps), _ptr(smp), _ptr(slp),
                                   _ptr(ws), ws.numel(), _stream(stream)))
    return dict(ids=ids, logprobs=lps, sample=smp, sample_logprob=slp)


class DraftHead:
    """Preallocated outputs + workspace for repeated dyna_draft_head calls."""

    def __init__(self, router: Router, layout: Layout, B: int, k: int, mode: int, k_t: int = 1,
                 temperature: float = 1.0, keep_logits=False, keep_clusters=True, device="cuda",
                 tail_beta: float = 0.0):
        import torch
        self.router, self.layout, self.B, self.k = router, layout, B, k
        self.mode, self.k_t, self.temperature, self.tail_beta = mode, k_t, temperature, tail_beta
        # DYNA_SEL_UNION: every row's logits span the step's shared shortlist
        self.cap = union_cap(layout, B, k) if (mode & SEL_UNION) and B > 1 else layout.cap(k)
        self.ids, self.logprobs, self.sample, self.sample_logprob = _select_outputs(B, k_t, mode, device)
        self.clusters = torch.empty((B, k), dtype=torch.int32, device=device) if keep_clusters else None
        self.logits = torch.full((B, self.cap), float("nan"), dtype=torch.float32,
                                 device=device) if keep_logits else None
        self.ws = workspace(layout, router, B, k, self.cap, device)
        self.ran = False  # the outputs hold a step

    def __call__(self, x, h, uniforms=None, stream=None, route_stream=None, x_ready=None,
                 layout: Optional[Layout] = None, router: Optional[Router] = None):
        L = layout or self.layout
        R = router or self.router
        rs = None if route_stream is None else route_stream.cuda_stream
        ev = None if x_ready is None else x_ready.cuda_event
        _check(lib().dyna_draft_head(R.c, L.c, _ptr(x), _ptr(h), _dtype_code(h), self.B, self.k,
                                     self.mode, self.k_t, self.temperature, self.tail_beta, _ptr(uniforms),
                                     _ptr(self.ids), _ptr(self.logprobs), _ptr(self.sample),
                                     _ptr(self.sample_logprob), _ptr(self.clusters),
                                     _ptr(self.logits), self.cap, _ptr(self.ws), self.ws.numel(),
                                     _stream(stream), rs, ev))
        self.ran = True
        return self


NOALLOC_SCRATCH_BYTES = 16 << 20  # DYNA_NOALLOC_SCRATCH_BYTES


def draft_head_noalloc(head: "DraftHead", x, h, uniforms=None, stream=None,
                       layout: Optional[Layout] = None, router: Optional[Router] = None):
    """dyna_draft_head_noalloc into head's preallocated outputs (its own
    workspace is not used: the library's static scratch stands in for it)."""
    L = layout or head.layout
    R = router or head.router
    _check(lib().dyna_draft_head_noalloc(R.c, L.c, _ptr(x), _ptr(h), _dtype_code(h), head.B, head.k,
                                         head.mode, head.k_t, head.temperature, head.tail_beta,
                                         _ptr(uniforms), _ptr(head.ids), _ptr(head.logprobs),
                                         _ptr(head.sample), _ptr(head.sample_logprob), _ptr(head.clusters),
                                         _ptr(head.logits), head.cap, _stream(stream)))
    head.ran = True
    return head


def draft_head(router: Router, layout: Layout, x, h, k: int, mode=SEL_ARGMAX, k_t=1,
               temperature=1.0, uniforms=None, keep_logits=True, stream=None, route_stream=None,
               tail_beta=0.0):
    """One dyna_draft_head call with fresh outputs (see DraftHead for repeated calls)."""
    head = DraftHead(router, layout, h.shape[0], k, mode, k_t, temperature, keep_logits=keep_logits,
                     device=h.device, tail_beta=tail_beta)
    head(x, h, uniforms, stream=stream, route_stream=route_stream)
    return head


def dense_workspace_bytes(n_rows: int, B: int) -> int:
    return int(lib().dyna_dense_workspace_bytes(n_rows, B))


class DenseHead:
    """dyna_dense_head over rows [0, n_rows) of W (dense when n_rows = V)."""

    def __init__(self, W, n_rows: int, B: int, mode: int, k_t: int = 1, temperature: float = 1.0,
                 keep_logits=False, device="cuda"):
        import torch
        self.W, self.n_rows, self.B = W, n_rows, B
        self.mode, self.k_t, self.temperature = mode, k_t, temperature
        self.ids, self.logprobs, self.sample, self.sample_logprob = _select_outputs(B, k_t, mode, device)
        self.logits = torch.empty((B, n_rows), dtype=torch.float32, device=device) if keep_logits else None
        n = dense_workspace_bytes(n_rows, B)
        self.ws = torch.empty(max(n, 1), dtype=torch.uint8, device=device)
        self.ran = False  # the outputs hold a step

    def __call__(self, h, uniforms=None, stream=None, W=None):
        W = self.W if W is None else W
        _check(lib().dyna_dense_head(_ptr(W), _dtype_code(W), self.n_rows, W.shape[1], _ptr(h),
                                     _dtype_code(h), self.B, self.mode, self.k_t, self.temperature,
                                     _ptr(uniforms), _ptr(self.ids), _ptr(self.logprobs),
                                     _ptr(self.sample), _ptr(self.sample_logprob), _ptr(self.logits),
                                     _ptr(self.ws), self.ws.numel(), _stream(stream)))
        self.ran = True
        return self


def cluster_budget(t, k0, k1, k_min=1, form=0):
    """Cluster budget k_c(t) (form 0: the paper's equation, 1: the appendix algorithm's)."""
    v = lib().dyna_cluster_budget(t, k0, k1, k_min, form)
    if v < 0:
        raise ValueError("invalid cluster budget arguments")
    return v


def static_budget(t, k_max):
    """PA-FR static shortlist size K_fr(t)."""
    v = lib().dyna_static_budget(t, k_max)
    if v < 0:
        raise ValueError("invalid static budget arguments")
    return v


def union_cap(layout: "Layout", B: int, k: int) -> int:
    """Logits row stride a DYNA_SEL_UNION step of B rows needs: min(V, B * cap_by_k[k])."""
    return min(layout.V, B * layout.cap(k))


def beam_expand(logprobs, ids, last_scores=None, n_out=None, stream=None, out=None):
    """dyna_beam_expand -> (scores[n_out], parent[n_out], ids[n_out]); out: an
    existing (scores, parent, ids) triple to write instead of fresh tensors."""
    import torch
    B, k_t = logprobs.shape
    n_out = k_t if n_out is None else n_out
    dev = logprobs.device
    if out is not None:
        sc, par, tok = out
        for t, dt in zip(out, (torch.float32, torch.int32, torch.int32)):
            _need(t, "out")
            if t.dtype != dt or t.numel() < n_out:
                raise ValueError("beam_expand: out tensors must be (float32, int32, int32) of n_out entries")
    else:
        sc = torch.empty(n_out, dtype=torch.float32, device=dev)
        par = torch.empty(n_out, dtype=torch.int32, device=dev)
        tok = torch.empty(n_out, dtype=torch.int32, device=dev)
    _check(lib().dyna_beam_expand(_ptr(logprobs), _ptr(ids), _ptr(last_scores), B, k_t, n_out, _ptr(sc),
                                  _ptr(par), _ptr(tok), _stream(stream)))
    return sc, par, tok


# ---------------------------------------------------------------- partition builder
def kmeans_workspace(W, M: int):
    import torch
    V, d = W.shape
    n = int(lib().dyna_kmeans_workspace_bytes(V, d, M))
    return torch.empty(max(n, 1), dtype=torch.uint8, device=W.device)


def kmeans_assign(W, centroids, ws=None, stream=None, want_score=False):
    """dyna_kmeans_assign -> (assign[V] int32, score[V] float32 or None)."""
    import torch
    V, d = W.shape
    M = centroids.shape[0]
    ws = kmeans_workspace(W, M) if ws is None else ws
    a = torch.empty(V, dtype=torch.int32, device=W.device)
    sc = torch.empty(V, dtype=torch.float32, device=W.device) if want_score else None
    _check(lib().dyna_kmeans_assign(_ptr(W), _dtype_code(W), V, d, _ptr(centroids), M, _ptr(a), _ptr(sc),
                                    _ptr(ws), ws.numel(), _stream(stream)))
    return a, sc


def kmeans_update(W, assign, centroids, ws=None, stream=None):
    """dyna_kmeans_update, in place on centroids (fp32 [M, d])."""
    V, d = W.shape
    M = centroids.shape[0]
    ws = kmeans_workspace(W, M) if ws is None else ws
    _check(lib().dyna_kmeans_update(_ptr(W), _dtype_code(W), V, d, _ptr(assign), M, _ptr(centroids), _ptr(ws),
                                    ws.numel(), _stream(stream)))
    return centroids


def kmeans(W, M: int, init_ids, iters: int, ws=None, stream=None, keep_centroids=True):
    """dyna_kmeans -> (cluster_of[V] int32, centroids[M, d] float32 or None)."""
    import torch
    V, d = W.shape
    ws = kmeans_workspace(W, M) if ws is None else ws
    cl = torch.empty(V, dtype=torch.int32, device=W.device)
    mu = torch.empty((M, d), dtype=torch.float32, device=W.device) if keep_centroids else None
    _check(lib().dyna_kmeans(_ptr(W), _dtype_code(W), V, d, M, _ptr(init_ids), iters, _ptr(cl), _ptr(mu),
                             _ptr(ws), ws.numel(), _stream(stream)))
    return cl, mu


# ---------------------------------------------------------------- verification with the target model
def _typed(t, name, dtype, shape, device):
    """A contiguous tensor of this dtype, shape and device."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")


def _dims(t, name, n):
    _need(t, name, contiguous=False)
    if t.dim() != n:
        raise ValueError(f"{name} must have {n} dimension{'s' if n > 1 else ''}")
    return t.shape


def _stream_device(stream, device):
    if stream.device != device:
        raise ValueError(f"stream is on {stream.device}, the tensors are on {device}")


def _launch(device, call, *args):
    """call(*args, stream) on the device of its tensors (made the current one for
    the time of the call) and that device's current stream."""
    import torch
    stream = torch._C._cuda_getCurrentRawStream(device.index)
    if device.index == torch._C._cuda_getDevice():
        _check(call(*args, stream))
    else:
        with torch.cuda.device(device):
            _check(call(*args, stream))


@dataclass
class DraftStep:
    """One drafted position of B chains, as a draft head wrote it (tensors are
    kept alive here): the sampled tokens with the log-probability of each, the
    draft logits they were sampled from and the clusters those span.  Tokens
    alone are drafts proposed outright (argmax drafts)."""
    tokens: object
    logprobs: Optional[object] = None
    logits: Optional[object] = None
    clusters: Optional[object] = None
    temperature: float = 1.0
    tail_beta: float = 0.0
    shared: bool = False

    def __post_init__(self):
        import torch
        (B,), dev, k, cap = _dims(self.tokens, "tokens", 1), self.tokens.device, 0, 0
        _typed(self.tokens, "tokens", torch.int32, (B,), dev)
        if self.logits is not None:
            cap = _dims(self.logits, "logits", 2)[1]
            _typed(self.logits, "logits", torch.float32, (B, cap), dev)
            _need(self.logprobs, "logprobs")
            _typed(self.logprobs, "logprobs", torch.float32, (B,), dev)
        if self.clusters is not None:
            k = _dims(self.clusters, "clusters", 2)[1]
            _typed(self.clusters, "clusters", torch.int32, (B, k), dev)
        self.B, self.device = B, dev
        self._c = _DraftStep(_ptr(self.tokens), _ptr(self.logprobs), _ptr(self.logits), _ptr(self.clusters), k, cap,
                             int(self.shared), self.temperature, self.tail_beta)

    @classmethod
    def of(cls, head, stream=None) -> "DraftStep":
        """The step that the last run of a DraftHead (keep_logits, keep_clusters)
        or DenseHead (keep_logits) wrote: its sample and the distribution it came
        from, or its best tokens, proposed outright, when it does not sample.

        The step is a copy, made on `stream` (the head's): the head may run again,
        for the next position.  A head that runs once a cycle needs no copy:
        DraftStep(head.sample, head.sample_logprob, head.logits, head.clusters, ...)
        stands for whatever its buffers hold when the chain is judged."""
        if not head.ran:
            raise ValueError("the head has not run: its step is taken behind the run")
        if stream is not None:
            import torch
            _stream_device(stream, (head.ids if head.sample is None else head.sample).device)
            with torch.cuda.stream(stream):
                return cls.of(head)
        if head.sample is None:
            return cls(head.ids[:, 0].clone())
        if head.logits is None or (isinstance(head, DraftHead) and head.clusters is None):
            raise ValueError("a sampled step needs a head that keeps its logits and clusters")
        sampled = head.sample.clone(), head.sample_logprob.clone(), head.logits.clone()
        if isinstance(head, DenseHead):
            return cls(*sampled, temperature=head.temperature)
        return cls(*sampled, head.clusters.clone(), head.temperature, head.tail_beta,
                   bool(head.mode & SEL_UNION) and head.B > 1)


def token_rows(layout: Layout, stream=None):
    """dyna_token_rows -> [V, 2] int32: (cluster, layout row) of every token."""
    import torch
    if stream is not None:
        _stream_device(stream, layout.perm.device)
        with torch.cuda.stream(stream):
            return token_rows(layout)
    out = torch.empty((layout.V, 2), dtype=torch.int32, device=layout.perm.device)
    _launch(out.device, lib().dyna_token_rows, layout.c, _ptr(out))
    return out


def verify_workspace(B, rows, V, M=0, device="cuda"):
    import torch
    n = int(lib().dyna_verify_workspace_bytes(B, rows, V, M))
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device)


class _Verifier:
    def __init__(self, B, rows, V, temperature, M, device):
        import torch
        self.B, self.rows, self.V, self.temperature = B, rows, V, float(temperature)
        if self.temperature != 0.0 and _F(self.temperature).value == 0.0:
            raise ValueError(f"temperature {temperature} is 0 in 32 bits, which would ask for greedy verification")
        dev = torch.empty(0, device=device).device
        self.device = dev
        self.lengths = torch.empty(B, dtype=torch.int32, device=dev)
        self.ids = torch.empty((B, rows), dtype=torch.int32, device=dev)
        self.logprobs = torch.empty((B, rows), dtype=torch.float32, device=dev)
        self.ws = verify_workspace(B, rows, V, M, dev)

    def _inputs(self, target, uniforms):
        """The target's dtype code and strides, after the checks both forms share."""
        import torch
        if not target.is_cuda:
            raise ValueError("target must be a device tensor")
        if target.device != self.device:
            raise ValueError(f"target is on {target.device}, not on {self.device}")
        if target.shape != (self.B, self.rows, self.V):
            raise ValueError(f"target must have shape {(self.B, self.rows, self.V)}, not {tuple(target.shape)}")
        batch, row, one = target.stride()
        if one != 1 and self.V > 1:
            raise ValueError("target's last dimension must be contiguous")
        if uniforms is not None:
            _typed(uniforms, "uniforms", torch.float32, (self.B, self.rows), self.device)
        elif self.temperature > 0.0:
            raise ValueError("uniforms are required with a temperature above 0")
        return _dtype_code(target), row, batch


class ChainVerifier(_Verifier):
    """Preallocated outputs + workspace for repeated dyna_verify_chain calls:
    lengths [B], ids and logprobs [B, n + 1].  temperature 0 is greedy; layout
    is that of the draft heads whose logits span clusters: its token rows are
    made here, and waited for (verify_chain does so in every call)."""

    def __init__(self, B: int, n: int, V: int, temperature: float = 1.0, layout: Optional[Layout] = None,
                 device="cuda"):
        import torch
        if layout is not None:
            at = torch.empty(0, device=device).device
            if layout.perm.device != at:
                raise ValueError(f"layout is on {layout.perm.device}, not on {at}")
        super().__init__(B, n + 1, V, temperature, layout.M if layout is not None else 0, device)
        self.n, self.layout = n, layout
        self.token_rows = token_rows(layout) if layout is not None else None
        if layout is not None and not torch.cuda.is_current_stream_capturing():
            # calls on other streams read it too
            torch.cuda.current_stream(self.device).synchronize()
        self._steps = (_DraftStep * max(n, 1))()
        self._fixed = (layout.c if layout is not None else None, _ptr(self.token_rows), _ptr(self.lengths),
                       _ptr(self.ids), _ptr(self.logprobs), _ptr(self.ws), self.ws.numel())

    def __call__(self, target, steps, uniforms=None, lens=None, stream=None):
        """target [B, n + 1, V] logits, steps: n DraftSteps, uniforms [B, n + 1],
        lens [B] int32 (drafts of each request)."""
        import torch
        if stream is not None:
            _stream_device(stream, self.device)
            with torch.cuda.stream(stream):
                return self(target, steps, uniforms, lens)
        code, row, batch = self._inputs(target, uniforms)
        if lens is not None:
            _typed(lens, "lens", torch.int32, (self.B,), self.device)
        if len(steps) != self.n:
            raise ValueError(f"{len(steps)} steps, not {self.n}")
        for i, s in enumerate(steps):
            if s.B != self.B:
                raise ValueError(f"step {i} has {s.B} rows, not {self.B}")
            if s.device != self.device:
                raise ValueError(f"step {i} is on {s.device}, not on {self.device}")
            if s.clusters is not None and self.layout is None:
                raise ValueError(f"step {i} has clusters: the verifier needs their layout")
            self._steps[i] = s._c
        _launch(self.device, lib().dyna_verify_chain, _ptr(target), code, self.V, row, batch, self.B, self.n,
                self._steps, _ptr(lens), self.temperature, *self._fixed[:2], _ptr(uniforms), *self._fixed[2:])
        return self


class TreeVerifier(_Verifier):
    """Preallocated outputs + workspace for repeated dyna_verify_tree calls:
    lengths [B]; ids, logprobs and nodes [B, N]."""

    def __init__(self, B: int, N: int, V: int, temperature: float = 1.0, device="cuda"):
        import torch
        super().__init__(B, N, V, temperature, 0, device)
        self.N = N
        self.nodes = torch.empty((B, N), dtype=torch.int32, device=self.device)
        self._fixed = (_ptr(self.lengths), _ptr(self.ids), _ptr(self.logprobs), _ptr(self.nodes), _ptr(self.ws),
                       self.ws.numel())

    def __call__(self, target, tokens, parents, uniforms=None, stream=None):
        """target [B, N, V] logits, tokens [B, N], parents [N] or [B, N], uniforms [B, N]."""
        import torch
        if stream is not None:
            _stream_device(stream, self.device)
            with torch.cuda.stream(stream):
                return self(target, tokens, parents, uniforms)
        code, row, batch = self._inputs(target, uniforms)
        _typed(tokens, "tokens", torch.int32, (self.B, self.N), self.device)
        shared = parents.dim() == 1
        _typed(parents, "parents", torch.int32, (self.N,) if shared else (self.B, self.N), self.device)
        _launch(self.device, lib().dyna_verify_tree, _ptr(target), code, self.V, row, batch, self.B, self.N,
                _ptr(tokens), _ptr(parents), 0 if shared else self.N, self.temperature, _ptr(uniforms), *self._fixed)
        return self


def verify_chain(target, steps, uniforms=None, lens=None, temperature=1.0, layout=None, stream=None):
    """One dyna_verify_chain call with fresh outputs (see ChainVerifier for repeated calls)."""
    if stream is not None:  # the outputs and the workspace are that stream's too
        import torch
        _stream_device(stream, target.device)
        with torch.cuda.stream(stream):
            return verify_chain(target, steps, uniforms, lens, temperature, layout)
    v = ChainVerifier(target.shape[0], len(steps), target.shape[2], temperature, layout, target.device)
    return v(target, steps, uniforms, lens)


def verify_tree(target, tokens, parents, uniforms=None, temperature=1.0, stream=None):
    """One dyna_verify_tree call with fresh outputs (see TreeVerifier for repeated calls)."""
    if stream is not None:  # the outputs and the workspace are that stream's too
        import torch
        _stream_device(stream, target.device)
        with torch.cuda.stream(stream):
            return verify_tree(target, tokens, parents, uniforms, temperature)
    v = TreeVerifier(target.shape[0], target.shape[1], target.shape[2], temperature, target.device)
    return v(target, tokens, parents, uniforms)


# ---------------------------------------------------------------- learning from the target's top tokens
def _matrix(t, name):
    """A [rows, cols] device tensor with contiguous rows -> (dtype code, row stride)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return _dtype_code(t), (t.stride(0) if t.shape[0] > 1 else t.shape[1])


def _gradient(out, t):
    """The gradient to write (a fresh one without `out`) and its row stride."""
    import torch
    if out is None:
        return torch.empty(t.shape, dtype=t.dtype, device=t.device), t.shape[1]
    if out.shape != t.shape or out.dtype != t.dtype:
        raise ValueError("out must have the shape and dtype of its input")
    stride = _matrix(out, "out")[1]
    if out.device != t.device:
        raise ValueError(f"out is on {out.device}, not on {t.device}")
    return out, stride


def distill_workspace(N: int, V: int, device="cuda"):
    import torch
    return torch.empty(max(int(lib().dyna_distill_workspace_bytes(N, V)), 1), dtype=torch.uint8, device=device)


def _teacher_list(t, ids, values, weights):
    """Checks a teacher's list against rows t -> entries of each row."""
    import torch
    N, dev = t.shape[0], t.device
    K = _dims(ids, "ids", 2)[1]
    _typed(ids, "ids", torch.int32, (N, K), dev)
    if values is not None:
        _typed(values, "values", torch.bfloat16 if values.dtype is torch.bfloat16 else torch.float32, (N, K), dev)
    if weights is not None:
        _typed(weights, "weights", torch.float32, (N,), dev)
    return K


def distill(logits, ids, values, temperature=1.0, tail=False, weights=None, want_grad=True, want_stats=False,
            out=None, ws=None, stream=None):
    """dyna_distill -> (loss [N], stats [N, 2] or None, grad [N, V] or None).

    logits [N, V]: the student's; ids, values [N, K]: the teacher's top list, as
    DenseHead's top-k_t writes it; weights [N]: d objective / d loss of each row
    (0: padding).  grad is weights * d loss / d logits: the training loop passes
    it on with ``logits.backward(grad)``.  out: an existing gradient to write."""
    import torch
    dev = logits.device
    if stream is not None:
        _stream_device(stream, dev)
        with torch.cuda.stream(stream):
            return distill(logits, ids, values, temperature, tail, weights, want_grad, want_stats, out, ws)
    code, stride = _matrix(logits, "logits")
    K = _teacher_list(logits, ids, values, weights)
    N, V = logits.shape
    loss = torch.empty(N, dtype=torch.float32, device=dev)
    stats = torch.empty((N, 2), dtype=torch.float64, device=dev) if want_stats else None
    grad, gstride = _gradient(out, logits) if want_grad else (None, V)
    if ws is None:
        ws = distill_workspace(N, V, dev)
    elif ws.device != dev:
        raise ValueError(f"ws is on {ws.device}, not on {dev}")
    _launch(dev, lib().dyna_distill, _ptr(logits), code, V, stride, N, _ptr(ids), _ptr(values), _dtype_code(values),
            K, int(tail), temperature, _ptr(weights), _ptr(loss), _ptr(stats), _ptr(grad), gstride, _ptr(ws),
            ws.numel())
    return loss, stats, grad


def distill_grad(logits, stats, ids, values, temperature=1.0, tail=False, weights=None, out=None, stream=None):
    """dyna_distill_grad -> grad [N, V], from the stats of an earlier distill call."""
    import torch
    dev = logits.device
    if stream is not None:
        _stream_device(stream, dev)
        with torch.cuda.stream(stream):
            return distill_grad(logits, stats, ids, values, temperature, tail, weights, out)
    code, stride = _matrix(logits, "logits")
    K = _teacher_list(logits, ids, values, weights)
    N, V = logits.shape
    _typed(stats, "stats", torch.float64, (N, 2), dev)
    grad, gstride = _gradient(out, logits)
    _launch(dev, lib().dyna_distill_grad, _ptr(logits), code, V, stride, N, _ptr(ids), _ptr(values),
            _dtype_code(values), K, int(tail), temperature, _ptr(weights), _ptr(stats), _ptr(grad), gstride)
    return grad


def router_loss(scores, ids, cluster_of, pos_weight=1.0, weights=None, want_grad=True, out=None, stream=None):
    """dyna_router_loss -> (loss [N], grad [N, M] or None).

    scores [N, M]: the router's; ids [N, L]: the teacher's top tokens, whose
    clusters are the labels; grad as in distill (out may be `scores` itself)."""
    import torch
    dev = scores.device
    if stream is not None:
        _stream_device(stream, dev)
        with torch.cuda.stream(stream):
            return router_loss(scores, ids, cluster_of, pos_weight, weights, want_grad, out)
    code, stride = _matrix(scores, "scores")
    L = _teacher_list(scores, ids, None, weights)
    V = _dims(cluster_of, "cluster_of", 1)[0]
    _typed(cluster_of, "cluster_of", torch.int32, (V,), dev)
    N, M = scores.shape
    loss = torch.empty(N, dtype=torch.float32, device=dev)
    grad, gstride = _gradient(out, scores) if want_grad else (None, M)
    _launch(dev, lib().dyna_router_loss, _ptr(scores), code, M, stride, N, _ptr(ids), L, _ptr(cluster_of), V,
            pos_weight, _ptr(weights), _ptr(loss), _ptr(grad), gstride)
    return loss, grad


# ---------------------------------------------------------------- four-bit rows
_EMPTY_WS = 256  # bytes of a workspace that nothing reads


@dataclass
class QuantRows:
    """Four-bit rows (quantize_rows; the tensor is kept alive here): 17 bytes to 32 columns, in the library's
    own order."""
    rows: int
    d: int
    data: object

    def __post_init__(self):
        import torch
        n = quant_bytes(self.rows, self.d)
        if n == 0:
            raise ValueError(f"four-bit rows of shape {(self.rows, self.d)} are not supported")
        if self.data.dtype is not torch.uint8 or not self.data.is_contiguous() or self.data.numel() < n:
            raise ValueError(f"data must be {n} contiguous bytes")
        self._c = _Quant(self.rows, self.d, _ptr(self.data))

    @property
    def c(self):
        return ctypes.byref(self._c)

    @property
    def device(self):
        return self.data.device


def quant_bytes(rows: int, d: int) -> int:
    return int(lib().dyna_quant_bytes(rows, d))


def _on(stream, device):
    """The context of a call on `stream`, checked against the tensors' device."""
    import torch
    _stream_device(stream, device)
    return torch.cuda.stream(stream)


def _quant(q, name, device):
    if not isinstance(q, QuantRows):
        raise TypeError(f"{name} must be QuantRows, not {type(q).__name__}")
    if not q.data.is_cuda:
        raise ValueError(f"{name} must be on a device")
    if q.device != device:
        raise ValueError(f"{name} is on {q.device}, not on {device}")


def quantize_rows(x, out: Optional[QuantRows] = None, stream=None) -> QuantRows:
    """dyna_quantize_rows: x [rows, d] (fp32 or bf16, contiguous rows) in four-bit form; out: rows of the same
    shape to write again."""
    import torch
    code, stride = _matrix(x, "x")
    if stream is not None:
        with _on(stream, x.device):
            return quantize_rows(x, out)
    rows, d = x.shape
    if out is None:
        out = QuantRows(rows, d, torch.empty(quant_bytes(rows, d), dtype=torch.uint8, device=x.device))
    else:
        _quant(out, "out", x.device)
        if (out.rows, out.d) != (rows, d):
            raise ValueError(f"out has shape {(out.rows, out.d)}, not {(rows, d)}")
    _launch(x.device, lib().dyna_quantize_rows, _ptr(x), code, rows, d, stride, _ptr(out.data))
    return out


def dequantize_rows(q: QuantRows, dtype=None, out=None, stream=None):
    """dyna_dequantize_rows -> the values that q stands for, [rows, d] in dtype (fp32 or bf16, fp32 by default)
    or in `out`."""
    import torch
    _quant(q, "q", getattr(q, "device", None))
    if stream is not None:
        with _on(stream, q.device):
            return dequantize_rows(q, dtype, out)
    if out is None:
        out = torch.empty((q.rows, q.d), dtype=torch.float32 if dtype is None else dtype, device=q.device)
    elif out.shape != (q.rows, q.d) or (dtype is not None and out.dtype != dtype):
        raise ValueError(f"out must have shape {(q.rows, q.d)}" + (f" and be {dtype}" if dtype is not None else ""))
    code, stride = _matrix(out, "out")
    if out.device != q.device:
        raise ValueError(f"out is on {out.device}, not on {q.device}")
    _launch(q.device, lib().dyna_dequantize_rows, q.c, _ptr(out), code, stride)
    return out


def quant_product_workspace(B: int, d: int, device="cuda"):
    import torch
    n = int(lib().dyna_quant_product_workspace_bytes(B, d))
    return torch.empty(max(n, _EMPTY_WS), dtype=torch.uint8, device=device)


def quant_product(a, W: QuantRows, n_rows: Optional[int] = None, out=None, out_dtype=None, ws=None, stream=None):
    """dyna_quant_product -> [B, n_rows]: contexts a ([B, d] fp32 or bf16, or QuantRows) times the first n_rows
    four-bit rows (all of them by default); the result is fp32, out_dtype or `out`."""
    import torch
    _quant(W, "W", getattr(W, "device", None))
    dev = W.device
    if stream is not None:
        with _on(stream, dev):
            return quant_product(a, W, n_rows, out, out_dtype, ws)
    four = isinstance(a, QuantRows)
    if four:
        _quant(a, "a", dev)
        B, d, code, stride = a.rows, a.d, 0, 0
    else:
        code, stride = _matrix(a, "a")
        B, d = a.shape
        if a.device != dev:
            raise ValueError(f"a is on {a.device}, not on {dev}")
    if d != W.d:
        raise ValueError(f"a has {d} columns, W {W.d}")
    n_rows = W.rows if n_rows is None else n_rows
    if out is None:
        out = torch.empty((B, n_rows), dtype=torch.float32 if out_dtype is None else out_dtype, device=dev)
    elif out.shape != (B, n_rows) or (out_dtype is not None and out.dtype != out_dtype):
        raise ValueError(f"out must have shape {(B, n_rows)}" + (f" and be {out_dtype}" if out_dtype is not None else ""))
    ocode, ostride = _matrix(out, "out")
    if out.device != dev:
        raise ValueError(f"out is on {out.device}, not on {dev}")
    if ws is None:
        ws = quant_product_workspace(1 if four else B, d, dev)
    elif ws.device != dev:
        raise ValueError(f"ws is on {ws.device}, not on {dev}")
    _launch(dev, lib().dyna_quant_product, W.c, n_rows, None if four else _ptr(a), code, stride, a.c if four else None,
            B, _ptr(out), ocode, ostride, _ptr(ws), ws.numel())
    return out


def quant_shortlist_logits(layout: Layout, W: QuantRows, h, sel_sorted, sel_rowoff, row_len, cap=None, ws=None,
                           out=None, stream=None):
    """dyna_quant_shortlist_logits -> logits [B, cap] fp32 (slots past row_len untouched): shortlist_logits over
    four-bit rows, W = quantize_rows(layout.W_perm); ws = workspace(layout, None, B, k, cap).  W_perm is not read:
    layout.with_weights(None) lets go of it."""
    import torch
    _quant(W, "W", getattr(W, "device", None))
    dev = W.device
    if stream is not None:
        with _on(stream, dev):
            return quant_shortlist_logits(layout, W, h, sel_sorted, sel_rowoff, row_len, cap, ws, out)
    if layout.perm.device != dev:
        raise ValueError(f"layout is on {layout.perm.device}, not on {dev}")
    B, k = _dims(sel_sorted, "sel_sorted", 2)
    _typed(sel_sorted, "sel_sorted", torch.int32, (B, k), dev)
    _typed(sel_rowoff, "sel_rowoff", torch.int32, (B, k + 1), dev)
    _typed(row_len, "row_len", torch.int32, (B,), dev)
    _typed(h, "h", torch.bfloat16 if h.dtype is torch.bfloat16 else torch.float32, (B, layout.d), dev)
    if out is None:
        cap = layout.cap(k) if cap is None else cap
        out = torch.full((B, cap), float("nan"), dtype=torch.float32, device=dev)
    else:
        cap = out.shape[1] if cap is None else cap
        _typed(out, "out", torch.float32, (B, cap), dev)
    if ws is None:
        ws = workspace(layout, None, B, k, cap, dev)
    elif ws.device != dev:
        raise ValueError(f"ws is on {ws.device}, not on {dev}")
    _launch(dev, lib().dyna_quant_shortlist_logits, layout.c, W.c, _ptr(h), _dtype_code(h), B, k, _ptr(sel_sorted),
            _ptr(sel_rowoff), _ptr(row_len), _ptr(out), cap, _ptr(ws), ws.numel())
    return out


# ---------------------------------------------------------------- log-probabilities of given tokens
@dataclass
class ShortlistRows:
    """The shortlists that rows of draft logits span, as shortlist() wrote them for each row; one row of them
    stands for every row of logits (a step whose rows share their union: shortlist(layout, clusters.view(1, -1))).
    token_rows: token_rows(layout), made here (and waited for) when not given."""
    layout: Layout
    sel_sorted: object
    sel_rowoff: object
    row_len: object
    token_rows: Optional[object] = None

    def __post_init__(self):
        import torch
        dev = self.layout.perm.device
        N, k = _dims(self.sel_sorted, "sel_sorted", 2)
        _typed(self.sel_sorted, "sel_sorted", torch.int32, (N, k), dev)
        _typed(self.sel_rowoff, "sel_rowoff", torch.int32, (N, k + 1), dev)
        _typed(self.row_len, "row_len", torch.int32, (N,), dev)
        if self.token_rows is None:
            self.token_rows = token_rows(self.layout)
            if not torch.cuda.is_current_stream_capturing():
                # calls on other streams read it too
                torch.cuda.current_stream(dev).synchronize()
        _typed(self.token_rows, "token_rows", torch.int32, (self.layout.V, 2), dev)
        self.N, self.device = N, dev
        self._c = _ShortlistRows(ctypes.addressof(self.layout._c), _ptr(self.token_rows), _ptr(self.sel_sorted),
                                 _ptr(self.sel_rowoff), _ptr(self.row_len), k, int(N == 1))


def _shortlist_arg(rows, N, device):
    """The C argument for rows of logits (None without shortlists)."""
    if rows is None:
        return None
    if rows.device != device:
        raise ValueError(f"rows are on {rows.device}, the logits on {device}")
    if rows.N not in (1, N):
        raise ValueError(f"rows holds {rows.N} shortlists for {N} rows of logits")
    return ctypes.byref(rows._c)


@dataclass
class TokenLogprobs:
    """logprobs [N, T], entropy [N]; top_ids and top_logprobs [N, top] or None; stats [N, 3] for
    token_logprobs_grad or None."""
    logprobs: object
    entropy: object
    top_ids: Optional[object] = None
    top_logprobs: Optional[object] = None
    stats: Optional[object] = None


def token_logprobs_workspace(N: int, V: int, T: int = 1, top: int = 0, device="cuda"):
    import torch
    n = int(lib().dyna_token_logprobs_workspace_bytes(N, V, T, top))
    return torch.empty(max(n, _EMPTY_WS), dtype=torch.uint8, device=device)


def token_logprobs(logits, tokens, temperature=1.0, top=0, rows: Optional[ShortlistRows] = None, want_stats=False,
                   ws=None, stream=None) -> TokenLogprobs:
    """dyna_token_logprobs: log-probabilities of tokens [N, T] (or [N]) in softmax(logits / temperature), the rows'
    entropy and their `top` best tokens.  rows: the shortlists that the logits span (tokens are vocabulary ids all
    the same); want_stats: keep what token_logprobs_grad needs."""
    import torch
    code, stride = _matrix(logits, "logits")
    dev = logits.device
    if stream is not None:
        with _on(stream, dev):
            return token_logprobs(logits, tokens, temperature, top, rows, want_stats, ws)
    N, V = logits.shape
    shape = _token_shape(tokens, N, dev)
    T = shape[1] if len(shape) == 2 else 1
    out = TokenLogprobs(torch.empty(shape, dtype=torch.float32, device=dev),
                        torch.empty(N, dtype=torch.float32, device=dev))
    if top > 0:
        out.top_ids = torch.empty((N, top), dtype=torch.int32, device=dev)
        out.top_logprobs = torch.empty((N, top), dtype=torch.float32, device=dev)
    if want_stats:
        out.stats = torch.empty((N, 3), dtype=torch.float64, device=dev)
    if ws is None:
        ws = token_logprobs_workspace(N, V, T, top, dev)
    elif ws.device != dev:
        raise ValueError(f"ws is on {ws.device}, not on {dev}")
    _launch(dev, lib().dyna_token_logprobs, _ptr(logits), code, V, stride, N, _shortlist_arg(rows, N, dev), _ptr(tokens),
            T, temperature, top, _ptr(out.logprobs), _ptr(out.entropy), _ptr(out.top_ids), _ptr(out.top_logprobs),
            _ptr(out.stats), _ptr(ws), ws.numel())
    return out


def _token_shape(tokens, N, device):
    import torch
    if tokens.dim() not in (1, 2):
        raise ValueError("tokens must have one or two dimensions")
    shape = (N,) if tokens.dim() == 1 else (N, tokens.shape[1])
    _typed(tokens, "tokens", torch.int32, shape, device)
    return shape


def token_logprobs_grad(logits, stats, tokens, grad_logprobs, grad_entropy=None, temperature=1.0,
                        rows: Optional[ShortlistRows] = None, out=None, stream=None):
    """dyna_token_logprobs_grad -> the gradient [N, V] of sum(grad_logprobs * logprobs) + sum(grad_entropy * entropy)
    with respect to the logits, from the stats of a token_logprobs call: the training loop passes it on with
    ``logits.backward(grad)``.  out: an existing gradient to write."""
    import torch
    code, stride = _matrix(logits, "logits")
    dev = logits.device
    if stream is not None:
        with _on(stream, dev):
            return token_logprobs_grad(logits, stats, tokens, grad_logprobs, grad_entropy, temperature, rows, out)
    N, V = logits.shape
    shape = _token_shape(tokens, N, dev)
    T = shape[1] if len(shape) == 2 else 1
    _typed(stats, "stats", torch.float64, (N, 3), dev)
    _typed(grad_logprobs, "grad_logprobs", torch.float32, shape, dev)
    if grad_entropy is not None:
        _typed(grad_entropy, "grad_entropy", torch.float32, (N,), dev)
    if out is None and rows is not None:
        out = torch.zeros(logits.shape, dtype=logits.dtype, device=dev)  # nothing is written behind a shortlist
    grad, gstride = _gradient(out, logits)
    _launch(dev, lib().dyna_token_logprobs_grad, _ptr(logits), code, V, stride, N, _shortlist_arg(rows, N, dev),
            _ptr(tokens), T, temperature, _ptr(stats), _ptr(grad_logprobs), _ptr(grad_entropy), _ptr(grad), gstride)
    return grad
