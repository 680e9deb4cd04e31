"""ctypes binding of libmoespec.so: argument marshalling only.

Every function takes torch tensors living on the GPU (device memory and streams are PyTorch's
job here), checks dtype / shape / contiguity, passes raw pointers and sizes through the C ABI and
raises ``MoeSpecError`` on a non-zero status.  No step of the method is computed in Python.
The library must have been built (``python -m paper_2602_16052_amd.build``); there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, Structure, c_char_p, c_float, c_int32, c_int64, c_size_t, c_void_p
from dataclasses import dataclass
from typing import Dict, Optional

import torch

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libmoespec.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED_SHAPE, ERR_WORKSPACE_TOO_SMALL, ERR_HIP = range(5)
F32, BF16 = 0, 1
TRUNCATE, SUBSTITUTE = 0, 1
GATE_SOFTMAX, GATE_SIGMOID = 0, 1
BLOCK_GATE_NONE, BLOCK_GATE_CHANNEL, BLOCK_GATE_TOKEN, BLOCK_GATE_ELEMENT = range(4)
CACHE_PLAIN, CACHE_I8, CACHE_E4M3 = range(3)

EXPORTS = ("moespec_abi_version", "moespec_status_string", "moespec_check_desc", "moespec_workspace_bytes",
           "moespec_route", "moespec_budget", "moespec_expert_ffn", "moespec_layer_forward",
           "moespec_layer_forward_traced", "moespec_layer_forward_static", "moespec_stack_forward", "moespec_rms_scale",
           "moespec_calibration_count", "moespec_static_shortlist", "moespec_coverage_curve",
           "moespec_reconstruction_error", "moespec_oracle_ranking", "moespec_stream_read",
           "moespec_check_attn_desc", "moespec_attn_workspace_bytes", "moespec_tree_attention", "moespec_cache_weights",
           "moespec_cache_commit", "moespec_evict_workspace_bytes", "moespec_cache_evict", "moespec_block_norm",
           "moespec_head_rope", "moespec_paged_write", "moespec_paged_read", "moespec_paged_attention_workspace_bytes",
           "moespec_paged_attention", "moespec_verify_workspace_bytes", "moespec_draft_verify")


class MoeSpecError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class Desc(Structure):
    _fields_ = [("d", c_int32), ("n_experts", c_int32), ("top_k", c_int32), ("d_ff", c_int32),
                ("dtype", c_int32), ("renorm", c_int32), ("gate", c_int32)]


class Weights(Structure):
    _fields_ = [("w_router", c_void_p), ("b_router", c_void_p), ("w_gate", c_void_p), ("w_up", c_void_p),
                ("w_down", c_void_p)]


class Taps(Structure):
    _fields_ = [("probs", c_void_p), ("scores", c_void_p), ("budget_ids", c_void_p), ("tok_ids", c_void_p),
                ("tok_w", c_void_p), ("seg_expert", c_void_p), ("seg_off", c_void_p), ("perm", c_void_p),
                ("n_loaded", c_void_p)]


class CAttnDesc(Structure):
    _fields_ = [("n_heads", c_int32), ("n_kv_heads", c_int32), ("head_dim", c_int32), ("capacity", c_int32),
                ("dtype", c_int32), ("scale", c_float)]


class Tree(Structure):
    _fields_ = [("n_seq", c_int32), ("n_tokens", c_int32), ("max_tree", c_int32), ("q_stride", c_int64),
                ("kv_stride", c_int64), ("tree_off", c_void_p), ("tree_mask", c_void_p)]


class Block(Structure):
    _fields_ = [("post_norm", c_int32), ("gate_kind", c_int32), ("gate_sigmoid", c_int32), ("scale", c_float),
                ("eps", c_float), ("w_post", c_void_p), ("gate", c_void_p), ("w_pre", c_void_p)]


class Rope(Structure):
    _fields_ = [("rot_dim", c_int32), ("interleaved", c_int32), ("norm", c_int32), ("eps", c_float), ("w_q", c_void_p),
                ("w_k", c_void_p), ("freq", c_void_p), ("positions", c_void_p), ("cache_len", c_void_p),
                ("q_out_stride", c_int64), ("k_out_stride", c_int64)]


class CPagedCache(Structure):
    _fields_ = [("code", c_int32), ("n_pages", c_int32), ("page_size", c_int32), ("max_pages", c_int32), ("k_pages", c_void_p),
                ("v_pages", c_void_p), ("k_scale", c_void_p), ("v_scale", c_void_p), ("page_table", c_void_p)]


class Verify(Structure):
    _fields_ = [("vocab", c_int32), ("dtype", c_int32), ("logit_stride", c_int64), ("draft_stride", c_int64),
                ("logits", c_void_p), ("draft_logits", c_void_p), ("temperature", c_void_p)]


TRACE_POINTS = 5
TRACE_STAGES = ("prologue", "gate_up", "down", "combine")   # intervals between consecutive trace points


_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """dlopen the library and declare its signatures.  Raises if it has not been built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise FileNotFoundError(f"{p} is missing: build it with `python -m paper_2602_16052_amd.build` "
                                "(there is no non-HIP fallback)")
    lib = ctypes.CDLL(p)
    lib.moespec_abi_version.restype = c_int32
    lib.moespec_abi_version.argtypes = []
    lib.moespec_status_string.restype = c_char_p
    lib.moespec_status_string.argtypes = [c_int32]
    lib.moespec_check_desc.restype = c_int32
    lib.moespec_check_desc.argtypes = [POINTER(Desc)]
    lib.moespec_workspace_bytes.restype = c_size_t
    lib.moespec_workspace_bytes.argtypes = [POINTER(Desc), c_int32]
    lib.moespec_route.restype = c_int32
    lib.moespec_route.argtypes = [POINTER(Desc), POINTER(Weights), c_void_p, c_int32, c_void_p, c_void_p, c_void_p,
                                  c_void_p, c_size_t, c_void_p]
    lib.moespec_budget.restype = c_int32
    lib.moespec_budget.argtypes = [POINTER(Desc), c_void_p, c_int32, c_int32, c_int32, c_void_p, c_void_p, c_void_p,
                                   c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                   c_void_p]
    lib.moespec_expert_ffn.restype = c_int32
    lib.moespec_expert_ffn.argtypes = [POINTER(Desc), POINTER(Weights), c_void_p, c_int32, c_int32, c_void_p,
                                       c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_size_t, c_void_p]
    lib.moespec_layer_forward.restype = c_int32
    lib.moespec_layer_forward.argtypes = [POINTER(Desc), POINTER(Weights), c_void_p, c_int32, c_int32, c_int32,
                                          c_void_p, c_void_p, c_void_p, POINTER(Taps), c_void_p, c_size_t, c_void_p]
    lib.moespec_layer_forward_traced.restype = c_int32
    lib.moespec_layer_forward_traced.argtypes = [POINTER(Desc), POINTER(Weights), c_void_p, c_int32, c_int32, c_int32,
                                                 c_void_p, c_void_p, c_void_p, c_void_p, POINTER(c_void_p), c_void_p,
                                                 c_size_t, c_void_p]
    lib.moespec_layer_forward_static.restype = c_int32
    lib.moespec_layer_forward_static.argtypes = [POINTER(Desc), POINTER(Weights), c_void_p, c_int32, c_int32, c_int32,
                                                 c_void_p, c_void_p, c_void_p, c_void_p]
    lib.moespec_stack_forward.restype = c_int32
    lib.moespec_stack_forward.argtypes = [POINTER(Desc), POINTER(Weights), c_int32, c_void_p, c_int32, c_int32, c_int32,
                                          c_int32, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.moespec_rms_scale.restype = c_int32
    lib.moespec_rms_scale.argtypes = [POINTER(Desc), c_void_p, c_int32, c_void_p, c_void_p]
    lib.moespec_calibration_count.restype = c_int32
    lib.moespec_calibration_count.argtypes = [POINTER(Desc), c_void_p, c_int32, c_void_p, c_void_p]
    lib.moespec_static_shortlist.restype = c_int32
    lib.moespec_static_shortlist.argtypes = [POINTER(Desc), c_void_p, c_int32, c_void_p, c_void_p]
    lib.moespec_coverage_curve.restype = c_int32
    lib.moespec_coverage_curve.argtypes = [POINTER(Desc), c_void_p, c_void_p, c_void_p]
    lib.moespec_reconstruction_error.restype = c_int32
    lib.moespec_reconstruction_error.argtypes = [POINTER(Desc), c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                                                 c_size_t, c_void_p]
    lib.moespec_oracle_ranking.restype = c_int32
    lib.moespec_oracle_ranking.argtypes = [POINTER(Desc), POINTER(Weights), c_void_p, c_int32, c_int32, c_void_p,
                                           c_void_p, c_void_p, c_size_t, c_void_p]
    lib.moespec_stream_read.restype = c_int32
    lib.moespec_stream_read.argtypes = [c_void_p, c_size_t, c_void_p, c_void_p]
    P = c_void_p
    lib.moespec_check_attn_desc.restype = c_int32
    lib.moespec_check_attn_desc.argtypes = [POINTER(CAttnDesc)]
    lib.moespec_attn_workspace_bytes.restype = c_size_t
    lib.moespec_attn_workspace_bytes.argtypes = [POINTER(CAttnDesc), c_int32, c_int32, c_int32, c_int32]
    lib.moespec_tree_attention.restype = c_int32
    lib.moespec_tree_attention.argtypes = [POINTER(CAttnDesc), POINTER(Tree), P, P, P, P, P, P, c_int32, P, P, P, c_size_t, P]
    lib.moespec_cache_weights.restype = c_int32
    lib.moespec_cache_weights.argtypes = [POINTER(CAttnDesc), POINTER(Tree), P, P, P, P, c_int32, P, P, c_float, P, P, P, P,
                                          c_size_t, P]
    lib.moespec_cache_commit.restype = c_int32
    lib.moespec_cache_commit.argtypes = [POINTER(CAttnDesc), c_int32, POINTER(Tree), P, P, P, P, P, c_int32, P, P, P, P, P, P]
    lib.moespec_evict_workspace_bytes.restype = c_size_t
    lib.moespec_evict_workspace_bytes.argtypes = [POINTER(CAttnDesc), c_int32, c_int32, c_int32]
    lib.moespec_cache_evict.restype = c_int32
    lib.moespec_cache_evict.argtypes = [POINTER(CAttnDesc), c_int32, c_int32, P, P, P, P, c_int32, c_int32, c_int32, P, P, P,
                                        P, P, P, c_size_t, P]
    lib.moespec_block_norm.restype = c_int32
    lib.moespec_block_norm.argtypes = [POINTER(Desc), POINTER(Block), P, P, c_int32, P, P, P]
    lib.moespec_head_rope.restype = c_int32
    lib.moespec_head_rope.argtypes = [POINTER(CAttnDesc), POINTER(Rope), POINTER(Tree), P, P, P, P, P]
    lib.moespec_paged_write.restype = c_int32
    lib.moespec_paged_write.argtypes = [POINTER(CAttnDesc), c_int32, POINTER(CPagedCache), POINTER(Tree), P, P, P, P, c_int32, P, P,
                                        P]
    lib.moespec_paged_read.restype = c_int32
    lib.moespec_paged_read.argtypes = [POINTER(CAttnDesc), c_int32, c_int32, POINTER(CPagedCache), P, P, c_int32, P, P, P]
    lib.moespec_paged_attention_workspace_bytes.restype = c_size_t
    lib.moespec_paged_attention_workspace_bytes.argtypes = [POINTER(CAttnDesc), POINTER(CPagedCache), c_int32, c_int32]
    lib.moespec_paged_attention.restype = c_int32
    lib.moespec_paged_attention.argtypes = [POINTER(CAttnDesc), POINTER(CPagedCache), c_int32, P, c_int64, P, c_int32, P, P, P,
                                            c_size_t, P]
    lib.moespec_verify_workspace_bytes.restype = c_size_t
    lib.moespec_verify_workspace_bytes.argtypes = [POINTER(Verify), c_int32, c_int32]
    lib.moespec_draft_verify.restype = c_int32
    lib.moespec_draft_verify.argtypes = [POINTER(Verify), POINTER(Tree), P, P, P, P, P, c_int32, P, P, P, c_size_t, P]
    if path is None:
        _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().moespec_status_string(int(status)).decode()


def abi_version() -> int:
    return int(load_library().moespec_abi_version())


@dataclass
class LayerDesc:
    d: int
    n_experts: int
    top_k: int
    d_ff: int
    dtype: int          # F32 or BF16
    renorm: bool
    gate: int = 0       # GATE_SOFTMAX or GATE_SIGMOID

    def c(self) -> Desc:
        return Desc(self.d, self.n_experts, self.top_k, self.d_ff, self.dtype, int(self.renorm), int(self.gate))

    @property
    def torch_dtype(self) -> torch.dtype:
        return torch.bfloat16 if self.dtype == BF16 else torch.float32


def check_desc(desc: LayerDesc) -> int:
    c = desc.c()
    return int(load_library().moespec_check_desc(ctypes.byref(c)))


def workspace_bytes(desc: LayerDesc, M_max: int) -> int:
    c = desc.c()
    return int(load_library().moespec_workspace_bytes(ctypes.byref(c), int(M_max)))


def alloc_workspace(desc: LayerDesc, M_max: int, device="cuda") -> torch.Tensor:
    n = workspace_bytes(desc, M_max)
    if n == 0:
        raise MoeSpecError(ERR_INVALID_ARG, "moespec_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _ptr(t: Optional[torch.Tensor], dtype: Optional[torch.dtype] = None, numel: Optional[int] = None,
         name: str = "tensor") -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} needs at least {numel} elements, got {t.numel()}")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:  # the raw handle of torch.cuda.current_stream(), without building the object (2 us of a stage call)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None
    return stream.cuda_stream or None


def _weights(desc: LayerDesc, w: Dict[str, torch.Tensor], router: bool, experts: bool) -> Weights:
    N, d, F, dt = desc.n_experts, desc.d, desc.d_ff, desc.torch_dtype
    cw = Weights()
    if router:
        cw.w_router = _ptr(w["w_router"], dt, N * d, "w_router")
        cw.b_router = _ptr(w.get("b_router"), torch.float32, N, "b_router")
    if experts:
        cw.w_gate = _ptr(w["w_gate"], dt, N * F * d, "w_gate")
        cw.w_up = _ptr(w["w_up"], dt, N * F * d, "w_up")
        cw.w_down = _ptr(w["w_down"], dt, N * d * F, "w_down")
    return cw


def _check(status: int, where: str):
    if status != OK:
        raise MoeSpecError(int(status), where)


def moespec_route(desc: LayerDesc, weights: Dict[str, torch.Tensor], h: torch.Tensor, ws: torch.Tensor,
                  stream=None, want_topk: bool = True):
    """Eq. (1) + Section 2.1.  Returns dict(probs[M,N] f64, topk_ids[M,k] i32, topk_w[M,k] f32)."""
    M, N, k = h.shape[0], desc.n_experts, desc.top_k
    dev = h.device
    probs = torch.empty((M, N), dtype=torch.float64, device=dev)
    ids = torch.empty((M, k), dtype=torch.int32, device=dev) if want_topk else None
    tw = torch.empty((M, k), dtype=torch.float32, device=dev) if want_topk else None
    cd, cw = desc.c(), _weights(desc, weights, True, False)
    st = load_library().moespec_route(ctypes.byref(cd), ctypes.byref(cw), _ptr(h, desc.torch_dtype, M * desc.d, "h"),
                                      M, probs.data_ptr(), ids.data_ptr() if want_topk else None,
                                      tw.data_ptr() if want_topk else None, _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "moespec_route")
    return dict(probs=probs, topk_ids=ids, topk_w=tw)


def moespec_budget(desc: LayerDesc, probs: torch.Tensor, B: int, policy: int, ws: torch.Tensor,
                   ext_shortlist: Optional[torch.Tensor] = None, stream=None):
    """Eq. (5), shortlist, Eq. (7)/(8), segments.  Returns a dict of the documented outputs."""
    M, N, k = probs.shape[0], desc.n_experts, desc.top_k
    dev = probs.device
    i32 = dict(dtype=torch.int32, device=dev)
    out = dict(scores=torch.empty(N, dtype=torch.float64, device=dev), budget_ids=torch.empty(max(B, 1), **i32),
               tok_ids=torch.empty((M, k), **i32), tok_w=torch.empty((M, k), dtype=torch.float32, device=dev),
               seg_expert=torch.empty(max(B, 1), **i32), seg_off=torch.empty(max(B, 1) + 1, **i32),
               perm=torch.empty(M * k, **i32), n_loaded=torch.empty(1, **i32))
    cd = desc.c()
    st = load_library().moespec_budget(
        ctypes.byref(cd), _ptr(probs, torch.float64, M * N, "probs"), M, int(B), int(policy),
        _ptr(ext_shortlist, torch.int32, max(B, 0), "ext_shortlist"), *(t.data_ptr() for t in out.values()), _ptr(ws),
        ws.numel(), _stream(stream))
    _check(st, "moespec_budget")
    return out


def moespec_expert_ffn(desc: LayerDesc, weights: Dict[str, torch.Tensor], h: torch.Tensor, seg_expert: torch.Tensor,
                       seg_off: torch.Tensor, perm: torch.Tensor, tok_ids: torch.Tensor, tok_w: torch.Tensor,
                       ws: torch.Tensor, residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                       stream=None) -> torch.Tensor:
    """Experts over the loaded set + weighted combine.  Returns out[M, d] in the layer dtype."""
    M, k, dt = h.shape[0], desc.top_k, desc.torch_dtype
    n_seg = seg_expert.numel()
    if out is None:
        out = torch.empty((M, desc.d), dtype=dt, device=h.device)
    cd, cw = desc.c(), _weights(desc, weights, False, True)
    st = load_library().moespec_expert_ffn(
        ctypes.byref(cd), ctypes.byref(cw), _ptr(h, dt, M * desc.d, "h"), M, n_seg,
        _ptr(seg_expert, torch.int32, n_seg, "seg_expert"), _ptr(seg_off, torch.int32, n_seg + 1, "seg_off"),
        _ptr(perm, torch.int32, M * k, "perm"), _ptr(tok_ids, torch.int32, M * k, "tok_ids"),
        _ptr(tok_w, torch.float32, M * k, "tok_w"), _ptr(residual, dt, M * desc.d, "residual"),
        _ptr(out, dt, M * desc.d, "out"), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "moespec_expert_ffn")
    return out


class HipEvents:
    """A fixed set of timing-enabled hipEvent_t handles (created through libamdhip64 directly, so that
    their raw handles can cross the C ABI).  Used for the library's optional trace hook."""

    def __init__(self, n: int):
        self._hip = ctypes.CDLL("libamdhip64.so")
        self._hip.hipEventCreate.argtypes = [POINTER(c_void_p)]
        self._hip.hipEventElapsedTime.argtypes = [POINTER(ctypes.c_float), c_void_p, c_void_p]
        self._hip.hipEventSynchronize.argtypes = [c_void_p]
        self._hip.hipEventDestroy.argtypes = [c_void_p]
        self._hip.hipEventRecord.argtypes = [c_void_p, c_void_p]
        self.handles = (c_void_p * n)()
        for i in range(n):
            ev = c_void_p()
            if self._hip.hipEventCreate(ctypes.byref(ev)) != 0:
                raise MoeSpecError(ERR_HIP, "hipEventCreate")
            self.handles[i] = ev

    def record(self, i: int, stream=None):
        if self._hip.hipEventRecord(self.handles[i], _stream(stream)) != 0:
            raise MoeSpecError(ERR_HIP, "hipEventRecord")

    def synchronize(self, i: int):
        if self._hip.hipEventSynchronize(self.handles[i]) != 0:
            raise MoeSpecError(ERR_HIP, "hipEventSynchronize")

    def elapsed_ms(self, i: int, j: int) -> float:
        ms = ctypes.c_float()
        if self._hip.hipEventElapsedTime(ctypes.byref(ms), self.handles[i], self.handles[j]) != 0:
            raise MoeSpecError(ERR_HIP, "hipEventElapsedTime")
        return float(ms.value)

    def __del__(self):
        try:
            for ev in self.handles:
                if ev:
                    self._hip.hipEventDestroy(ev)
        except Exception:
            pass


class LayerForwardCall:
    """moespec_layer_forward with its arguments marshalled once: calling the object only crosses the
    C ABI (for tight loops, where per-call marshalling would cost more than the kernels).  With ``trace`` the call
    goes through moespec_layer_forward_traced, which records the events at the stage boundaries."""

    def __init__(self, desc: LayerDesc, weights: Dict[str, torch.Tensor], h: torch.Tensor, B: int, policy: int,
                 ws: torch.Tensor, out: torch.Tensor, ext_shortlist: Optional[torch.Tensor] = None,
                 residual: Optional[torch.Tensor] = None, trace: Optional[HipEvents] = None,
                 n_loaded: Optional[torch.Tensor] = None, stream=None):
        M, dt = h.shape[0], desc.torch_dtype
        self._keep = (weights, h, ws, out, ext_shortlist, residual, trace, n_loaded)
        lib = load_library()
        self._cd, self._cw = desc.c(), _weights(desc, weights, True, True)
        head = (ctypes.byref(self._cd), ctypes.byref(self._cw), _ptr(h, dt, M * desc.d, "h"), M, int(B),
                int(policy), _ptr(ext_shortlist, torch.int32, max(int(B), 0), "ext_shortlist"),
                _ptr(residual, dt, M * desc.d, "residual"), _ptr(out, dt, M * desc.d, "out"))
        tail = (_ptr(ws), ws.numel(), _stream(stream))
        if trace is not None:
            if len(trace.handles) < TRACE_POINTS:
                raise ValueError(f"trace needs {TRACE_POINTS} events")
            self._fn, self._name = lib.moespec_layer_forward_traced, "moespec_layer_forward_traced"
            self._args = head + (_ptr(n_loaded, torch.int32, 1, "n_loaded"),
                                 ctypes.cast(trace.handles, POINTER(c_void_p))) + tail
        else:
            self._fn, self._name = lib.moespec_layer_forward, "moespec_layer_forward"
            self._taps = None
            if n_loaded is not None:
                self._taps = Taps()
                self._taps.n_loaded = _ptr(n_loaded, torch.int32, 1, "n_loaded")
            self._args = head + (ctypes.byref(self._taps) if self._taps is not None else None,) + tail

    def __call__(self):
        st = self._fn(*self._args)
        if st != OK:
            raise MoeSpecError(int(st), self._name)


def moespec_layer_forward(desc: LayerDesc, weights: Dict[str, torch.Tensor], h: torch.Tensor, B: int, policy: int,
                          ws: torch.Tensor, ext_shortlist: Optional[torch.Tensor] = None,
                          residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                          taps: bool = False, stream=None):
    """Algorithm 1 in one call.  Returns ``out`` or, with ``taps=True``, ``(out, dict of intermediates)``."""
    M, N, k, dt = h.shape[0], desc.n_experts, desc.top_k, desc.torch_dtype
    dev = h.device
    if out is None:
        out = torch.empty((M, desc.d), dtype=dt, device=dev)
    tap_t = None
    ctaps = None
    if taps:
        i32 = dict(dtype=torch.int32, device=dev)
        nb = max(int(B), 1)
        tap_t = dict(probs=torch.empty((M, N), dtype=torch.float64, device=dev),
                     scores=torch.empty(N, dtype=torch.float64, device=dev), budget_ids=torch.empty(nb, **i32),
                     tok_ids=torch.empty((M, k), **i32), tok_w=torch.empty((M, k), dtype=torch.float32, device=dev),
                     seg_expert=torch.empty(nb, **i32), seg_off=torch.empty(nb + 1, **i32),
                     perm=torch.empty(M * k, **i32), n_loaded=torch.empty(1, **i32))
        ctaps = Taps(**{key: _ptr(val) for key, val in tap_t.items()})
    cd, cw = desc.c(), _weights(desc, weights, True, True)
    st = load_library().moespec_layer_forward(
        ctypes.byref(cd), ctypes.byref(cw), _ptr(h, dt, M * desc.d, "h"), M, int(B), int(policy),
        _ptr(ext_shortlist, torch.int32, max(int(B), 0), "ext_shortlist"), _ptr(residual, dt, M * desc.d, "residual"),
        _ptr(out, dt, M * desc.d, "out"), ctypes.byref(ctaps) if ctaps is not None else None, _ptr(ws), ws.numel(),
        _stream(stream))
    _check(st, "moespec_layer_forward")
    return (out, tap_t) if taps else out


def moespec_rms_scale(desc: LayerDesc, h: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x[t] = h[t] / rms(h[t]) (the input scaling of the layer stack).  Returns x[M, d] in the layer dtype."""
    M, dt = h.shape[0], desc.torch_dtype
    if out is None:
        out = torch.empty_like(h)
    cd = desc.c()
    st = load_library().moespec_rms_scale(ctypes.byref(cd), _ptr(h, dt, M * desc.d, "h"), M,
                                          _ptr(out, dt, M * desc.d, "x"), _stream(stream))
    _check(st, "moespec_rms_scale")
    return out


class StackForwardCall:
    """moespec_stack_forward with its arguments marshalled once (h is updated in place on every call)."""

    def __init__(self, desc: LayerDesc, layers, h: torch.Tensor, B: int, policy: int, ws: torch.Tensor,
                 pre_norm: bool = True, budget_ids: Optional[torch.Tensor] = None,
                 tok_ids: Optional[torch.Tensor] = None, stream=None):
        M, dt, L = h.shape[0], desc.torch_dtype, len(layers)
        self._keep = (layers, h, ws, budget_ids, tok_ids)
        self._fn = load_library().moespec_stack_forward
        self._cd = desc.c()
        self._cw = (Weights * L)(*[_weights(desc, w, True, True) for w in layers])
        self._args = (ctypes.byref(self._cd), self._cw, L, _ptr(h, dt, M * desc.d, "h"), M, int(B), int(policy),
                      int(bool(pre_norm)), _ptr(budget_ids, torch.int32, L * max(int(B), 1), "budget_ids"),
                      _ptr(tok_ids, torch.int32, L * M * desc.top_k, "tok_ids"), _ptr(ws), ws.numel(), _stream(stream))

    def __call__(self):
        st = self._fn(*self._args)
        if st != OK:
            raise MoeSpecError(int(st), "moespec_stack_forward")


def moespec_stack_forward(desc: LayerDesc, layers, h: torch.Tensor, B: int, policy: int, ws: torch.Tensor,
                          pre_norm: bool = True, taps: bool = False, stream=None):
    """The layer stack h <- h + MoE_S(x) over ``layers`` (a list of weight dicts), in place on ``h``.
    Returns ``h`` or, with ``taps=True``, ``(h, dict(budget_ids[L, B], tok_ids[L, M, k]))``."""
    L, M = len(layers), h.shape[0]
    tap = None
    if taps:
        i32 = dict(dtype=torch.int32, device=h.device)
        tap = dict(budget_ids=torch.empty((L, max(int(B), 1)), **i32), tok_ids=torch.empty((L, M, desc.top_k), **i32))
    StackForwardCall(desc, layers, h, B, policy, ws, pre_norm, tap["budget_ids"] if tap else None,
                     tap["tok_ids"] if tap else None, stream)()
    return (h, tap) if taps else h


STATIC_SCRATCH_BYTES = 48 << 20


def moespec_layer_forward_static(desc: LayerDesc, weights: Dict[str, torch.Tensor], h: torch.Tensor, B: int,
                                 policy: int, out: torch.Tensor, ext_shortlist: Optional[torch.Tensor] = None,
                                 residual: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Algorithm 1 in one call on the library's own fixed scratch array: no workspace argument, nothing allocated
    (``out`` is the caller's).  Returns ``out``."""
    M, dt = h.shape[0], desc.torch_dtype
    cd, cw = desc.c(), _weights(desc, weights, True, True)
    st = load_library().moespec_layer_forward_static(
        ctypes.byref(cd), ctypes.byref(cw), _ptr(h, dt, M * desc.d, "h"), M, int(B), int(policy),
        _ptr(ext_shortlist, torch.int32, max(int(B), 0), "ext_shortlist"), _ptr(residual, dt, M * desc.d, "residual"),
        _ptr(out, dt, M * desc.d, "out"), _stream(stream))
    _check(st, "moespec_layer_forward_static")
    return out


def moespec_calibration_count(desc: LayerDesc, topk_ids: torch.Tensor, counts: torch.Tensor, stream=None) -> torch.Tensor:
    """Eq. (4): counts[i] += number of rows of topk_ids [M, k] that contain expert i.  Returns counts."""
    M = topk_ids.shape[0]
    cd = desc.c()
    st = load_library().moespec_calibration_count(
        ctypes.byref(cd), _ptr(topk_ids, torch.int32, M * desc.top_k, "topk_ids"), M,
        _ptr(counts, torch.int64, desc.n_experts, "counts"), _stream(stream))
    _check(st, "moespec_calibration_count")
    return counts


def moespec_static_shortlist(desc: LayerDesc, counts: torch.Tensor, B: int, stream=None) -> torch.Tensor:
    """The B most frequently selected experts (Eq. (4)), most frequent first; int32 [B], usable as ext_shortlist."""
    out = torch.empty(max(int(B), 1), dtype=torch.int32, device=counts.device)
    cd = desc.c()
    st = load_library().moespec_static_shortlist(ctypes.byref(cd), _ptr(counts, torch.int64, desc.n_experts, "counts"),
                                                 int(B), _ptr(out), _stream(stream))
    _check(st, "moespec_static_shortlist")
    return out


def moespec_coverage_curve(desc: LayerDesc, scores: torch.Tensor, stream=None) -> torch.Tensor:
    """Section 4.6: share of the routing probability captured by the top-B experts, B = 1..N; float64 [N]."""
    out = torch.empty(desc.n_experts, dtype=torch.float64, device=scores.device)
    cd = desc.c()
    st = load_library().moespec_coverage_curve(ctypes.byref(cd), _ptr(scores, torch.float64, desc.n_experts, "scores"),
                                               _ptr(out), _stream(stream))
    _check(st, "moespec_coverage_curve")
    return out


def moespec_reconstruction_error(desc: LayerDesc, out_budgeted: torch.Tensor, out_full: torch.Tensor,
                                 ws: torch.Tensor, stream=None) -> torch.Tensor:
    """Section 4.5: float64 [3] = (||O_S - O*||^2 / ||O*||^2, numerator, denominator)."""
    M, dt = out_full.shape[0], desc.torch_dtype
    err = torch.empty(3, dtype=torch.float64, device=out_full.device)
    cd = desc.c()
    st = load_library().moespec_reconstruction_error(
        ctypes.byref(cd), _ptr(out_budgeted, dt, M * desc.d, "out_budgeted"), _ptr(out_full, dt, M * desc.d, "out_full"),
        M, _ptr(err), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "moespec_reconstruction_error")
    return err


def moespec_oracle_ranking(desc: LayerDesc, weights: Dict[str, torch.Tensor], h: torch.Tensor, B: int, ws: torch.Tensor,
                           stream=None):
    """Eq. (6): greedy oracle ordering.  Returns (ranking int32 [B], err float64 [B])."""
    M, dt = h.shape[0], desc.torch_dtype
    ranking = torch.empty(max(int(B), 1), dtype=torch.int32, device=h.device)
    err = torch.empty(max(int(B), 1), dtype=torch.float64, device=h.device)
    cd, cw = desc.c(), _weights(desc, weights, True, True)
    st = load_library().moespec_oracle_ranking(ctypes.byref(cd), ctypes.byref(cw), _ptr(h, dt, M * desc.d, "h"), M, int(B),
                                               _ptr(ranking), _ptr(err), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "moespec_oracle_ranking")
    return ranking, err


STREAM_READ_WORDS = 256


def moespec_stream_read(buf: torch.Tensor, checksum: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Measurement aid: stream `buf` (contiguous, a multiple of 16 bytes) once through a plain read kernel.
    Every workgroup adds the sum modulo 2^32 of the 32-bit words it read to its word of `checksum`
    (int32 [STREAM_READ_WORDS], zeroed here if not given); `checksum.sum()` modulo 2^32 is the buffer's checksum."""
    if not (buf.is_cuda and buf.is_contiguous()):
        raise ValueError("buf: expected a contiguous GPU tensor")
    if checksum is None:
        checksum = torch.zeros(STREAM_READ_WORDS, dtype=torch.int32, device=buf.device)
    st = load_library().moespec_stream_read(buf.data_ptr(), buf.numel() * buf.element_size(),
                                            _ptr(checksum, torch.int32, STREAM_READ_WORDS, "checksum"),
                                            _stream(stream))
    _check(st, "moespec_stream_read")
    return checksum


# ---- Tree attention, its cache, the norm between two blocks.  The calls come as objects with their arguments marshalled once (a
# program keeps one per layer, next to its buffers) and as functions that build one, allocate what is not given and call it.  Tensors
# are checked for device, type, exact shape and layout; the call runs on `stream` or, without one, on the stream that is current
# for the tensors' device at the time of the call.


@dataclass
class AttnDesc:
    """Shape of one attention layer (host side of moespec_attn_desc).  scale None: 1 / sqrt(head_dim)."""
    n_heads: int
    n_kv_heads: int
    head_dim: int
    capacity: int
    dtype: int          # F32 or BF16
    scale: Optional[float] = None

    def c(self) -> CAttnDesc:
        scale = self.scale if self.scale is not None else max(int(self.head_dim), 1) ** -0.5
        return CAttnDesc(self.n_heads, self.n_kv_heads, self.head_dim, self.capacity, self.dtype, scale)

    @property
    def torch_dtype(self) -> torch.dtype:
        return torch.bfloat16 if self.dtype == BF16 else torch.float32


def check_attn_desc(desc: AttnDesc) -> int:
    c = desc.c()
    return int(load_library().moespec_check_attn_desc(ctypes.byref(c)))


def attn_workspace_bytes(desc: AttnDesc, n_seq: int, M_max: int, max_tree: int, max_len: int) -> int:
    c = desc.c()
    return int(load_library().moespec_attn_workspace_bytes(ctypes.byref(c), int(n_seq), int(M_max), int(max_tree),
                                                           int(max_len)))


def alloc_attn_workspace(desc: AttnDesc, n_seq: int, M_max: int, max_tree: int, max_len: int, device="cuda") -> torch.Tensor:
    n = attn_workspace_bytes(desc, n_seq, M_max, max_tree, max_len)
    if n == 0:
        raise MoeSpecError(ERR_INVALID_ARG, "moespec_attn_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def evict_workspace_bytes(desc: AttnDesc, n_layers: int, n_seq: int, budget: int) -> int:
    c = desc.c()
    return int(load_library().moespec_evict_workspace_bytes(ctypes.byref(c), int(n_layers), int(n_seq), int(budget)))


def alloc_evict_workspace(desc: AttnDesc, n_layers: int, n_seq: int, budget: int, device="cuda") -> torch.Tensor:
    n = evict_workspace_bytes(desc, n_layers, n_seq, budget)
    if n == 0:
        raise MoeSpecError(ERR_INVALID_ARG, "moespec_evict_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


class _Call:
    """A C call on one device: its arguments but the stream, and what they point to."""

    def __init__(self, name: str, device: torch.device, args, keep, stream):
        self._fn, self._name, self._args, self._keep = getattr(load_library(), name), name, args, keep
        self._device, self._stream = device.index if device.index is not None else torch.cuda.current_device(), stream
        if stream is not None and getattr(stream, "device_index", self._device) != self._device:
            raise ValueError(f"stream must belong to cuda:{self._device}, got one of {stream.device}")

    def __call__(self):
        if torch.cuda.current_device() == self._device:
            st = self._fn(*self._args, _stream(self._stream))
        else:
            with torch.cuda.device(self._device):
                st = self._fn(*self._args, _stream(self._stream))
        if st != OK:
            raise MoeSpecError(int(st), self._name)


def _allocating(stream):
    """Where a function allocates for a call on `stream`: there, so that fills come before the call and memory that is freed after
    it is reused behind it."""
    return torch.cuda.stream(stream)  # (of None: as things are)


class _Args:
    """Pointers of tensors that have to lie on one device."""

    def __init__(self):
        self.device = None

    def on(self, t: torch.Tensor, name: str):
        if not t.is_cuda:
            raise ValueError(f"{name} must be a GPU tensor")
        if self.device is None:
            self.device = t.device
        elif t.device != self.device:
            raise ValueError(f"{name} must be on {self.device}, got {t.device}")

    def ptr(self, t: Optional[torch.Tensor], dtype: torch.dtype, shape, name: str) -> Optional[int]:
        """Pointer of a contiguous tensor of exactly this shape, or None."""
        if t is None:
            return None
        self.on(t, name)
        if t.dtype != dtype:
            raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return t.data_ptr()

    def rows(self, t: torch.Tensor, dtype: torch.dtype, shape, name: str):
        """Pointer and row stride of a tensor [.., tokens, heads, head_dim] whose rows are contiguous, wherever they lie."""
        self.on(t, name)
        if t.dtype != dtype:
            raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
        heads, dim = t.shape[-2:]
        st = t.stride()
        one = t.shape[-3] == 1  # a single row: the layers are as far apart as rows would be
        row = st[-3] if not one else st[0] if len(shape) == 4 and t.shape[0] > 1 else heads * dim
        if (dim > 1 and st[-1] != 1) or (heads > 1 and st[-2] != dim) or row < heads * dim or \
                (len(shape) == 4 and t.shape[0] > 1 and st[0] != t.shape[1] * row):
            raise ValueError(f"{name}: a token's heads must lie in a row, and rows and layers be equally far apart")
        return t.data_ptr(), row

    def scratch(self, ws: torch.Tensor):
        self.on(ws, "ws")
        if not ws.is_contiguous() or ws.dtype != torch.uint8:
            raise ValueError("ws must be a contiguous uint8 tensor")
        return ws.data_ptr(), ws.numel()


def _sizes(M: int, tree_off: Optional[torch.Tensor], max_tree: Optional[int]):
    """Sequences of a batch and the rows of its largest tree: as given, or every token row."""
    return (1 if tree_off is None else tree_off.numel() - 1), (M if max_tree is None else int(max_tree))


def _tree(a: _Args, M: int, n_seq: int, max_tree: int, q_stride: int, kv_stride: int, tree_off, tree_mask) -> Tree:
    return Tree(n_seq, M, max_tree, q_stride, kv_stride, a.ptr(tree_off, torch.int32, (n_seq + 1,), "tree_off"),
                a.ptr(tree_mask, torch.int32, (M, (max_tree + 31) // 32), "tree_mask"))


class TreeAttentionCall(_Call):
    """moespec_tree_attention.  q [M, H, D], k_tree, v_tree [M, Hk, D] (views with longer rows are taken as they are); k_cache,
    v_cache [n_seq, Hk, capacity, D]; cache_len [n_seq] int32; out [M, H, D]; lse [M, H] float32 or None; tree_off [n_seq + 1]
    int32 or None (one tree of all rows); tree_mask [M, ceil(max_tree / 32)] int32, the packed bits of the trees, or None (chains);
    max_tree, max_len: bounds on a tree's rows and a cache's entries, M and the capacity if None; max_len 0: no cache."""

    def __init__(self, desc: AttnDesc, q: torch.Tensor, k_tree: torch.Tensor, v_tree: torch.Tensor,
                 k_cache: Optional[torch.Tensor], v_cache: Optional[torch.Tensor], cache_len: Optional[torch.Tensor],
                 ws: torch.Tensor, out: torch.Tensor, lse: Optional[torch.Tensor] = None,
                 tree_off: Optional[torch.Tensor] = None, tree_mask: Optional[torch.Tensor] = None,
                 max_tree: Optional[int] = None, max_len: Optional[int] = None, stream=None):
        a, dt, H, Hk, D = _Args(), desc.torch_dtype, desc.n_heads, desc.n_kv_heads, desc.head_dim
        M = q.shape[0]
        S, most = _sizes(M, tree_off, max_tree)
        max_len = (0 if k_cache is None else desc.capacity) if max_len is None else int(max_len)
        (qp, qs), (kp, ks) = a.rows(q, dt, (M, H, D), "q"), a.rows(k_tree, dt, (M, Hk, D), "k_tree")
        vp, vs = a.rows(v_tree, dt, (M, Hk, D), "v_tree")
        if vs != ks:
            raise ValueError("k_tree and v_tree must have the same row stride")
        cache = (S, Hk, desc.capacity, D)
        self._cd, self._tree = desc.c(), _tree(a, M, S, most, qs, ks, tree_off, tree_mask)
        args = (ctypes.byref(self._cd), ctypes.byref(self._tree), qp, kp, vp, a.ptr(k_cache, dt, cache, "k_cache"),
                a.ptr(v_cache, dt, cache, "v_cache"), a.ptr(cache_len, torch.int32, (S,), "cache_len"), max_len,
                a.ptr(out, dt, (M, H, D), "out"), a.ptr(lse, torch.float32, (M, H), "lse"), *a.scratch(ws))
        super().__init__("moespec_tree_attention", a.device, args,
                         (q, k_tree, v_tree, k_cache, v_cache, cache_len, ws, out, lse, tree_off, tree_mask), stream)


def moespec_tree_attention(desc: AttnDesc, q, k_tree, v_tree, k_cache=None, v_cache=None, cache_len=None, ws=None, out=None,
                           lse=None, tree_off=None, tree_mask=None, max_tree=None, max_len=None, stream=None):
    """Attention of drafted tokens over cache and tree (TreeAttentionCall).  Returns (out, lse).  Without tree_off all rows
    are one tree; padding rows of a new `out` are not written."""
    M = q.shape[0]
    S, most = _sizes(M, tree_off, max_tree)
    with _allocating(stream):
        if out is None:
            out = torch.empty((M, desc.n_heads, desc.head_dim), dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.empty((M, desc.n_heads), dtype=torch.float32, device=q.device)
        if ws is None:
            ws = alloc_attn_workspace(desc, S, M, most, (0 if k_cache is None else desc.capacity) if max_len is None else max_len,
                                      q.device)
    TreeAttentionCall(desc, q, k_tree, v_tree, k_cache, v_cache, cache_len, ws, out, lse, tree_off, tree_mask, max_tree,
                      max_len, stream)()
    return out, lse


class CacheWeightsCall(_Call):
    """moespec_cache_weights: the attention weight that every key received.  Tensors as in TreeAttentionCall; lse [M, H] float32;
    cache_w, cache_w_in [n_seq, Hk, capacity] float32 (cache_w = decay * cache_w_in + weight; cache_w_in may be cache_w or
    None); tree_w [M, Hk] float32 or None; row_weight [M] float32 or None."""

    def __init__(self, desc: AttnDesc, q: torch.Tensor, k_tree: torch.Tensor, k_cache: Optional[torch.Tensor],
                 cache_len: Optional[torch.Tensor], lse: torch.Tensor, ws: torch.Tensor, cache_w: Optional[torch.Tensor],
                 tree_w: Optional[torch.Tensor] = None, cache_w_in: Optional[torch.Tensor] = None, decay: float = 1.0,
                 row_weight: Optional[torch.Tensor] = None, tree_off: Optional[torch.Tensor] = None,
                 tree_mask: Optional[torch.Tensor] = None, max_tree: Optional[int] = None, max_len: Optional[int] = None,
                 stream=None):
        a, dt, H, Hk, D = _Args(), desc.torch_dtype, desc.n_heads, desc.n_kv_heads, desc.head_dim
        M = q.shape[0]
        S, most = _sizes(M, tree_off, max_tree)
        max_len = (0 if k_cache is None else desc.capacity) if max_len is None else int(max_len)
        (qp, qs), (kp, ks) = a.rows(q, dt, (M, H, D), "q"), a.rows(k_tree, dt, (M, Hk, D), "k_tree")
        self._cd, self._tree = desc.c(), _tree(a, M, S, most, qs, ks, tree_off, tree_mask)
        w = (S, Hk, desc.capacity)
        args = (ctypes.byref(self._cd), ctypes.byref(self._tree), qp, kp, a.ptr(k_cache, dt, (*w, D), "k_cache"),
                a.ptr(cache_len, torch.int32, (S,), "cache_len"), max_len, a.ptr(lse, torch.float32, (M, H), "lse"),
                a.ptr(row_weight, torch.float32, (M,), "row_weight"), float(decay),
                a.ptr(cache_w_in, torch.float32, w, "cache_w_in"), a.ptr(cache_w, torch.float32, w, "cache_w"),
                a.ptr(tree_w, torch.float32, (M, Hk), "tree_w"), *a.scratch(ws))
        super().__init__("moespec_cache_weights", a.device, args,
                         (q, k_tree, k_cache, cache_len, lse, ws, cache_w, tree_w, cache_w_in, row_weight, tree_off, tree_mask),
                         stream)


def moespec_cache_weights(desc: AttnDesc, q, k_tree, k_cache, cache_len, lse, ws=None, cache_w=None, tree_w=None, cache_w_in=None,
                          decay=1.0, row_weight=None, tree_off=None, tree_mask=None, max_tree=None, max_len=None, stream=None):
    """Weight that every cached key and every key of the trees received (CacheWeightsCall).  Returns (cache_w, tree_w)."""
    M = q.shape[0]
    S, most = _sizes(M, tree_off, max_tree)
    with _allocating(stream):
        if cache_w is None and k_cache is not None:
            cache_w = torch.zeros((S, desc.n_kv_heads, desc.capacity), dtype=torch.float32, device=q.device)
        if tree_w is None:
            tree_w = torch.zeros((M, desc.n_kv_heads), dtype=torch.float32, device=q.device)
        if ws is None:
            ws = alloc_attn_workspace(desc, S, M, most, (0 if k_cache is None else desc.capacity) if max_len is None else max_len,
                                      q.device)
    CacheWeightsCall(desc, q, k_tree, k_cache, cache_len, lse, ws, cache_w, tree_w, cache_w_in, decay, row_weight, tree_off,
                     tree_mask, max_tree, max_len, stream)()
    return cache_w, tree_w


class CacheCommitCall(_Call):
    """moespec_cache_commit: the accepted path appended to the caches of n_layers layers.  k_tree, v_tree [n_layers, M, Hk, D];
    path [n_seq, max_path] int32; n_path, cache_len, new_len [n_seq] int32; k_cache, v_cache [n_layers, n_seq, Hk, capacity, D];
    tree_w [n_layers, M, Hk] and cache_w [n_layers, n_seq, Hk, capacity] float32, both or neither."""

    def __init__(self, desc: AttnDesc, k_tree: torch.Tensor, v_tree: torch.Tensor, path: torch.Tensor, n_path: torch.Tensor,
                 k_cache: torch.Tensor, v_cache: torch.Tensor, cache_len: torch.Tensor,
                 new_len: Optional[torch.Tensor] = None, tree_w: Optional[torch.Tensor] = None,
                 cache_w: Optional[torch.Tensor] = None, tree_off: Optional[torch.Tensor] = None,
                 max_tree: Optional[int] = None, n_layers: int = 1, stream=None):
        a, dt, Hk, D, L, i32 = _Args(), desc.torch_dtype, desc.n_kv_heads, desc.head_dim, int(n_layers), torch.int32
        M = k_tree.shape[-3]
        S, most = _sizes(M, tree_off, max_tree)
        (kp, ks), (vp, vs) = a.rows(k_tree, dt, (L, M, Hk, D), "k_tree"), a.rows(v_tree, dt, (L, M, Hk, D), "v_tree")
        if vs != ks:
            raise ValueError("k_tree and v_tree must have the same row stride")
        self._cd, self._tree = desc.c(), _tree(a, M, S, most, 0, ks, tree_off, None)
        w = (L, S, Hk, desc.capacity)
        n = path.shape[-1]
        args = (ctypes.byref(self._cd), L, ctypes.byref(self._tree), kp, vp, a.ptr(tree_w, torch.float32, (L, M, Hk), "tree_w"),
                a.ptr(path, i32, (S, n), "path"), a.ptr(n_path, i32, (S,), "n_path"), n, a.ptr(k_cache, dt, (*w, D), "k_cache"),
                a.ptr(v_cache, dt, (*w, D), "v_cache"), a.ptr(cache_w, torch.float32, w, "cache_w"),
                a.ptr(cache_len, i32, (S,), "cache_len"), a.ptr(new_len, i32, (S,), "new_len"))
        super().__init__("moespec_cache_commit", a.device, args,
                         (k_tree, v_tree, path, n_path, k_cache, v_cache, cache_len, new_len, tree_w, cache_w, tree_off), stream)


def moespec_cache_commit(desc: AttnDesc, k_tree, v_tree, path, n_path, k_cache, v_cache, cache_len, new_len=None, tree_w=None,
                         cache_w=None, tree_off=None, max_tree=None, n_layers=1, stream=None) -> torch.Tensor:
    """Accepted paths appended to the caches, in place (CacheCommitCall).  Returns new_len."""
    if new_len is None:
        with _allocating(stream):
            new_len = torch.empty_like(cache_len)
    CacheCommitCall(desc, k_tree, v_tree, path, n_path, k_cache, v_cache, cache_len, new_len, tree_w, cache_w, tree_off, max_tree,
                    n_layers, stream)()
    return new_len


class CacheEvictCall(_Call):
    """moespec_cache_evict: caches [n_layers, n_seq, Hk, capacity, D] with weights [n_layers, n_seq, Hk, capacity] float32 cut to
    `budget` entries, the `recent` last ones among them, into k_out, v_out, w_out (the same with a capacity of their own).  kept
    [n_layers, n_seq, Hk, budget] int32 and new_len [n_seq] int32 may be None."""

    def __init__(self, desc: AttnDesc, k_cache: torch.Tensor, v_cache: torch.Tensor, cache_w: torch.Tensor,
                 cache_len: torch.Tensor, budget: int, recent: int, k_out: torch.Tensor, v_out: torch.Tensor,
                 w_out: torch.Tensor, ws: torch.Tensor, kept: Optional[torch.Tensor] = None,
                 new_len: Optional[torch.Tensor] = None, n_layers: int = 1, stream=None):
        a, dt, Hk, D, L, i32 = _Args(), desc.torch_dtype, desc.n_kv_heads, desc.head_dim, int(n_layers), torch.int32
        S, room = cache_len.numel(), k_out.shape[-2]
        w, o = (L, S, Hk, desc.capacity), (L, S, Hk, room)
        self._cd = desc.c()
        args = (ctypes.byref(self._cd), L, S, a.ptr(k_cache, dt, (*w, D), "k_cache"), a.ptr(v_cache, dt, (*w, D), "v_cache"),
                a.ptr(cache_w, torch.float32, w, "cache_w"), a.ptr(cache_len, i32, (S,), "cache_len"), int(budget), int(recent),
                room, a.ptr(k_out, dt, (*o, D), "k_out"), a.ptr(v_out, dt, (*o, D), "v_out"),
                a.ptr(w_out, torch.float32, o, "w_out"), a.ptr(kept, i32, (L, S, Hk, int(budget)), "kept"),
                a.ptr(new_len, i32, (S,), "new_len"), *a.scratch(ws))
        super().__init__("moespec_cache_evict", a.device, args,
                         (k_cache, v_cache, cache_w, cache_len, k_out, v_out, w_out, ws, kept, new_len), stream)


def moespec_cache_evict(desc: AttnDesc, k_cache, v_cache, cache_w, cache_len, budget, recent, n_layers=1, stream=None):
    """Caches cut to a budget (CacheEvictCall).  Returns dict(k, v, w, kept, new_len); entries of k, v, w behind new_len are 0."""
    L, S, Hk, D, dev = int(n_layers), cache_len.numel(), desc.n_kv_heads, desc.head_dim, k_cache.device
    n = max(int(budget), 1)
    with _allocating(stream):
        k, v = (torch.zeros((L, S, Hk, n, D), dtype=k_cache.dtype, device=dev) for _ in range(2))
        w = torch.zeros((L, S, Hk, n), dtype=torch.float32, device=dev)
        kept = torch.empty((L, S, Hk, n), dtype=torch.int32, device=dev)
        new_len = torch.empty_like(cache_len)
        ws = torch.empty(max(evict_workspace_bytes(desc, L, S, n), 1), dtype=torch.uint8, device=dev)
    CacheEvictCall(desc, k_cache, v_cache, cache_w, cache_len, budget, recent, k, v, w, ws, kept if budget == n else None, new_len,
                   n_layers, stream)()
    return dict(k=k, v=v, w=w, kept=kept, new_len=new_len)


class BlockNormCall(_Call):
    """moespec_block_norm: r = residual + scale * gate * norm(y), x = norm(r).  y, residual, r, x [M, d] in the layer's dtype
    (residual None: 0; r or x None: not wanted); w_post, w_pre [d] or None; gate by gate_kind: [d], [M], [M, d] or None."""

    def __init__(self, desc: LayerDesc, y: torch.Tensor, residual: Optional[torch.Tensor], r: Optional[torch.Tensor],
                 x: Optional[torch.Tensor], post_norm: bool = False, w_post: Optional[torch.Tensor] = None,
                 gate: Optional[torch.Tensor] = None, gate_kind: int = BLOCK_GATE_NONE, gate_sigmoid: bool = False,
                 scale: float = 1.0, w_pre: Optional[torch.Tensor] = None, eps: float = 0.0, stream=None):
        a, dt, d = _Args(), desc.torch_dtype, desc.d
        M = y.shape[0]
        shapes = {BLOCK_GATE_CHANNEL: (d,), BLOCK_GATE_TOKEN: (M,), BLOCK_GATE_ELEMENT: (M, d)}
        yp = a.ptr(y, dt, (M, d), "y")
        self._cd = desc.c()
        self._block = Block(int(bool(post_norm)), int(gate_kind), int(bool(gate_sigmoid)), scale, eps,
                            a.ptr(w_post, dt, (d,), "w_post"), a.ptr(gate, dt, shapes.get(gate_kind, ()), "gate"),
                            a.ptr(w_pre, dt, (d,), "w_pre"))
        args = (ctypes.byref(self._cd), ctypes.byref(self._block), yp, a.ptr(residual, dt, (M, d), "residual"), M,
                a.ptr(r, dt, (M, d), "r"), a.ptr(x, dt, (M, d), "x"))
        super().__init__("moespec_block_norm", a.device, args, (y, residual, r, x, w_post, gate, w_pre), stream)


def moespec_block_norm(desc: LayerDesc, y, residual=None, r=None, x=None, post_norm=False, w_post=None, gate=None,
                       gate_kind=BLOCK_GATE_NONE, gate_sigmoid=False, scale=1.0, w_pre=None, eps=0.0, stream=None):
    """From a block's output to the residual stream and the next block's input (BlockNormCall).  Returns (r, x)."""
    with _allocating(stream):
        r = torch.empty_like(y) if r is None else r
        x = torch.empty_like(y) if x is None else x
    BlockNormCall(desc, y, residual, r, x, post_norm, w_post, gate, gate_kind, gate_sigmoid, scale, w_pre, eps, stream)()
    return r, x


# ---- Around both halves of a serving step: head norm and rotation, a paged cache, single tokens over it, verification.

class HeadRopeCall(_Call):
    """moespec_head_rope: queries q [M, H, D] and keys k [M, Hk, D] (views with longer rows are taken as they are; one of them may be
    None, with its output) normed for each head and rotated, into q_out, k_out: the same shapes, views too, or q and k
    themselves.  freq [rot_dim / 2] float32; w_q, w_k [D] or None; the place of a token is positions [M] int32, or cache_len
    [n_seq] int32 (None: 0) plus its depth in the tree that tree_off, tree_mask and max_tree describe (TreeAttentionCall)."""

    def __init__(self, desc: AttnDesc, q: Optional[torch.Tensor], k: Optional[torch.Tensor], q_out: Optional[torch.Tensor],
                 k_out: Optional[torch.Tensor], freq: Optional[torch.Tensor], rot_dim: Optional[int] = None,
                 interleaved: bool = False, norm: bool = False, w_q: Optional[torch.Tensor] = None,
                 w_k: Optional[torch.Tensor] = None, eps: float = 0.0, positions: Optional[torch.Tensor] = None,
                 cache_len: Optional[torch.Tensor] = None, tree_off: Optional[torch.Tensor] = None,
                 tree_mask: Optional[torch.Tensor] = None, max_tree: Optional[int] = None, stream=None):
        a, dt, i32, H, Hk, D = _Args(), desc.torch_dtype, torch.int32, desc.n_heads, desc.n_kv_heads, desc.head_dim
        if q is None and k is None:
            raise ValueError("q and k must not both be None")
        M = (k if q is None else q).shape[0]
        S, most = _sizes(M, tree_off, max_tree)
        rot = (D if freq is not None else 0) if rot_dim is None else int(rot_dim)
        rows = lambda t, n, name: (None, 0) if t is None else a.rows(t, dt, (M, n, D), name)  # noqa: E731
        (qp, qs), (kp, ks) = rows(q, H, "q"), rows(k, Hk, "k")
        (qop, qos), (kop, kos) = rows(q_out, H, "q_out"), rows(k_out, Hk, "k_out")
        self._cd, self._tree = desc.c(), _tree(a, M, S, most, qs, ks, tree_off, tree_mask)
        self._rope = Rope(rot, int(bool(interleaved)), int(bool(norm)), eps, a.ptr(w_q, dt, (D,), "w_q"), a.ptr(w_k, dt, (D,), "w_k"),
                          a.ptr(freq, torch.float32, (rot // 2,), "freq"), a.ptr(positions, i32, (M,), "positions"),
                          a.ptr(cache_len, i32, (S,), "cache_len"), qos, kos)
        args = (ctypes.byref(self._cd), ctypes.byref(self._rope), ctypes.byref(self._tree), qp, kp, qop, kop)
        super().__init__("moespec_head_rope", a.device, args,
                         (q, k, q_out, k_out, freq, w_q, w_k, positions, cache_len, tree_off, tree_mask), stream)


def moespec_head_rope(desc: AttnDesc, q, k, q_out=None, k_out=None, freq=None, rot_dim=None, interleaved=False, norm=False, w_q=None,
                      w_k=None, eps=0.0, positions=None, cache_len=None, tree_off=None, tree_mask=None, max_tree=None, stream=None):
    """Queries and keys made ready for attention (HeadRopeCall).  Returns (q_out, k_out); padding rows of new ones are not written."""
    with _allocating(stream):
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q_out is None and q is not None else q_out
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device) if k_out is None and k is not None else k_out
    HeadRopeCall(desc, q, k, q_out, k_out, freq, rot_dim, interleaved, norm, w_q, w_k, eps, positions, cache_len, tree_off, tree_mask,
                 max_tree, stream)()
    return q_out, k_out


@dataclass
class PagedCache:
    """Keys and values of n_layers layers in pages of a pool (host side of moespec_paged_cache).  k_pages, v_pages [n_layers, n_pages,
    Hk, page_size, D] in the layer's dtype (CACHE_PLAIN), int8 (CACHE_I8) or float8_e4m3fn (CACHE_E4M3); page_table [n_seq,
    max_pages] int32: entry e of a sequence lies in page page_table[s, e // page_size]; k_scale, v_scale [n_layers, n_pages, Hk,
    page_size] float32 with codes, else None."""
    code: int
    k_pages: torch.Tensor
    v_pages: torch.Tensor
    page_table: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None

    @property
    def n_layers(self) -> int:
        return self.k_pages.shape[0]

    @property
    def max_entries(self) -> int:
        return self.page_table.shape[1] * self.k_pages.shape[3]

    def c(self, a: _Args, desc: AttnDesc, n_seq: int, layer: Optional[int] = None) -> CPagedCache:
        """The struct with checked pointers: of all layers, or of one."""
        held = {CACHE_PLAIN: desc.torch_dtype, CACHE_I8: torch.int8, CACHE_E4M3: torch.float8_e4m3fn}.get(self.code)
        if held is None:
            raise ValueError(f"unknown cache code {self.code}")
        if self.k_pages.dim() != 5 or self.page_table.dim() != 2:
            raise ValueError("k_pages must be [n_layers, n_pages, Hk, page_size, D] and page_table [n_seq, max_pages]")
        L, n_pages, _, size, _ = self.k_pages.shape
        if layer is not None and not 0 <= layer < L:
            raise ValueError(f"layer must be in 0 .. {L - 1}, got {layer}")
        shape = (L, n_pages, desc.n_kv_heads, size, desc.head_dim)
        at = lambda t, dt, sh, name: None if t is None else a.ptr(t, dt, sh, name) and t[layer or 0].data_ptr()  # noqa: E731
        return CPagedCache(self.code, n_pages, size, self.page_table.shape[1], at(self.k_pages, held, shape, "k_pages"),
                           at(self.v_pages, held, shape, "v_pages"), at(self.k_scale, torch.float32, shape[:-1], "k_scale"),
                           at(self.v_scale, torch.float32, shape[:-1], "v_scale"),
                           a.ptr(self.page_table, torch.int32, (n_seq, self.page_table.shape[1]), "page_table"))

    def tensors(self):
        return (self.k_pages, self.v_pages, self.page_table, self.k_scale, self.v_scale)


def alloc_paged_cache(desc: AttnDesc, code: int, n_pages: int, page_size: int, page_table: torch.Tensor,
                      n_layers: int = 1) -> PagedCache:
    """A pool of n_pages pages for each layer, on the table's device.  Its contents are undefined."""
    held = {CACHE_PLAIN: desc.torch_dtype, CACHE_I8: torch.int8, CACHE_E4M3: torch.float8_e4m3fn}[code]
    shape, dev = (n_layers, n_pages, desc.n_kv_heads, page_size, desc.head_dim), page_table.device
    pages = [torch.empty(shape, dtype=held, device=dev) for _ in range(2)]
    scales = [None if code == CACHE_PLAIN else torch.empty(shape[:-1], dtype=torch.float32, device=dev) for _ in range(2)]
    return PagedCache(code, *pages, page_table, *scales)


class PagedWriteCall(_Call):
    """moespec_paged_write: accepted paths, or whole trees (path and n_path None), appended to the pages of all of the cache's layers.
    k_tree, v_tree [n_layers, M, Hk, D]; path [n_seq, max_path] int32; n_path, cache_len, new_len [n_seq] int32."""

    def __init__(self, desc: AttnDesc, cache: PagedCache, k_tree: torch.Tensor, v_tree: torch.Tensor, cache_len: torch.Tensor,
                 path: Optional[torch.Tensor] = None, n_path: Optional[torch.Tensor] = None,
                 new_len: Optional[torch.Tensor] = None, tree_off: Optional[torch.Tensor] = None,
                 max_tree: Optional[int] = None, stream=None):
        a, dt, Hk, D, L, i32 = _Args(), desc.torch_dtype, desc.n_kv_heads, desc.head_dim, cache.n_layers, torch.int32
        M = k_tree.shape[-3]
        S, most = _sizes(M, tree_off, max_tree)
        (kp, ks), (vp, vs) = a.rows(k_tree, dt, (L, M, Hk, D), "k_tree"), a.rows(v_tree, dt, (L, M, Hk, D), "v_tree")
        if vs != ks:
            raise ValueError("k_tree and v_tree must have the same row stride")
        self._cd, self._cache, self._tree = desc.c(), cache.c(a, desc, S), _tree(a, M, S, most, 0, ks, tree_off, None)
        n = 0 if path is None else path.shape[-1]
        args = (ctypes.byref(self._cd), L, ctypes.byref(self._cache), ctypes.byref(self._tree), kp, vp,
                a.ptr(path, i32, (S, n), "path"), a.ptr(n_path, i32, (S,), "n_path"), n, a.ptr(cache_len, i32, (S,), "cache_len"),
                a.ptr(new_len, i32, (S,), "new_len"))
        super().__init__("moespec_paged_write", a.device, args,
                         (*cache.tensors(), k_tree, v_tree, cache_len, path, n_path, new_len, tree_off), stream)


def moespec_paged_write(desc: AttnDesc, cache: PagedCache, k_tree, v_tree, cache_len, path=None, n_path=None, new_len=None,
                        tree_off=None, max_tree=None, stream=None) -> torch.Tensor:
    """Keys and values appended to the pages, in place (PagedWriteCall).  Returns new_len."""
    if new_len is None:
        with _allocating(stream):
            new_len = torch.empty_like(cache_len)
    PagedWriteCall(desc, cache, k_tree, v_tree, cache_len, path, n_path, new_len, tree_off, max_tree, stream)()
    return new_len


class PagedReadCall(_Call):
    """moespec_paged_read: entries first .. cache_len - 1 (first [n_seq] int32 or None: 0) into contiguous caches k_cache, v_cache
    [n_layers, n_seq, Hk, capacity, D]; max_len: a bound on the lengths, what cache and table have room for if None."""

    def __init__(self, desc: AttnDesc, cache: PagedCache, cache_len: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                 first: Optional[torch.Tensor] = None, max_len: Optional[int] = None, stream=None):
        a, dt, i32, S = _Args(), desc.torch_dtype, torch.int32, cache_len.numel()
        dense = (cache.n_layers, S, desc.n_kv_heads, desc.capacity, desc.head_dim)
        self._cd, self._cache = desc.c(), cache.c(a, desc, S)
        args = (ctypes.byref(self._cd), cache.n_layers, S, ctypes.byref(self._cache), a.ptr(first, i32, (S,), "first"),
                a.ptr(cache_len, i32, (S,), "cache_len"), min(desc.capacity, cache.max_entries) if max_len is None else int(max_len),
                a.ptr(k_cache, dt, dense, "k_cache"), a.ptr(v_cache, dt, dense, "v_cache"))
        super().__init__("moespec_paged_read", a.device, args, (*cache.tensors(), first, cache_len, k_cache, v_cache), stream)


def moespec_paged_read(desc: AttnDesc, cache: PagedCache, cache_len, k_cache=None, v_cache=None, first=None, max_len=None,
                       stream=None):
    """Entries in pages laid out as contiguous caches (PagedReadCall).  Returns (k_cache, v_cache); entries of new ones that are not
    read are 0."""
    dense = (cache.n_layers, cache_len.numel(), desc.n_kv_heads, desc.capacity, desc.head_dim)
    with _allocating(stream):
        k_cache, v_cache = (torch.zeros(dense, dtype=desc.torch_dtype, device=cache_len.device) if t is None else t
                            for t in (k_cache, v_cache))
    PagedReadCall(desc, cache, cache_len, k_cache, v_cache, first, max_len, stream)()
    return k_cache, v_cache


def paged_attention_workspace_bytes(desc: AttnDesc, cache: PagedCache, n_seq: int, max_len: int) -> int:
    c = desc.c()
    p = CPagedCache(cache.code, cache.k_pages.shape[1], cache.k_pages.shape[3], cache.page_table.shape[1],
                    *(None if t is None else t.data_ptr() for t in (cache.k_pages, cache.v_pages, cache.k_scale, cache.v_scale)),
                    cache.page_table.data_ptr())
    return int(load_library().moespec_paged_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(p), int(n_seq), int(max_len)))


def alloc_paged_attention_workspace(desc: AttnDesc, cache: PagedCache, n_seq: int, max_len: int) -> torch.Tensor:
    n = paged_attention_workspace_bytes(desc, cache, n_seq, max_len)
    if n == 0:
        raise MoeSpecError(ERR_INVALID_ARG, "moespec_paged_attention_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=cache.page_table.device)


class PagedAttentionCall(_Call):
    """moespec_paged_attention: one new token of every sequence, q [n_seq, H, D] (a view with longer rows is taken as it is), over the
    entries in a layer's pages; cache_len [n_seq] int32; out [n_seq, H, D]; lse [n_seq, H] float32 or None; max_len: a bound on
    the lengths, what the table has room for if None."""

    def __init__(self, desc: AttnDesc, cache: PagedCache, q: torch.Tensor, cache_len: torch.Tensor, ws: torch.Tensor,
                 out: torch.Tensor, lse: Optional[torch.Tensor] = None, max_len: Optional[int] = None, layer: int = 0, stream=None):
        a, dt, S, H, D = _Args(), desc.torch_dtype, q.shape[0], desc.n_heads, desc.head_dim
        qp, qs = a.rows(q, dt, (S, H, D), "q")
        self._cd, self._cache = desc.c(), cache.c(a, desc, S, int(layer))
        args = (ctypes.byref(self._cd), ctypes.byref(self._cache), S, qp, qs, a.ptr(cache_len, torch.int32, (S,), "cache_len"),
                cache.max_entries if max_len is None else int(max_len), a.ptr(out, dt, (S, H, D), "out"),
                a.ptr(lse, torch.float32, (S, H), "lse"), *a.scratch(ws))
        super().__init__("moespec_paged_attention", a.device, args, (*cache.tensors(), q, cache_len, ws, out, lse), stream)


def moespec_paged_attention(desc: AttnDesc, cache: PagedCache, q, cache_len, ws=None, out=None, lse=None, max_len=None, layer=0,
                            stream=None):
    """Attention of one new token of every sequence over its pages (PagedAttentionCall).  Returns (out, lse)."""
    S, H = q.shape[0], desc.n_heads
    with _allocating(stream):
        if out is None:
            out = torch.empty((S, H, desc.head_dim), dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.empty((S, H), dtype=torch.float32, device=q.device)
        if ws is None:
            ws = alloc_paged_attention_workspace(desc, cache, S, cache.max_entries if max_len is None else max_len)
    PagedAttentionCall(desc, cache, q, cache_len, ws, out, lse, max_len, layer, stream)()
    return out, lse


@dataclass
class VerifyDesc:
    """The vocabulary and the dtype (F32 or BF16) of the logits that drafts are judged by."""
    vocab: int
    dtype: int

    @property
    def torch_dtype(self) -> torch.dtype:
        return torch.bfloat16 if self.dtype == BF16 else torch.float32


def verify_workspace_bytes(desc: VerifyDesc, n_seq: int, M_max: int, sampled: bool = False) -> int:
    """sampled: with the drafter's logits."""
    v = Verify(desc.vocab, desc.dtype, 0, 0, None, 16 if sampled else None, None)
    return int(load_library().moespec_verify_workspace_bytes(ctypes.byref(v), int(n_seq), int(M_max)))


def alloc_verify_workspace(desc: VerifyDesc, n_seq: int, M_max: int, sampled: bool = False, device="cuda") -> torch.Tensor:
    n = verify_workspace_bytes(desc, n_seq, M_max, sampled)
    if n == 0:
        raise MoeSpecError(ERR_INVALID_ARG, "moespec_verify_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


class DraftVerifyCall(_Call):
    """moespec_draft_verify: from the target's logits [M, vocab] (and, for drafts sampled in chains, the drafter's draft_logits [M,
    vocab]; rows of both may be longer in memory) and the uniform numbers u_accept [M], u_sample [n_seq] float64 to the accepted
    path [n_seq, max_path] int32, n_path and next_token [n_seq] int32, and accepted [M] float32 (1 or 0) or None.  tokens [M] int32;
    temperature [n_seq] float32 or None (1), of both distributions: a drafter that samples at another one, t', passes its logits times
    temperature / t'; tree_off, tree_mask, max_tree as in TreeAttentionCall, row 0 of a tree its root."""

    def __init__(self, desc: VerifyDesc, logits: torch.Tensor, tokens: torch.Tensor, u_accept: torch.Tensor, u_sample: torch.Tensor,
                 path: torch.Tensor, n_path: torch.Tensor, next_token: torch.Tensor, ws: torch.Tensor,
                 draft_logits: Optional[torch.Tensor] = None, temperature: Optional[torch.Tensor] = None,
                 accepted: Optional[torch.Tensor] = None, tree_off: Optional[torch.Tensor] = None,
                 tree_mask: Optional[torch.Tensor] = None, max_tree: Optional[int] = None, stream=None):
        a, i32, f64 = _Args(), torch.int32, torch.float64
        M = logits.shape[0]
        S, most = _sizes(M, tree_off, max_tree)

        def rows(t, name):
            if t is None:
                return None, 0
            a.on(t, name)
            if t.dtype != desc.torch_dtype or tuple(t.shape) != (M, desc.vocab):
                raise ValueError(f"{name} must be {desc.torch_dtype} of shape {(M, desc.vocab)}, got {t.dtype} of {tuple(t.shape)}")
            if t.stride(1) != 1 or (M > 1 and t.stride(0) < desc.vocab):
                raise ValueError(f"{name}: the logits of a token must lie in a row")
            return t.data_ptr(), t.stride(0) if M > 1 else 0

        (lp, ls), (dp, ds) = rows(logits, "logits"), rows(draft_logits, "draft_logits")
        n = path.shape[-1]
        self._verify = Verify(desc.vocab, desc.dtype, ls, ds, lp, dp, a.ptr(temperature, torch.float32, (S,), "temperature"))
        self._tree = _tree(a, M, S, most, 0, 0, tree_off, tree_mask)
        args = (ctypes.byref(self._verify), ctypes.byref(self._tree), a.ptr(tokens, i32, (M,), "tokens"),
                a.ptr(u_accept, f64, (M,), "u_accept"), a.ptr(u_sample, f64, (S,), "u_sample"), a.ptr(path, i32, (S, n), "path"),
                a.ptr(n_path, i32, (S,), "n_path"), n, a.ptr(next_token, i32, (S,), "next_token"),
                a.ptr(accepted, torch.float32, (M,), "accepted"), *a.scratch(ws))
        super().__init__("moespec_draft_verify", a.device, args,
                         (logits, tokens, u_accept, u_sample, path, n_path, next_token, ws, draft_logits, temperature, accepted,
                          tree_off, tree_mask), stream)


def moespec_draft_verify(desc: VerifyDesc, logits, tokens, u_accept, u_sample, max_path, draft_logits=None, temperature=None,
                         tree_off=None, tree_mask=None, max_tree=None, ws=None, stream=None):
    """Verification of drafted tokens (DraftVerifyCall).  Returns dict(path, n_path, next_token, accepted); accepted is 0 for rows of
    no sequence."""
    M, dev = logits.shape[0], logits.device
    S, _ = _sizes(M, tree_off, max_tree)
    with _allocating(stream):
        path = torch.empty((S, int(max_path)), dtype=torch.int32, device=dev)
        n_path, next_token = (torch.empty(S, dtype=torch.int32, device=dev) for _ in range(2))
        accepted = torch.zeros(M, dtype=torch.float32, device=dev)
        if ws is None:
            ws = alloc_verify_workspace(desc, S, M, draft_logits is not None, dev)
    DraftVerifyCall(desc, logits, tokens, u_accept, u_sample, path, n_path, next_token, ws, draft_logits, temperature, accepted,
                    tree_off, tree_mask, max_tree, stream)()
    return dict(path=path, n_path=n_path, next_token=next_token, accepted=accepted)
