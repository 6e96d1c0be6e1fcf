"""Thin ctypes binding of libcsp.so: same names as the C interface, argument marshalling only.

Every step of the path runs inside the CUDA library; PyTorch is used for device memory and for
the current stream.  There is no CPU fallback: if the library is missing, import of the symbols
fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcsp.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_ARCH, ERR_CUDA, ERR_TIMEOUT = range(7)
F32, BF16 = 0, 1
COMBINE_OR, COMBINE_AND = 0, 1
SELECT_SEGMENTED, SELECT_GLOBAL, SELECT_OVERALL = 0, 1, 2
HEADS_PER_KV, HEADS_MEAN_ALL = 0, 1
DEV_K_CLAMPED, DEV_CAPACITY, DEV_TIMEOUT, DEV_BAD_LEN = 1, 2, 4, 8

EXPORTS = ("csp_workspace_bytes", "csp_workspace_reset", "csp_score", "csp_select", "csp_compact",
           "csp_prune_layer", "csp_host_staging_bytes", "csp_prune_layer_host", "csp_device_status",
           "csp_status_string", "csp_prune_layer_static", "csp_static_workspace_limit",
           "csp_decode_workspace_bytes", "csp_decode_attn", "csp_decode_step_workspace_bytes", "csp_decode_step",
           "csp_weight_histogram", "csp_probe_ex2_rate", "csp_prune_layer_paged",
           "csp_decode_attn_paged", "csp_select_compact", "csp_chunk_workspace_bytes", "csp_chunk_attn", "csp_chunk_attn_paged",
           "csp_append_workspace_bytes", "csp_append_paged", "csp_pages_workspace_bytes", "csp_pages_fork",
           "csp_pages_reserve", "csp_pages_free", "csp_pages_compact", "csp_pages_copy")
HIST_BINS, HIST_LO, HIST_WIDTH = 64, -32.0, 0.5


class CspError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (csp_status {code})")


class CTensor(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_t", C.c_int64)]


class CPages(C.Structure):
    _fields_ = [("page_table", C.c_void_p), ("max_pages", C.c_int32), ("page_rows", C.c_int32), ("n_pages", C.c_int32)]


class CScoreMods(C.Structure):
    _fields_ = [("softcap", C.c_float), ("slopes", C.c_void_p),
                ("positions", C.c_void_p), ("pos_stride_b", C.c_int64), ("pos_stride_h", C.c_int64),
                ("documents", C.c_void_p), ("doc_stride_b", C.c_int64), ("doc_stride_h", C.c_int64),
                ("prefix", C.c_void_p), ("prefix_stride_b", C.c_int64), ("prefix_stride_h", C.c_int64)]


class CPageState(C.Structure):
    _fields_ = [("page_table", C.c_void_p), ("held", C.c_void_p), ("refs", C.c_void_p), ("n_rows", C.c_void_p),
                ("batch", C.c_int32), ("n_heads", C.c_int32), ("max_pages", C.c_int32), ("page_rows", C.c_int32),
                ("n_pages", C.c_int32)]


class CParams(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("window", C.c_int32), ("recent", C.c_int32),
                ("max_len", C.c_int32), ("out_capacity", C.c_int32), ("dtype", C.c_int32),
                ("n", C.c_float), ("scale", C.c_float), ("combine", C.c_int32),
                ("select_mode", C.c_int32), ("head_reduce", C.c_int32)]


@dataclass
class Params:
    __slots__ = ("_made", "__dict__", "__weakref__")    # (_made is no attribute that vars() shows or a copy of it hands on)
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    window: int
    recent: int
    max_len: int
    out_capacity: int
    dtype: int = BF16
    n: float = 1.0
    scale: float = 0.0
    combine: int = COMBINE_OR
    select_mode: int = SELECT_SEGMENTED
    head_reduce: int = HEADS_PER_KV

    def _fields(self):
        return (self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.window,
                self.recent, self.max_len, self.out_capacity, self.dtype, self.n, self.scale,
                self.combine, self.select_mode, self.head_reduce)

    def c(self) -> CParams:
        return CParams(*self._fields())

    def _c(self) -> CParams:
        """What the calls below pass, which nobody changes: the struct of the last call, while nothing has changed."""
        now, made = self._fields(), getattr(self, "_made", None)
        if made is None or made[0] != now:
            made = self._made = (now, CParams(*now))
        return made[1]


@dataclass
class ScoreMods:
    """What chunk_attn does to the logits (csp_score_mods).  slopes fp32 [Hq]; positions, documents int32 [B, cap] (shared
    by the heads) or [B, Hkv, cap]; prefix int32 [B] or [B, 1] (shared) or [B, Hkv]."""
    softcap: float = 0.0
    slopes: Optional[torch.Tensor] = None
    positions: Optional[torch.Tensor] = None
    documents: Optional[torch.Tensor] = None
    prefix: Optional[torch.Tensor] = None

    def tensors(self):
        return [t for t in (self.slopes, self.positions, self.documents, self.prefix) if t is not None]

    def c(self, p: "Params") -> CScoreMods:
        m = CScoreMods(softcap=float(self.softcap))
        if self.slopes is not None:
            assert self.slopes.dtype == torch.float32 and self.slopes.is_contiguous() and self.slopes.numel() == p.n_q_heads
            m.slopes = self.slopes.data_ptr()
        for name, short in (("positions", "pos"), ("documents", "doc")):
            t = getattr(self, name)
            if t is None:
                continue
            assert t.dtype == torch.int32 and t.dim() in (2, 3) and t.stride(-1) == 1, f"{name}: int32 [B, (Hkv,) rows]"
            assert t.shape[0] == p.batch and t.shape[-1] >= p.out_capacity and (t.dim() == 2 or t.shape[1] == p.n_kv_heads)
            setattr(m, name, t.data_ptr())
            setattr(m, short + "_stride_b", t.stride(0))
            setattr(m, short + "_stride_h", t.stride(1) if t.dim() == 3 else 0)
        if self.prefix is not None:
            t = self.prefix
            assert t.dtype == torch.int32 and t.dim() in (1, 2) and t.shape[0] == p.batch
            assert t.dim() == 1 or t.shape[1] in (1, p.n_kv_heads)
            m.prefix, m.prefix_stride_b = t.data_ptr(), t.stride(0)
            m.prefix_stride_h = t.stride(1) if t.dim() == 2 and t.shape[1] > 1 else 0
        return m


@dataclass
class PageState:
    """Whose pages are whose (csp_page_state): int32 tensors page_table [B, max_pages], held [B], refs [n_pages],
    n_rows [B, heads], all dense and changed in place by the pages_* calls."""
    page_table: torch.Tensor
    held: torch.Tensor
    refs: torch.Tensor
    n_rows: torch.Tensor
    page_rows: int

    def c(self) -> CPageState:
        table, held, refs, rows = self.page_table, self.held, self.refs, self.n_rows
        for t in (table, held, refs, rows):
            assert t.dtype is torch.int32 and t.is_contiguous()
        ts, rs = table.shape, rows.shape
        assert len(ts) == 2 and len(rs) == 2 and held.numel() == ts[0] == rs[0]
        return CPageState(table.data_ptr(), held.data_ptr(), refs.data_ptr(), rows.data_ptr(), ts[0], rs[1], ts[1],
                          self.page_rows, refs.numel())


def new_page_state(batch: int, n_heads: int, max_pages: int, page_rows: int, n_pages: int, device="cuda") -> PageState:
    """A pool of n_pages free pages and `batch` sequences that hold none."""
    z = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device=device)  # noqa: E731
    return PageState(z(batch, max_pages).fill_(-1), z(batch), z(n_pages), z(batch, n_heads), page_rows)


_lib = None


def lib() -> C.CDLL:
    """Loads libcsp.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            # not built yet (fresh checkout): compile in-tree now; there is no other implementation to fall
            # back to, so a failed build is an import error
            try:
                from . import build as _build
                _build.build()
            except Exception as exc:  # noqa: BLE001
                raise ImportError(f"{LIB_PATH} is missing and could not be built with nvcc: {exc}") from exc
        l = C.CDLL(LIB_PATH)
        P = C.POINTER(CParams)
        vp, i64, sz = C.c_void_p, C.c_int64, C.c_size_t
        l.csp_workspace_bytes.restype = sz
        l.csp_workspace_bytes.argtypes = [P]
        l.csp_workspace_reset.restype = C.c_int
        l.csp_workspace_reset.argtypes = [vp, vp]
        l.csp_score.restype = C.c_int
        l.csp_score.argtypes = [P, CTensor, CTensor, vp, i64, i64, vp, vp, vp, vp, vp, sz, vp]
        l.csp_select.restype = C.c_int
        l.csp_select.argtypes = [P, vp, vp, vp, i64, i64, vp, vp, vp, vp, vp, vp, sz, vp]
        l.csp_compact.restype = C.c_int
        l.csp_compact.argtypes = [P, CTensor, CTensor, vp, i64, i64, vp, vp, CTensor, CTensor, vp, vp]
        l.csp_select_compact.restype = C.c_int
        l.csp_select_compact.argtypes = [P, vp, vp, CTensor, CTensor, vp, i64, i64, vp, vp, vp, CTensor, CTensor, vp, vp,
                                         vp, vp, sz, vp]
        l.csp_prune_layer.restype = C.c_int
        l.csp_prune_layer.argtypes = [P, CTensor, CTensor, CTensor, vp, i64, i64, vp, vp, vp, vp,
                                      CTensor, CTensor, vp, vp, vp, vp, vp, vp, sz, vp]
        l.csp_host_staging_bytes.restype = sz
        l.csp_host_staging_bytes.argtypes = [P]
        l.csp_prune_layer_host.restype = C.c_int
        l.csp_prune_layer_host.argtypes = [P, vp, vp, vp, vp, C.c_int, vp, vp, vp, vp, vp, vp, vp, vp,
                                           vp, sz, vp]
        l.csp_prune_layer_static.restype = C.c_int
        l.csp_prune_layer_static.argtypes = [P, CTensor, CTensor, CTensor, vp, i64, i64, vp, vp, vp, vp,
                                             CTensor, CTensor, vp, vp, vp, vp]
        l.csp_static_workspace_limit.restype = sz
        l.csp_static_workspace_limit.argtypes = []
        l.csp_decode_workspace_bytes.restype = sz
        l.csp_decode_workspace_bytes.argtypes = [P]
        l.csp_decode_attn.restype = C.c_int
        l.csp_decode_attn.argtypes = [P, CTensor, CTensor, CTensor, vp, vp, vp, sz, vp]
        l.csp_decode_step_workspace_bytes.restype = sz
        l.csp_decode_step_workspace_bytes.argtypes = [P]
        l.csp_decode_step.restype = C.c_int
        l.csp_decode_step.argtypes = [P, CTensor, CTensor, CTensor, vp, vp, i64, i64, vp, C.c_int32, vp, vp, vp, vp, sz, vp]
        l.csp_prune_layer_paged.restype = C.c_int
        l.csp_prune_layer_paged.argtypes = [P, CTensor, CTensor, CTensor, C.POINTER(CPages), vp, i64, i64, vp, vp, vp, vp,
                                            CTensor, CTensor, vp, vp, vp, vp, vp, vp, sz, vp]
        l.csp_decode_attn_paged.restype = C.c_int
        l.csp_decode_attn_paged.argtypes = [P, CTensor, CTensor, CTensor, C.POINTER(CPages), vp, vp, vp, sz, vp]
        M, G, S, i32 = C.POINTER(CScoreMods), C.POINTER(CPages), C.POINTER(CPageState), C.c_int32
        l.csp_chunk_workspace_bytes.restype = sz
        l.csp_chunk_workspace_bytes.argtypes = [P, i32]
        l.csp_chunk_attn.restype = C.c_int
        l.csp_chunk_attn.argtypes = [P, i32, CTensor, CTensor, CTensor, vp, vp, M, CTensor, vp, vp, sz, vp]
        l.csp_chunk_attn_paged.restype = C.c_int
        l.csp_chunk_attn_paged.argtypes = [P, i32, CTensor, CTensor, CTensor, G, vp, vp, M, CTensor, vp, vp, sz, vp]
        l.csp_append_workspace_bytes.restype = sz
        l.csp_append_workspace_bytes.argtypes = [P]
        l.csp_append_paged.restype = C.c_int
        l.csp_append_paged.argtypes = [P, i32, CTensor, CTensor, vp, CTensor, CTensor, G, vp, vp, vp, sz, vp]
        l.csp_pages_workspace_bytes.restype = sz
        l.csp_pages_workspace_bytes.argtypes = [S]
        l.csp_pages_fork.restype = C.c_int
        l.csp_pages_fork.argtypes = [S, vp, vp, i32, vp, sz, vp]
        l.csp_pages_reserve.restype = C.c_int
        l.csp_pages_reserve.argtypes = [S, vp, i32, vp, i32, vp, vp, sz, vp]
        l.csp_pages_free.restype = C.c_int
        l.csp_pages_free.argtypes = [S, vp, sz, vp]
        l.csp_pages_compact.restype = C.c_int
        l.csp_pages_compact.argtypes = [S, vp, i32, vp, vp, sz, vp]
        l.csp_pages_copy.restype = C.c_int
        l.csp_pages_copy.argtypes = [P, CTensor, CTensor, i32, i32, vp, i32, vp, vp, sz, vp]
        l.csp_probe_ex2_rate.restype = C.c_int
        l.csp_probe_ex2_rate.argtypes = [C.c_int32, C.c_int32, vp, sz, C.POINTER(C.c_int64), vp]
        l.csp_weight_histogram.restype = C.c_int
        l.csp_weight_histogram.argtypes = [P, CTensor, CTensor, vp, i64, i64, vp, vp, vp, vp, vp, vp, sz, vp]
        l.csp_device_status.restype = C.c_int
        l.csp_device_status.argtypes = [vp, vp, C.POINTER(C.c_int32)]
        l.csp_status_string.restype = C.c_char_p
        l.csp_status_string.argtypes = [C.c_int]
        _lib = l
    return _lib


def status_string(code: int) -> str:
    return lib().csp_status_string(int(code)).decode()


def _check(code: int, where: str):
    if code != OK:
        raise CspError(code, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream():
    # (current_stream() builds an object around this handle: 3 us, half of what a whole small call takes)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def tensor4(t: torch.Tensor) -> CTensor:
    """[B, H, T, d] tensor -> (pointer, element strides); the last axis must be contiguous."""
    s = t.stride()
    assert len(s) == 4 and (s[3] == 1 or t.shape[3] == 1), "head_dim axis must be contiguous"
    return CTensor(t.data_ptr(), s[0], s[1], s[2])


def _mod_strides(modality: torch.Tensor):
    """[B, L] (shared by the heads) or [B, H, L] labels -> (stride_b, stride_h)."""
    assert modality.dtype == torch.uint8 and modality.stride(-1) == 1
    if modality.dim() == 2:
        return modality.stride(0), 0
    return modality.stride(0), modality.stride(1)


def workspace_bytes(p: Params) -> int:
    cp = p._c()
    return int(lib().csp_workspace_bytes(C.byref(cp)))


def new_workspace(p: Params, device="cuda") -> torch.Tensor:
    """Allocates (with torch) and zeroes a workspace for these parameters."""
    n = workspace_bytes(p)
    if n == 0:
        raise CspError(ERR_UNSUPPORTED, "csp_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def workspace_reset(ws: torch.Tensor):
    _check(lib().csp_workspace_reset(_ptr(ws), _stream()), "csp_workspace_reset")


def decode_workspace_bytes(p: Params) -> int:
    cp = p._c()
    return int(lib().csp_decode_workspace_bytes(C.byref(cp)))


def new_decode_workspace(p: Params, device="cuda") -> torch.Tensor:
    """Allocates (with torch) and zeroes a workspace for csp_decode_attn."""
    n = decode_workspace_bytes(p)
    if n == 0:
        raise CspError(ERR_UNSUPPORTED, "csp_decode_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def decode_attn(p: Params, q, k, v, n_rows, out, ws):
    """q [B, Hq, d]; k, v [B, Hkv, out_capacity, d]; n_rows int32 [B, Hkv]; out fp32 [B, Hq, d] (dense)."""
    cp = p._c()
    assert q.dim() == 3 and q.stride(2) == 1 and out.is_contiguous() and out.dtype == torch.float32
    qt = CTensor(q.data_ptr(), q.stride(0), q.stride(1), q.shape[2])
    _check(lib().csp_decode_attn(C.byref(cp), qt, tensor4(k), tensor4(v), _ptr(n_rows), _ptr(out), _ptr(ws),
                                 ws.numel(), _stream()), "csp_decode_attn")


def new_decode_step_workspace(p: Params, device="cuda") -> torch.Tensor:
    """Allocates (with torch) and zeroes a workspace for csp_decode_step."""
    cp = p._c()
    n = int(lib().csp_decode_step_workspace_bytes(C.byref(cp)))
    if n == 0:
        raise CspError(ERR_UNSUPPORTED, "csp_decode_step_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def decode_step(p: Params, q, k, v, n_rows, modality, query_label, first_step, out, acc_self, acc_cross, ws):
    """csp_decode_attn plus the running intra / inter sums: modality uint8 [B, Hkv, cap] (or [B, cap]), query_label
    uint8 [B], acc_self / acc_cross fp32 [B, Hkv, cap] (dense)."""
    cp = p._c()
    assert q.dim() == 3 and q.stride(2) == 1 and out.is_contiguous() and out.dtype == torch.float32
    assert acc_self.is_contiguous() and acc_cross.is_contiguous() and acc_self.dtype == torch.float32
    assert query_label.dtype == torch.uint8 and query_label.is_contiguous()
    qt = CTensor(q.data_ptr(), q.stride(0), q.stride(1), q.shape[2])
    sb, sh = _mod_strides(modality)
    _check(lib().csp_decode_step(C.byref(cp), qt, tensor4(k), tensor4(v), _ptr(n_rows), _ptr(modality), sb, sh,
                                 _ptr(query_label), int(bool(first_step)), _ptr(out), _ptr(acc_self), _ptr(acc_cross),
                                 _ptr(ws), ws.numel(), _stream()), "csp_decode_step")


def score(p: Params, q_win, k, modality, seq_lens, score_self, score_cross, ws, lse=None):
    cp = p._c()
    sb, sh = _mod_strides(modality)
    _check(lib().csp_score(C.byref(cp), tensor4(q_win), tensor4(k), _ptr(modality), sb, sh, _ptr(seq_lens),
                           _ptr(lse), _ptr(score_self), _ptr(score_cross), _ptr(ws), ws.numel(), _stream()),
           "csp_score")


def weight_histogram(p: Params, q_win, k, modality, seq_lens, hist, ws, js=None, js_all=None, lse=None):
    """hist uint32-as-int32 [B, Hkv, 2, HIST_BINS]; js fp32 [B, Hkv]; js_all fp32 [1]."""
    cp = p._c()
    sb, sh = _mod_strides(modality)
    assert hist.is_contiguous() and hist.element_size() == 4
    _check(lib().csp_weight_histogram(C.byref(cp), tensor4(q_win), tensor4(k), _ptr(modality), sb, sh, _ptr(seq_lens),
                                      _ptr(lse), _ptr(hist), _ptr(js), _ptr(js_all), _ptr(ws), ws.numel(), _stream()),
           "csp_weight_histogram")


def probe_ex2_rate(fma_pipe: bool, iterations: int, sink: Optional[torch.Tensor] = None) -> int:
    """Enqueues the exponential-throughput probe on the current stream; returns how many exponentials it evaluates."""
    n = C.c_int64(0)
    _check(lib().csp_probe_ex2_rate(int(fma_pipe), int(iterations), _ptr(sink), 0 if sink is None else sink.numel(),
                                    C.byref(n), _stream()), "csp_probe_ex2_rate")
    return int(n.value)


def select(p: Params, score_self, score_cross, modality, seq_lens, budgets, keep_idx, n_out, ws,
           total_budget=None):
    cp = p._c()
    sb, sh = _mod_strides(modality)
    _check(lib().csp_select(C.byref(cp), _ptr(score_self), _ptr(score_cross), _ptr(modality), sb, sh,
                            _ptr(seq_lens), _ptr(budgets), _ptr(total_budget), _ptr(keep_idx), _ptr(n_out),
                            _ptr(ws), ws.numel(), _stream()), "csp_select")


def compact(p: Params, k, v, modality, keep_idx, n_out, k_out, v_out, mod_out=None):
    cp = p._c()
    sb, sh = _mod_strides(modality) if modality is not None else (0, 0)
    _check(lib().csp_compact(C.byref(cp), tensor4(k), tensor4(v), _ptr(modality), sb, sh, _ptr(keep_idx),
                             _ptr(n_out), tensor4(k_out), tensor4(v_out), _ptr(mod_out), _stream()),
           "csp_compact")


def select_compact(p: Params, score_self, score_cross, k, v, modality, seq_lens, budgets, k_out, v_out, mod_out, n_out,
                   ws, total_budget=None, keep_idx=None):
    cp = p._c()
    sb, sh = _mod_strides(modality)
    _check(lib().csp_select_compact(C.byref(cp), _ptr(score_self), _ptr(score_cross), tensor4(k), tensor4(v),
                                    _ptr(modality), sb, sh, _ptr(seq_lens), _ptr(budgets), _ptr(total_budget),
                                    tensor4(k_out), tensor4(v_out), _ptr(mod_out), _ptr(n_out), _ptr(keep_idx),
                                    _ptr(ws), ws.numel(), _stream()), "csp_select_compact")


def prune_layer(p: Params, q_win, k, v, modality, seq_lens, budgets, k_out, v_out, mod_out, n_out, ws,
                total_budget=None, lse=None, score_self=None, score_cross=None, keep_idx=None):
    cp = p._c()
    sb, sh = _mod_strides(modality)
    _check(lib().csp_prune_layer(C.byref(cp), tensor4(q_win), tensor4(k), tensor4(v), _ptr(modality), sb, sh,
                                 _ptr(seq_lens), _ptr(budgets), _ptr(total_budget), _ptr(lse),
                                 tensor4(k_out), tensor4(v_out), _ptr(mod_out), _ptr(n_out),
                                 _ptr(score_self), _ptr(score_cross), _ptr(keep_idx),
                                 _ptr(ws), ws.numel(), _stream()), "csp_prune_layer")


def prune_layer_paged(p: Params, q_win, k_pool, v_pool, page_table, modality, seq_lens, budgets, k_out, v_out, mod_out,
                      n_out, ws, total_budget=None, lse=None, score_self=None, score_cross=None, keep_idx=None):
    """k_pool, v_pool [n_pages, Hkv, page_rows, d]; page_table int32 [B, max_pages] (dense).  k_out / v_out dense
    [B, Hkv, cap, d], or the pools themselves for pruning in place."""
    cp = p._c()
    sb, sh = _mod_strides(modality)
    assert page_table.dtype == torch.int32 and page_table.is_contiguous() and page_table.dim() == 2
    pg = CPages(page_table.data_ptr(), page_table.shape[1], k_pool.shape[2], k_pool.shape[0])
    _check(lib().csp_prune_layer_paged(C.byref(cp), tensor4(q_win), tensor4(k_pool), tensor4(v_pool), C.byref(pg),
                                       _ptr(modality), sb, sh, _ptr(seq_lens), _ptr(budgets), _ptr(total_budget),
                                       _ptr(lse), tensor4(k_out), tensor4(v_out), _ptr(mod_out), _ptr(n_out),
                                       _ptr(score_self), _ptr(score_cross), _ptr(keep_idx), _ptr(ws), ws.numel(),
                                       _stream()), "csp_prune_layer_paged")


def decode_attn_paged(p: Params, q, k_pool, v_pool, page_table, n_rows, out, ws):
    """csp_decode_attn over pools [n_pages, Hkv, page_rows, d] addressed through page_table int32 [B, max_pages]."""
    cp = p._c()
    assert q.dim() == 3 and q.stride(2) == 1 and out.is_contiguous() and out.dtype == torch.float32
    assert page_table.dtype == torch.int32 and page_table.is_contiguous() and page_table.dim() == 2
    qt = CTensor(q.data_ptr(), q.stride(0), q.stride(1), q.shape[2])
    pg = CPages(page_table.data_ptr(), page_table.shape[1], k_pool.shape[2], k_pool.shape[0])
    _check(lib().csp_decode_attn_paged(C.byref(cp), qt, tensor4(k_pool), tensor4(v_pool), C.byref(pg), _ptr(n_rows),
                                       _ptr(out), _ptr(ws), ws.numel(), _stream()), "csp_decode_attn_paged")


def _here(*tensors):
    """The kernels run on the current device: refuses tensors that live elsewhere."""
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"tensor on {t.device}, but the current device is cuda:{dev}")


def _counts(t: Optional[torch.Tensor], shape):
    if t is None:
        return None
    assert t.dtype is torch.int32 and t.shape == shape and t.is_contiguous(), f"int32 tensor of shape {tuple(shape)} expected"
    return t.data_ptr()


def _status_workspace(n: int, where: str, device) -> torch.Tensor:
    if n == 0:
        raise CspError(ERR_UNSUPPORTED, where)
    return torch.zeros(n, dtype=torch.uint8, device=device)


def chunk_workspace_bytes(p: Params, max_new: int) -> int:
    cp = p._c()
    return int(lib().csp_chunk_workspace_bytes(C.byref(cp), int(max_new)))


def new_chunk_workspace(p: Params, max_new: int, device="cuda") -> torch.Tensor:
    """Allocates (with torch) and zeroes a workspace for chunk_attn with chunks of up to max_new tokens."""
    return _status_workspace(chunk_workspace_bytes(p, max_new), "csp_chunk_workspace_bytes", device)


def _chunk_args(p: Params, q, k, v, n_rows, out, ws, n_new, mods, lse):
    _here(q, k, v, n_rows, out, ws, n_new, lse, *(mods.tensors() if mods is not None else ()))
    shape, ks, vs, bf16 = q.shape, k.shape, v.shape, torch.bfloat16
    assert len(shape) == 4 and shape[0] == p.batch and shape[1] == p.n_q_heads and shape[3] == p.head_dim and out.shape == shape, \
        f"q and out: [B, Hq, new tokens, d] = ({p.batch}, {p.n_q_heads}, new tokens, {p.head_dim})"
    assert q.dtype is bf16 and k.dtype is bf16 and v.dtype is bf16 and out.dtype is bf16, "bf16 tensors expected"
    assert ks[1] == vs[1] == p.n_kv_heads and ks[3] == vs[3] == p.head_dim
    assert lse is None or (lse.dtype is torch.float32 and lse.shape == shape[:3] and lse.is_contiguous())
    return shape[2], _counts(n_rows, (p.batch, p.n_kv_heads)), _counts(n_new, (p.batch,)), \
        None if mods is None else C.byref(mods.c(p))


def chunk_attn(p: Params, q, k, v, n_rows, out, ws, n_new=None, mods: Optional[ScoreMods] = None, lse=None):
    """q, out bf16 [B, Hq, new tokens, d] (any strides); k, v [B, Hkv, out_capacity, d]; n_rows int32 [B, Hkv], the new rows
    included; n_new int32 [B]; lse fp32 [B, Hq, new tokens]."""
    cp = p._c()
    T, rows, new, m = _chunk_args(p, q, k, v, n_rows, out, ws, n_new, mods, lse)
    assert k.shape[0] == v.shape[0] == p.batch and k.shape[2] >= p.out_capacity and v.shape[2] >= p.out_capacity
    _check(lib().csp_chunk_attn(C.byref(cp), T, tensor4(q), tensor4(k), tensor4(v), rows, new, m, tensor4(out), _ptr(lse),
                                _ptr(ws), ws.numel(), _stream()), "csp_chunk_attn")


def chunk_attn_paged(p: Params, q, k_pool, v_pool, page_table, n_rows, out, ws, n_new=None,
                     mods: Optional[ScoreMods] = None, lse=None):
    """chunk_attn over pools [n_pages, Hkv, page_rows, d] addressed through page_table int32 [B, max_pages]."""
    cp = p._c()
    T, rows, new, m = _chunk_args(p, q, k_pool, v_pool, n_rows, out, ws, n_new, mods, lse)
    pg = _pool_pages(p, k_pool, v_pool, page_table)
    _check(lib().csp_chunk_attn_paged(C.byref(cp), T, tensor4(q), tensor4(k_pool), tensor4(v_pool), C.byref(pg), rows, new, m,
                                      tensor4(out), _ptr(lse), _ptr(ws), ws.numel(), _stream()), "csp_chunk_attn_paged")


def _pool_pages(p: Params, k_pool, v_pool, page_table) -> CPages:
    _here(k_pool, v_pool, page_table)
    ts, ks = page_table.shape, k_pool.shape
    assert page_table.dtype is torch.int32 and len(ts) == 2 and ts[0] == p.batch and page_table.is_contiguous()
    assert len(ks) == 4 and v_pool.shape == ks
    return CPages(page_table.data_ptr(), ts[1], ks[2], ks[0])


def new_append_workspace(p: Params, device="cuda") -> torch.Tensor:
    """Allocates (with torch) and zeroes a workspace for append_paged and pages_copy."""
    cp = p._c()
    return _status_workspace(int(lib().csp_append_workspace_bytes(C.byref(cp))), "csp_append_workspace_bytes", device)


def _cache_dtype(p: Params, *tensors):
    want = torch.float32 if p.dtype == F32 else torch.bfloat16
    for t in tensors:
        ts = t.shape
        assert t.dtype is want and len(ts) == 4 and ts[1] == p.n_kv_heads and ts[3] == p.head_dim


def append_paged(p: Params, k_new, v_new, k_pool, v_pool, page_table, n_rows, n_rows_out, ws, n_new=None):
    """k_new, v_new [B, Hkv, new tokens, d] go behind the n_rows rows of every head; n_rows_out may be n_rows."""
    cp = p._c()
    _here(k_new, v_new, n_rows, n_rows_out, ws, n_new)
    pg = _pool_pages(p, k_pool, v_pool, page_table)
    _cache_dtype(p, k_new, v_new, k_pool, v_pool)
    assert k_new.shape == v_new.shape and k_new.shape[0] == p.batch
    _check(lib().csp_append_paged(C.byref(cp), k_new.shape[2], tensor4(k_new), tensor4(v_new), _counts(n_new, (p.batch,)),
                                  tensor4(k_pool), tensor4(v_pool), C.byref(pg), _counts(n_rows, (p.batch, p.n_kv_heads)),
                                  _counts(n_rows_out, (p.batch, p.n_kv_heads)), _ptr(ws), ws.numel(), _stream()),
           "csp_append_paged")


def new_pages_workspace(state: PageState, device="cuda") -> torch.Tensor:
    """Allocates (with torch) and zeroes a workspace for the pages_* calls."""
    cs = state.c()
    return _status_workspace(int(lib().csp_pages_workspace_bytes(C.byref(cs))), "csp_pages_workspace_bytes", device)


def _page_state(state: PageState, ws, *tensors) -> CPageState:
    _here(state.page_table, state.held, state.refs, state.n_rows, ws, *tensors)
    return state.c()


def _moves(moves, n_moves):
    ms = moves.shape
    assert moves.dtype is torch.int32 and len(ms) == 2 and ms[1] == 2 and moves.is_contiguous()
    return moves.data_ptr(), ms[0], _counts(n_moves, (1,))


def pages_fork(state: PageState, src, dst, ws):
    """Sequence dst[i] (which holds no pages) becomes a copy of src[i] that shares its pages; src, dst int32 [n]."""
    cs = _page_state(state, ws, src, dst)
    n = src.numel()
    _check(lib().csp_pages_fork(C.byref(cs), _counts(src, (n,)), _counts(dst, (n,)), n, _ptr(ws), ws.numel(), _stream()),
           "csp_pages_fork")


def pages_reserve(state: PageState, moves, n_moves, ws, n_new=None, whole: bool = False):
    """Room for n_new[b] more rows in pages of the sequence's own (whole: all of its pages); moves int32 [most, 2] and
    n_moves int32 [1] receive what pages_copy has to copy."""
    cs = _page_state(state, ws, moves, n_moves, n_new)
    m, most, n = _moves(moves, n_moves)
    _check(lib().csp_pages_reserve(C.byref(cs), _counts(n_new, (state.page_table.shape[0],)), int(whole), m, most, n, _ptr(ws),
                                   ws.numel(), _stream()), "csp_pages_reserve")


def pages_free(state: PageState, ws):
    """Pages behind the rows in use go back to the pool."""
    cs = _page_state(state, ws)
    _check(lib().csp_pages_free(C.byref(cs), _ptr(ws), ws.numel(), _stream()), "csp_pages_free")


def pages_compact(state: PageState, moves, n_moves, ws):
    """Moves the pages in use to the front of the pool; moves and n_moves as for pages_reserve."""
    cs = _page_state(state, ws, moves, n_moves)
    m, most, n = _moves(moves, n_moves)
    _check(lib().csp_pages_compact(C.byref(cs), m, most, n, _ptr(ws), ws.numel(), _stream()), "csp_pages_compact")


def pages_copy(p: Params, k_pool, v_pool, moves, n_moves, ws):
    """Copies the pages listed in moves, K and V, all heads: one call per layer."""
    cp = p._c()
    _here(k_pool, v_pool, moves, n_moves, ws)
    _cache_dtype(p, k_pool, v_pool)
    assert k_pool.shape == v_pool.shape
    m, most, n = _moves(moves, n_moves)
    _check(lib().csp_pages_copy(C.byref(cp), tensor4(k_pool), tensor4(v_pool), k_pool.shape[0], k_pool.shape[2], m, most, n,
                                _ptr(ws), ws.numel(), _stream()), "csp_pages_copy")


def static_workspace_limit() -> int:
    return int(lib().csp_static_workspace_limit())


def prune_layer_static(p: Params, q_win, k, v, modality, seq_lens, budgets, k_out, v_out, mod_out, n_out,
                       total_budget=None, lse=None, dev_status_out=None):
    """csp_prune_layer without a caller workspace: the library's built-in scratch array is used, so
    nothing is allocated.  Raises CspError(ERR_WORKSPACE) for shapes beyond static_workspace_limit()."""
    cp = p._c()
    sb, sh = _mod_strides(modality)
    _check(lib().csp_prune_layer_static(C.byref(cp), tensor4(q_win), tensor4(k), tensor4(v), _ptr(modality), sb, sh,
                                        _ptr(seq_lens), _ptr(budgets), _ptr(total_budget), _ptr(lse),
                                        tensor4(k_out), tensor4(v_out), _ptr(mod_out), _ptr(n_out),
                                        _ptr(dev_status_out), _stream()), "csp_prune_layer_static")


def host_staging_bytes(p: Params) -> int:
    cp = p._c()
    return int(lib().csp_host_staging_bytes(C.byref(cp)))


def prune_layer_host(p: Params, q, k, v, modality, seq_lens, budgets, k_out, v_out, mod_out, n_out,
                     staging: torch.Tensor, total_budget=None) -> int:
    """All tensors but `staging` are dense CPU tensors (pinned for asynchronous copies).
    Returns the device status word."""
    cp = p._c()
    for t in (q, k, v, modality, seq_lens, budgets, k_out, v_out, n_out):
        assert t.device.type == "cpu" and t.is_contiguous()
    word = C.c_int32(0)
    _check(lib().csp_prune_layer_host(C.byref(cp), _ptr(q), _ptr(k), _ptr(v), _ptr(modality),
                                      int(modality.dim() == 3), _ptr(seq_lens), _ptr(budgets),
                                      _ptr(total_budget), _ptr(k_out), _ptr(v_out), _ptr(mod_out),
                                      _ptr(n_out), C.addressof(word), _ptr(staging), staging.numel(),
                                      _stream()), "csp_prune_layer_host")
    return int(word.value)


def device_status(ws: torch.Tensor) -> int:
    """Waits for the current stream, returns the status word (CSP_DEV_* bits) and clears it."""
    word = C.c_int32(0)
    rc = lib().csp_device_status(_ptr(ws), _stream(), C.byref(word))
    if rc not in (OK, ERR_TIMEOUT):
        raise CspError(rc, "csp_device_status")
    return int(word.value)
