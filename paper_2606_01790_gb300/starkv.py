"""Thin Python binding of the C ABI in ``include/starkv.h`` (ctypes).

Argument marshalling only: every step of the compression stage runs in the
CUDA kernels of ``libstarkv.so``.  Tensors are torch tensors (device memory for
the device calls, host memory for ``step_host``); their data pointers are
handed to the library unchanged.  There is no fallback: if the library is not
built, importing the first call raises.
"""
from __future__ import annotations

import builtins
import ctypes as C
import struct
from dataclasses import dataclass, fields
from pathlib import Path
from typing import List, Optional, Sequence

import numpy as np
import torch

LIB_PATH = Path(__file__).resolve().parent / "libstarkv.so"

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_CUDA, ERR_TIMEOUT, ERR_NOMEM, ERR_DEVICE = range(7)

ABI_FUNCTIONS = [
    "starkv_default_config", "starkv_init_state", "starkv_reset_seq", "starkv_destroy_state",
    "starkv_get_config", "starkv_workspace_bytes", "starkv_score_layer", "starkv_select",
    "starkv_compact", "starkv_step", "starkv_step_host", "starkv_check_device_error",
    "starkv_set_wait_limit", "starkv_set_timing", "starkv_kernel_times", "starkv_backward_launches",
    "starkv_last_error",
    "starkv_score_layer_noalloc", "starkv_selftest_wait", "starkv_slot_state_bytes", "starkv_export_slot",
    "starkv_import_slot", "starkv_window_attention",
    "starkv_pages_workspace_bytes", "starkv_pages_reset", "starkv_pages_extend", "starkv_pages_fork",
    "starkv_pages_free", "starkv_pages_compact", "starkv_pages_store", "starkv_pages_load",
    "starkv_tree_attention", "starkv_sink_attention",
    "starkv_tree_mass", "starkv_sink_mass", "starkv_pages_evict", "starkv_pages_bounds",
    "starkv_sparse_workspace_bytes", "starkv_sparse_attention",
]

KERNELS = ["score_lse", "score_accum", "pool", "calibrate", "compact", "attention", "attn_combine",
           "page_book", "page_copy", "page_gather", "page_move", "paged_attention", "paged_combine",
           "mass", "mass_sum", "mass_select", "page_bounds", "page_choose"]


SELECT_GLOBAL, SELECT_PER_HEAD = 0, 1   # starkv_config.select_mode


class StarkvError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"starkv status {status}: {msg}")
        self.status = status


class CConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_layers", "n_heads", "n_kv_heads", "head_dim", "window", "grid_rows", "grid_cols",
        "pool_kernel", "mi_bins", "mi_grid", "n_warmup", "n_ramp", "max_seqs")] + \
        [(n, C.c_float) for n in (
            "lambda_", "tau", "rho_mi", "rho_t", "delta", "d_min", "t_min", "t_max", "eps", "eps_h")] + \
        [(n, C.c_int32) for n in ("select_mode", "decay_mode", "aeb_mode", "mi_span")]


class CSeq(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("q", C.c_void_p), ("meta", C.c_void_p),
                ("meta_layer_stride", C.c_int64), ("L", C.c_int32), ("cur_frame", C.c_int32),
                ("budget", C.c_int32), ("slot", C.c_int32), ("k_out", C.c_void_p),
                ("v_out", C.c_void_p), ("meta_out", C.c_void_p), ("idx", C.c_void_p),
                ("S", C.c_void_p), ("score", C.c_void_p), ("stats", C.c_void_p),
                ("meta_group_stride", C.c_int64), ("lse", C.c_void_p), ("attn_o", C.c_void_p),
                ("attn_lse", C.c_void_p)]


class CPages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("layer_stride", C.c_int64), ("page_stride", C.c_int64),
                ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_rows", C.c_int32), ("max_pages", C.c_int32),
                ("table", C.c_void_p), ("len", C.c_void_p), ("refs", C.c_void_p)]


class CTokens(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("rows", C.c_void_p), ("n_tokens", C.c_void_p),
                ("n", C.c_int32), ("T", C.c_int32), ("seq_stride", C.c_int64), ("layer_stride", C.c_int64),
                ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class CQueries(C.Structure):
    _fields_ = [("q", C.c_void_p), ("o", C.c_void_p), ("lse", C.c_void_p), ("mask", C.c_void_p),
                ("rows", C.c_void_p), ("n_tokens", C.c_void_p), ("n", C.c_int32), ("T", C.c_int32),
                ("q_seq_stride", C.c_int64), ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("o_seq_stride", C.c_int64), ("o_token_stride", C.c_int64), ("o_head_stride", C.c_int64)]


class CMass(C.Structure):
    _fields_ = [("mass", C.c_void_p), ("layer_stride", C.c_int64), ("row_stride", C.c_int64), ("group_stride", C.c_int64),
                ("decay", C.c_float)]


class CBounds(C.Structure):
    _fields_ = [("b", C.c_void_p), ("layer_stride", C.c_int64), ("page_stride", C.c_int64)]


_lib: Optional[C.CDLL] = None


class CSlotHeader(C.Structure):
    """``starkv_slot_header``: the first 32 bytes of an exported slot state."""
    _fields_ = [("magic", C.c_uint32), ("version", C.c_uint32), ("n_layers", C.c_int32),
                ("n_kv_heads", C.c_int32), ("grid_rows", C.c_int32), ("grid_cols", C.c_int32),
                ("reserved", C.c_uint32 * 2)]


SLOT_MAGIC = 0x31564B53


def slot_state_bytes_for(n_layers: int, G: int, RC: int) -> int:
    """STARKV_SLOT_STATE_BYTES of the header."""
    return C.sizeof(CSlotHeader) + ((n_layers * 4 + 7) & ~7) + n_layers * G * 8 + n_layers * G * RC * 4


def lib() -> C.CDLL:
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = C.CDLL(str(LIB_PATH))
        st = C.c_void_p
        for name in ("starkv_score_layer", "starkv_select", "starkv_compact"):
            getattr(L, name).argtypes = [st, C.c_int32, C.POINTER(CSeq), C.c_int32, C.c_void_p,
                                         C.c_size_t, C.c_void_p]
        for name in ("starkv_step", "starkv_step_host", "starkv_window_attention"):
            getattr(L, name).argtypes = [st, C.POINTER(CSeq), C.c_int32, C.c_void_p, C.c_size_t,
                                         C.c_void_p]
        L.starkv_score_layer_noalloc.argtypes = [st, C.c_int32, C.POINTER(CSeq), C.c_int32, C.c_void_p]
        L.starkv_default_config.argtypes = [C.POINTER(CConfig)]
        L.starkv_default_config.restype = None
        L.starkv_init_state.argtypes = [C.POINTER(CConfig), C.POINTER(C.c_void_p), C.c_void_p]
        L.starkv_reset_seq.argtypes = [st, C.c_int32, C.c_void_p]
        L.starkv_destroy_state.argtypes = [st]
        L.starkv_get_config.argtypes = [st, C.POINTER(CConfig)]
        L.starkv_workspace_bytes.argtypes = [st, C.POINTER(CSeq), C.c_int32, C.c_int32,
                                             C.POINTER(C.c_size_t)]
        L.starkv_check_device_error.argtypes = [st, C.c_void_p]
        L.starkv_set_wait_limit.argtypes = [st, C.c_uint64]
        L.starkv_selftest_wait.argtypes = [st, C.c_uint64, C.c_void_p]
        L.starkv_slot_state_bytes.argtypes = [st, C.POINTER(C.c_size_t)]
        L.starkv_export_slot.argtypes = [st, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]
        L.starkv_import_slot.argtypes = [st, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]
        L.starkv_set_timing.argtypes = [st, C.c_int32]
        L.starkv_kernel_times.argtypes = [st, C.POINTER(C.c_int64), C.POINTER(C.c_float)]
        L.starkv_backward_launches.argtypes = [st, C.POINTER(C.c_int64)]
        pg, ws = C.c_void_p, [C.c_void_p, C.c_size_t, C.c_void_p]
        L.starkv_pages_workspace_bytes.argtypes = [st, pg, C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        L.starkv_pages_reset.argtypes = [st, pg, C.c_void_p]
        L.starkv_pages_extend.argtypes = [st, pg, C.c_void_p, C.c_void_p, C.c_int32] + ws
        L.starkv_pages_fork.argtypes = [st, pg, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32] + ws
        L.starkv_pages_free.argtypes = [st, pg, C.c_void_p, C.c_int32, C.c_void_p]
        L.starkv_pages_compact.argtypes = [st, pg, C.c_void_p, C.POINTER(CSeq), C.c_int32] + ws
        for name in ("starkv_pages_store", "starkv_pages_load"):
            getattr(L, name).argtypes = [st, pg, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.starkv_tree_attention.argtypes = [st, pg, C.c_int32, C.c_void_p] + ws
        L.starkv_sink_attention.argtypes = [st, pg, C.c_int32, C.c_void_p, C.c_int32, C.c_int32] + ws
        L.starkv_tree_mass.argtypes = [st, pg, C.c_int32, C.c_void_p, C.c_void_p] + ws
        L.starkv_sink_mass.argtypes = [st, pg, C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p] + ws
        L.starkv_pages_evict.argtypes = [st, pg, C.c_void_p, C.POINTER(CSeq), C.c_int32, C.c_void_p] + ws
        L.starkv_pages_bounds.argtypes = [st, pg, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                          C.c_void_p]
        L.starkv_sparse_workspace_bytes.argtypes = [st, pg, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        L.starkv_sparse_attention.argtypes = [st, pg, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                              C.c_void_p] + ws
        L.starkv_last_error.argtypes = []
        L.starkv_last_error.restype = C.c_char_p
        for name in ABI_FUNCTIONS:
            if name not in ("starkv_default_config", "starkv_last_error"):
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != OK:
        raise StarkvError(status, lib().starkv_last_error().decode())


@dataclass
class Config:
    """Mirror of ``starkv_config`` (defaults: ``starkv_default_config``)."""

    n_layers: int = 28
    n_heads: int = 28
    n_kv_heads: int = 4
    head_dim: int = 128
    window: int = 32
    grid_rows: int = 52
    grid_cols: int = 52
    pool_kernel: int = 5
    mi_bins: int = 8
    mi_grid: int = 8
    n_warmup: int = 5
    n_ramp: int = 10
    max_seqs: int = 1
    lambda_: float = 0.5
    tau: float = 1.0
    rho_mi: float = 0.9
    rho_t: float = 0.9
    delta: float = 0.2
    d_min: float = 0.1
    t_min: float = 0.95
    t_max: float = 1.05
    eps: float = 1e-6
    eps_h: float = 1e-12
    select_mode: int = 0    # SELECT_GLOBAL (the paper's) or SELECT_PER_HEAD
    decay_mode: int = 0     # 0 exponential (Eq. 9), 1 linear, 2 power law (readings)
    aeb_mode: int = 0       # 0 entropy, 1 peak confidence (reading)
    mi_span: int = 0        # 0 every historical visual token, 1 the newest frame's

    def to_c(self) -> CConfig:
        c = CConfig()
        for f in fields(self):
            setattr(c, f.name, getattr(self, f.name))
        return c

    @staticmethod
    def default() -> "Config":
        c = CConfig()
        lib().starkv_default_config(c)
        return Config(**{f.name: getattr(c, f.name) for f in fields(Config)})


def stats_stride(n_kv_heads: int) -> int:
    """Floats per layer in a stats buffer (``STARKV_STATS_STRIDE``)."""
    return 8 + 6 * n_kv_heads


def sel_rows(cfg: "Config") -> int:
    """Rows of idx / score / meta_out per layer: 1 (global selection) or G (per KV head)."""
    return cfg.n_kv_heads if cfg.select_mode == SELECT_PER_HEAD else 1


def pack_meta(is_visual, frame, row, col) -> np.ndarray:
    """Token metadata words of the ABI: bit 31 visual, 20..30 frame, 10..19 row, 0..9 col."""
    v = np.asarray(is_visual).astype(np.uint32) != 0
    f = np.asarray(frame).astype(np.uint32)
    r = np.asarray(row).astype(np.uint32)
    c = np.asarray(col).astype(np.uint32)
    if (f > 2047).any() or (r > 1023).any() or (c > 1023).any():
        raise ValueError("frame / row / col out of the metadata word's range")
    out = (v.astype(np.uint32) << np.uint32(31)) | (f << np.uint32(20)) | (r << np.uint32(10)) | c
    return np.where(v, out, np.uint32(0)).astype(np.uint32)


def unpack_meta(words: np.ndarray):
    w = np.asarray(words).astype(np.uint32)
    return ((w >> 31) & 1).astype(np.int32), ((w >> 20) & 0x7FF).astype(np.int32), \
        ((w >> 10) & 0x3FF).astype(np.int32), (w & 0x3FF).astype(np.int32)


def meta_tensor(words: np.ndarray) -> torch.Tensor:
    """uint32 metadata as an int32 tensor with the same bits (torch has no uint32 math)."""
    return torch.from_numpy(np.ascontiguousarray(words).view(np.int32))


@dataclass
class Seq:
    """One sequence of a call (``starkv_seq``).  Tensor layouts as in starkv.h."""

    k: Optional[torch.Tensor] = None
    v: Optional[torch.Tensor] = None
    q: Optional[torch.Tensor] = None
    meta: Optional[torch.Tensor] = None     # int32 view of the u32 words
    meta_layer_stride: int = 0
    L: int = 0
    cur_frame: int = 0
    budget: int = 0
    slot: int = 0
    k_out: Optional[torch.Tensor] = None
    v_out: Optional[torch.Tensor] = None
    meta_out: Optional[torch.Tensor] = None
    idx: Optional[torch.Tensor] = None
    S: Optional[torch.Tensor] = None
    score: Optional[torch.Tensor] = None
    stats: Optional[torch.Tensor] = None
    meta_group_stride: int = 0              # per-KV-head mode: one metadata row per group
    lse: Optional[torch.Tensor] = None      # f32 [n_layers][H][w] supplied row normalisers
    attn_o: Optional[torch.Tensor] = None   # f32 [n_layers][H][w][d] window_attention output
    attn_lse: Optional[torch.Tensor] = None  # f32 [n_layers][H][w] window_attention normalisers

    def to_c(self) -> CSeq:
        s = CSeq()
        for name in ("k", "v", "q", "meta", "k_out", "v_out", "meta_out", "idx", "S", "score", "stats", "lse",
                     "attn_o", "attn_lse"):
            setattr(s, name, _ptr(getattr(self, name)))
        s.meta_layer_stride = self.meta_layer_stride
        s.meta_group_stride = self.meta_group_stride
        s.L, s.cur_frame, s.budget, s.slot = self.L, self.cur_frame, self.budget, self.slot
        return s


# The fields of ``starkv_seq`` in order, packed in one go: a call marshals its
# sequences every time (nothing is kept of them), and one ctypes attribute store
# per field cost more than the launch it led to.  Values that do not pack go
# through ``Seq.to_c``, with ctypes' own conversions and errors.
_SEQ = struct.Struct("@4Pq4i7Pq3P")
assert _SEQ.size == C.sizeof(CSeq)


def _ptr(t: Optional[torch.Tensor]) -> int:
    if t is None:
        return 0
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _pack_seq(s: Seq) -> bytes:
    ptr = _ptr
    try:
        return _SEQ.pack(ptr(s.k), ptr(s.v), ptr(s.q), ptr(s.meta), s.meta_layer_stride, s.L, s.cur_frame, s.budget,
                         s.slot, ptr(s.k_out), ptr(s.v_out), ptr(s.meta_out), ptr(s.idx), ptr(s.S), ptr(s.score),
                         ptr(s.stats), s.meta_group_stride, ptr(s.lse), ptr(s.attn_o), ptr(s.attn_lse))
    except struct.error:
        return bytes(s.to_c())


def _seq_array(seqs: Sequence[Seq]):
    """The ``starkv_seq`` array of a call (one entry for an empty batch)."""
    buf = b"".join([_pack_seq(s) for s in seqs]) or bytes(_SEQ.size)
    return (CSeq * (len(buf) // _SEQ.size)).from_buffer_copy(buf)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if torch.cuda.is_initialized() and _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else 0
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


class State:
    """Owns a ``starkv_state`` (device-resident per-(slot, layer) state)."""

    def __init__(self, cfg: Config, stream=None):
        self.cfg = cfg
        self._c = cfg.to_c()
        h = C.c_void_p()
        _check(lib().starkv_init_state(C.byref(self._c), C.byref(h), _stream(stream)))
        self.handle = h

    def close(self) -> None:
        if self.handle:
            _check(lib().starkv_destroy_state(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def init_state(cfg: Config, stream=None) -> State:
    return State(cfg, stream)


def destroy_state(st: State) -> None:
    st.close()


def reset_seq(st: State, slot: int, stream=None) -> None:
    _check(lib().starkv_reset_seq(st.handle, slot, _stream(stream)))


def set_wait_limit(st: State, limit_ns: int) -> None:
    _check(lib().starkv_set_wait_limit(st.handle, int(limit_ns)))


def slot_state_bytes(st: State) -> int:
    n = C.c_size_t(0)
    _check(lib().starkv_slot_state_bytes(st.handle, C.byref(n)))
    return int(n.value)


def export_slot(st: State, slot: int, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Slot ``slot``'s carried state (n, MI EMA, m_g of every layer) as a uint8
    host tensor (page-locked unless ``out`` is given); valid once the stream
    has been synchronised."""
    n = slot_state_bytes(st)
    if out is None:
        out = torch.empty(n, dtype=torch.uint8, pin_memory=torch.cuda.is_available())
    _check(lib().starkv_export_slot(st.handle, int(slot), out.data_ptr(), out.numel() * out.element_size(),
                                    _stream(stream)))
    return out


def import_slot(st: State, slot: int, buf: torch.Tensor, stream=None) -> None:
    """Replaces slot ``slot``'s carried state with one written by ``export_slot``."""
    _check(lib().starkv_import_slot(st.handle, int(slot), buf.data_ptr(), buf.numel() * buf.element_size(),
                                    _stream(stream)))


def selftest_wait(st: State, limit_ns: int, stream=None) -> None:
    """Runs the bounded-wait failure path once: a device wait that nothing
    completes gives up after ``limit_ns`` and latches ERR_TIMEOUT, which the
    next ``check_device_error`` raises."""
    _check(lib().starkv_selftest_wait(st.handle, int(limit_ns), _stream(stream)))


def workspace_bytes(st: State, seqs: Sequence[Seq], host: bool = False) -> int:
    arr = _seq_array(seqs)
    n = C.c_size_t()
    _check(lib().starkv_workspace_bytes(st.handle, arr, len(seqs), int(host), C.byref(n)))
    return int(n.value)


def workspace(st: State, seqs: Sequence[Seq], host: bool = False, device=None) -> torch.Tensor:
    return torch.empty(workspace_bytes(st, seqs, host), dtype=torch.uint8,
                       device=device or torch.device("cuda"))


def _call_layer(fn, st: State, layer: int, seqs: Sequence[Seq], ws: torch.Tensor, stream) -> None:
    arr = _seq_array(seqs)
    _check(fn(st.handle, layer, arr, len(seqs), ws.data_ptr(), ws.numel(), _stream(stream)))


def score_layer(st: State, layer: int, seqs: Sequence[Seq], ws: torch.Tensor, stream=None) -> None:
    _call_layer(lib().starkv_score_layer, st, layer, seqs, ws, stream)


def score_layer_noalloc(st: State, layer: int, seqs: Sequence[Seq], stream=None) -> None:
    """``starkv_score_layer`` without a workspace: for callers that cannot
    allocate device memory; the library's static 16 MiB scratch is used."""
    arr = _seq_array(seqs)
    _check(lib().starkv_score_layer_noalloc(st.handle, layer, arr, len(seqs), _stream(stream)))


def select(st: State, layer: int, seqs: Sequence[Seq], ws: torch.Tensor, stream=None) -> None:
    _call_layer(lib().starkv_select, st, layer, seqs, ws, stream)


def compact(st: State, layer: int, seqs: Sequence[Seq], ws: torch.Tensor, stream=None) -> None:
    _call_layer(lib().starkv_compact, st, layer, seqs, ws, stream)


def step(st: State, seqs: Sequence[Seq], ws: torch.Tensor, stream=None) -> None:
    arr = _seq_array(seqs)
    _check(lib().starkv_step(st.handle, arr, len(seqs), ws.data_ptr(), ws.numel(), _stream(stream)))


def window_attention(st: State, seqs: Sequence[Seq], ws: torch.Tensor, stream=None) -> None:
    """Attention output (``attn_o``, optional) and normaliser (``attn_lse``) of
    the window rows over the past keys, for every layer of every sequence."""
    arr = _seq_array(seqs)
    _check(lib().starkv_window_attention(st.handle, arr, len(seqs), ws.data_ptr(), ws.numel(),
                                         _stream(stream)))


def step_host(st: State, seqs: Sequence[Seq], ws: torch.Tensor, stream=None) -> None:
    arr = _seq_array(seqs)
    _check(lib().starkv_step_host(st.handle, arr, len(seqs), ws.data_ptr(), ws.numel(),
                                  _stream(stream)))


def check_device_error(st: State, stream=None) -> None:
    _check(lib().starkv_check_device_error(st.handle, _stream(stream)))


def device_error_status(st: State, stream=None) -> int:
    return lib().starkv_check_device_error(st.handle, _stream(stream))


def set_timing(st: State, on: bool) -> None:
    _check(lib().starkv_set_timing(st.handle, int(on)))


def kernel_times(st: State):
    """{kernel: (launches, total_ms)} since the previous read."""
    n = len(KERNELS)
    launches = (C.c_int64 * n)()
    ms = (C.c_float * n)()
    _check(lib().starkv_kernel_times(st.handle, launches, ms))
    return {k: (int(launches[i]), float(ms[i])) for i, k in enumerate(KERNELS)}


def backward_launches(st: State) -> int:
    """Launches of scoring pass 2 that went through their tiles backwards, so far."""
    n = C.c_int64(0)
    _check(lib().starkv_backward_launches(st.handle, C.byref(n)))
    return int(n.value)


# ---------------------------------------------------------------- paged cache

class Pages:
    """A paged cache (``starkv_pages``): pool, page table, lengths and page counts, all the
    caller's.  The tensors are checked once, when the object is made, and stay its own.

    k, v   bf16 [n_layers][n_pages][G][page_size][d], the last three contiguous, the same strides
    table  i32 [n_rows][max_pages];  len  i32 [n_rows];  refs  i32 [n_pages]
    """

    __slots__ = ("_k", "_v", "_table", "_len", "_refs", "_packed", "_shape", "_device")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, len: torch.Tensor, refs: torch.Tensor):
        if k.dim() != 5 or v.shape != k.shape or v.stride() != k.stride():
            raise ValueError("pages: k and v are [n_layers, n_pages, G, page_size, d] with the same strides")
        nl, n_pages, G, P, d = k.shape
        if k.stride()[2:] != (P * d, d, 1):
            raise ValueError("pages: a page of a layer must be contiguous")
        _expect(torch.bfloat16, k, v)
        _expect(torch.int32, table, len, refs)
        if table.dim() != 2 or len.numel() != table.shape[0] or refs.numel() != n_pages:
            raise ValueError("pages: table is [n_rows, max_pages], len [n_rows], refs [n_pages]")
        if builtins.len({t.device for t in (k, v, table, len, refs)}) != 1:
            raise ValueError("pages: tensors on more than one device")
        self._k, self._v, self._table, self._len, self._refs = k, v, table, len, refs
        self._shape, self._device = (nl, G, d), k.get_device()
        self._packed = bytes(CPages(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), n_pages, P, *table.shape,
                                    _ptr(table), _ptr(len), _ptr(refs)))

    k = property(lambda self: self._k)
    v = property(lambda self: self._v)
    table = property(lambda self: self._table)
    len = property(lambda self: self._len)
    refs = property(lambda self: self._refs)

    def to_c(self) -> CPages:
        return CPages.from_buffer_copy(self._packed)


@dataclass
class Tokens:
    """Tokens outside the pages (``starkv_tokens``): the last n_tokens[i] of row rows[i]."""

    k: torch.Tensor                          # bf16 [n][layers][T][G][d], any strides with d contiguous
    v: Optional[torch.Tensor] = None         # the same, or None: keys only
    rows: Optional[torch.Tensor] = None      # i32 [n], or None: rows 0, 1, ...
    n_tokens: Optional[torch.Tensor] = None  # i32 [n], or None: T each


@dataclass
class Queries:
    """Queries of the attention calls and of the mass calls (``starkv_queries``)."""

    q: torch.Tensor                          # bf16 [n][T][H][d], any strides with d contiguous
    o: Optional[torch.Tensor] = None         # bf16, the same shape (attention; the mass calls do not look at it)
    lse: Optional[torch.Tensor] = None       # f32 [n][T][H] (the mass calls read it)
    mask: Optional[torch.Tensor] = None      # i64 [n][T] (the bits of the u64 words), tree calls only
    rows: Optional[torch.Tensor] = None      # i32 [n], or None: rows 0, 1, ...
    n_tokens: Optional[torch.Tensor] = None  # i32 [n], or None: T each


def _expect(dtype: torch.dtype, *tensors: Optional[torch.Tensor]) -> None:
    for t in tensors:
        if t is not None and t.dtype != dtype:
            raise ValueError(f"expected {dtype}, got {t.dtype}")


def _on(pages: Pages, *tensors: Optional[torch.Tensor]) -> None:
    """The call's tensors lie where its pages do."""
    dev = pages._device
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"a tensor on {t.device}, pages on {pages.k.device}")


def _stream_on(pages: Pages, stream) -> int:
    """The stream of a call whose pages lie on the current CUDA device."""
    dev = pages._device
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError(f"pages on {pages.k.device}: the paged calls take tensors of the current CUDA device")
    return _raw_stream(dev) if stream is None and _raw_stream is not None else _stream(stream)


def _ids(t: Optional[torch.Tensor], n: int, what: str) -> int:
    if t is None:
        return 0
    if t.dtype is not torch.int32:
        raise ValueError(f"expected {torch.int32}, got {t.dtype}")
    if t.numel() != n:
        raise ValueError(f"{what}: {t.numel()} entries for {n} sequences")
    return _ptr(t)


_TOKENS = struct.Struct("@4P2i4q")
_QUERIES = struct.Struct("@6P2i6q")
assert _TOKENS.size == C.sizeof(CTokens) and _QUERIES.size == C.sizeof(CQueries)


def _c_tokens(st: State, pages: Pages, tok: Tokens) -> bytes:
    k, v, rows, count = tok.k, tok.v, tok.rows, tok.n_tokens
    if k.dim() != 5:
        raise ValueError("tokens: k is [n, layers, T, G, d]")
    n, nl, T, G, d = k.shape
    s0, s1, s2, s3, s4 = k.stride()
    if G != st.cfg.n_kv_heads or d != st.cfg.head_dim or s4 != 1:
        raise ValueError("tokens: k is [n, layers, T, G, d] with d contiguous")
    if v is not None and (v.shape != k.shape or v.stride() != k.stride()):
        raise ValueError("tokens: v has k's shape and strides")
    if k.dtype is not torch.bfloat16 or (v is not None and v.dtype is not torch.bfloat16):
        raise ValueError(f"tokens: expected {torch.bfloat16}")
    _on(pages, k, v, rows, count)
    # (an axis of one entry is never stepped along: its stride may be any)
    return _TOKENS.pack(k.data_ptr(), 0 if v is None else v.data_ptr(), _ids(rows, n, "rows"), _ids(count, n, "n_tokens"), n, T,
                        s0 if n > 1 else d, s1 if nl > 1 else d, s2 if T > 1 else d, s3 if G > 1 else d)


def _c_queries(st: State, pages: Pages, qs: Queries, weigh: bool = False) -> bytes:
    q, o, lse, mask, rows, count = qs.q, qs.o, qs.lse, qs.mask, qs.rows, qs.n_tokens
    if weigh:     # (a mass call does not look at o)
        o = q
        if lse is None:
            raise ValueError("queries: lse is missing")
    if q.dim() != 4 or o is None or o.shape != q.shape:
        raise ValueError("queries: q is [n, T, H, d], o of the same shape")
    n, T, H, d = q.shape
    s0, s1, s2, s3 = q.stride()
    o0, o1, o2, o3 = (s0, s1, s2, s3) if weigh else o.stride()
    if H != st.cfg.n_heads or d != st.cfg.head_dim or s3 != 1 or o3 != 1:
        raise ValueError("queries: q and o are [n, T, H, d] with d contiguous")
    if q.dtype is not torch.bfloat16 or o.dtype is not torch.bfloat16:
        raise ValueError(f"queries: expected {torch.bfloat16}, got {q.dtype} and {o.dtype}")
    _on(pages, q, o, lse, mask, rows, count)
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (n, T, H)):
        raise ValueError("queries: lse is f32 [n, T, H]")
    if mask is not None and (mask.dtype is not torch.int64 or mask.shape != (n, T)):
        raise ValueError("queries: mask is i64 [n, T]")
    if n < 2:      # (an axis of one entry is never stepped along: its stride may be any)
        s0 = o0 = d
    if T < 2:
        s1 = o1 = d
    if H < 2:
        s2 = o2 = d
    return _QUERIES.pack(q.data_ptr(), o.data_ptr(), _ptr(lse), _ptr(mask), _ids(rows, n, "rows"),
                         _ids(count, n, "n_tokens"), n, T, s0, s1, s2, o0, o1, o2)


def _c_pages(st: State, pages: Pages) -> bytes:
    cfg = st.cfg
    if pages._shape != (cfg.n_layers, cfg.n_kv_heads, cfg.head_dim):
        raise ValueError("pages: k is not of the state's layers, KV heads and head dimension")
    return pages._packed


def make_pages(st: State, n_pages: int, page_size: int, n_rows: int, max_pages: int, device=None, stream=None) -> Pages:
    """An empty paged cache in newly allocated tensors."""
    dev = device or torch.device("cuda", torch.cuda.current_device())
    shape = (st.cfg.n_layers, n_pages, st.cfg.n_kv_heads, page_size, st.cfg.head_dim)
    pages = Pages(k=torch.empty(shape, dtype=torch.bfloat16, device=dev),
                  v=torch.empty(shape, dtype=torch.bfloat16, device=dev),
                  table=torch.zeros((n_rows, max_pages), dtype=torch.int32, device=dev),
                  len=torch.empty(n_rows, dtype=torch.int32, device=dev),
                  refs=torch.empty(n_pages, dtype=torch.int32, device=dev))
    pages_reset(st, pages, stream)
    return pages


def pages_workspace(st: State, pages: Pages, n: int, T: int = 1) -> torch.Tensor:
    """Workspace for the paged calls over at most ``n`` rows and ``T`` queries of each."""
    b = C.c_size_t()
    _check(lib().starkv_pages_workspace_bytes(st.handle, _c_pages(st, pages), n, T, C.byref(b)))
    return torch.empty(int(b.value), dtype=torch.uint8, device=pages.k.device)


def pages_reset(st: State, pages: Pages, stream=None) -> None:
    c = _c_pages(st, pages)
    _check(lib().starkv_pages_reset(st.handle, c, _stream_on(pages, stream)))


def pages_extend(st: State, pages: Pages, rows: Optional[torch.Tensor], n_new: torch.Tensor, ws: torch.Tensor,
                 stream=None) -> None:
    """Room for ``n_new[i]`` more tokens of ``rows[i]``; shared last pages are copied first."""
    c, n = _c_pages(st, pages), n_new.numel()
    _on(pages, rows, n_new, ws)
    _check(lib().starkv_pages_extend(st.handle, c, _ids(rows, n, "rows"), _ids(n_new, n, "n_new"), n,
                                     _ptr(ws), ws.numel(), _stream_on(pages, stream)))


def pages_fork(st: State, pages: Pages, src: torch.Tensor, dst: torch.Tensor, ws: torch.Tensor, deep: bool = False,
               stream=None) -> None:
    """Row ``dst[i]`` becomes a copy of ``src[i]``, sharing its pages (``deep``: with pages of its own)."""
    c, n = _c_pages(st, pages), dst.numel()
    _on(pages, src, dst, ws)
    _check(lib().starkv_pages_fork(st.handle, c, _ids(src, n, "src"), _ids(dst, n, "dst"), n, int(deep),
                                   _ptr(ws), ws.numel(), _stream_on(pages, stream)))


def pages_free(st: State, pages: Pages, rows: torch.Tensor, stream=None) -> None:
    """Empties rows; pages that no row holds any more are free."""
    c, n = _c_pages(st, pages), rows.numel()
    _on(pages, rows)
    _check(lib().starkv_pages_free(st.handle, c, _ids(rows, n, "rows"), n, _stream_on(pages, stream)))


def _check_kept(cfg: Config, i: int, s: Seq) -> None:
    """What a compaction reads and writes of a sequence: 32-bit words, as many as the call goes through."""
    rows, B, n = sel_rows(cfg), s.budget, s.budget + cfg.window
    for name, t, kinds, last, need in (("idx", s.idx, (torch.int32,), B, cfg.n_layers * rows * B),
                                       ("meta_out", s.meta_out, _WORDS, n, cfg.n_layers * rows * n),
                                       ("meta", s.meta, _WORDS, None,
                                        (cfg.n_layers - 1) * s.meta_layer_stride + (rows - 1) * s.meta_group_stride + s.L)):
        if t is None:
            continue
        if t.dtype not in kinds:
            raise ValueError(f"seq {i}: {name}: expected {kinds[0]}, got {t.dtype}")
        if t.numel() < need or (last and t.dim() > 1 and t.shape[-1] != last):
            raise ValueError(f"seq {i}: {name} of shape {tuple(t.shape)}: the call goes through {need} words"
                             + ("" if last is None else f", {last} a row"))


_WORDS = (torch.int32, torch.uint32)


def pages_compact(st: State, pages: Pages, rows: Optional[torch.Tensor], seqs: Sequence[Seq], ws: torch.Tensor,
                  stream=None) -> None:
    """Every layer of ``rows[i]`` keeps the tokens ``seqs[i].idx`` and the window (``starkv_compact`` on pages)."""
    c = _c_pages(st, pages)
    _on(pages, rows, ws, *(t for s in seqs for t in (s.idx, s.meta, s.meta_out)))
    for i, s in enumerate(seqs):
        _check_kept(st.cfg, i, s)
    _check(lib().starkv_pages_compact(st.handle, c, _ids(rows, len(seqs), "rows"), _seq_array(seqs), len(seqs),
                                      _ptr(ws), ws.numel(), _stream_on(pages, stream)))


def pages_store(st: State, pages: Pages, layer0: int, tokens: Tokens, stream=None) -> None:
    """``tokens`` into the last places of their rows, layers layer0, layer0 + 1, ..."""
    c, tok = _c_pages(st, pages), _c_tokens(st, pages, tokens)
    _check(lib().starkv_pages_store(st.handle, c, layer0, tokens.k.shape[1], tok, _stream_on(pages, stream)))


def pages_load(st: State, pages: Pages, layer0: int, tokens: Tokens, stream=None) -> None:
    """The last tokens of their rows into ``tokens``."""
    c, tok = _c_pages(st, pages), _c_tokens(st, pages, tokens)
    _check(lib().starkv_pages_load(st.handle, c, layer0, tokens.k.shape[1], tok, _stream_on(pages, stream)))


def tree_attention(st: State, pages: Pages, layer: int, queries: Queries, ws: torch.Tensor, stream=None) -> None:
    """Attention of each row's last (drafted) tokens over its cache; ``queries.mask`` names the drafted ones seen."""
    c, q = _c_pages(st, pages), _c_queries(st, pages, queries)
    _on(pages, ws)
    _check(lib().starkv_tree_attention(st.handle, c, layer, q, _ptr(ws), ws.numel(),
                                       _stream_on(pages, stream)))


def sink_attention(st: State, pages: Pages, layer: int, queries: Queries, n_sink: int, window: int, ws: torch.Tensor,
                   stream=None) -> None:
    """Causal attention over the first ``n_sink`` tokens and the last ``window``."""
    c, q = _c_pages(st, pages), _c_queries(st, pages, queries)
    _on(pages, ws)
    _check(lib().starkv_sink_attention(st.handle, c, layer, q, n_sink, window, _ptr(ws),
                                       ws.numel(), _stream_on(pages, stream)))


# ---------------------------------------------------------------- attention mass, chosen pages

_MASS, _BOUNDS = struct.Struct("@P3qf4x"), struct.Struct("@P2q")
assert _MASS.size == C.sizeof(CMass) and _BOUNDS.size == C.sizeof(CBounds)


class Mass:
    """What each cached token has had of the queries' attention (``starkv_mass``).  The tensor is checked once, when the
    object is made, and stays its own.

    data   f32 [n_layers][n_rows][G][tokens], tokens contiguous, max_pages * page_size of them or more
    decay  factor of what a token has had so far, when a call adds to it
    """

    __slots__ = ("_data", "_decay", "_packed", "_shape")

    def __init__(self, data: torch.Tensor, decay: float = 1.0):
        if data.dim() != 4 or data.stride(3) != 1:
            raise ValueError("mass: data is [n_layers, n_rows, G, tokens] with the tokens contiguous")
        _expect(torch.float32, data)
        self._data, self._decay = data, float(decay)
        layers, rows, groups, tokens = data.shape
        self._shape = layers, rows, groups, tokens
        s0, s1, s2, _ = data.stride()
        # (an axis of one entry is never stepped along: its stride may be any)
        words = (data.data_ptr(), s0 if layers > 1 else tokens, s1 if rows > 1 else tokens, s2 if groups > 1 else tokens)
        try:
            self._packed = _MASS.pack(*words, self._decay)
        except OverflowError:      # (past 32 bits: infinity, which the calls refuse)
            self._packed = bytes(CMass(*words, self._decay))

    data = property(lambda self: self._data)
    decay = property(lambda self: self._decay)


def make_mass(st: State, pages: Pages, decay: float = 1.0) -> Mass:
    """A mass for the rows of ``pages`` (the calls that add to it start new tokens at 0)."""
    rows, max_pages = pages.table.shape
    return Mass(torch.zeros((st.cfg.n_layers, rows, st.cfg.n_kv_heads, max_pages * pages.k.shape[3]), dtype=torch.float32,
                            device=pages.k.device), decay)


def _c_mass(st: State, pages: Pages, mass: Mass) -> bytes:
    layers, rows, groups, tokens = mass._shape
    n_rows, max_pages = pages.table.shape
    if layers != st.cfg.n_layers or rows != n_rows or groups != st.cfg.n_kv_heads or tokens < max_pages * pages.k.shape[3]:
        raise ValueError("mass: data is [n_layers, n_rows, G, max_pages * page_size or more]")
    _on(pages, mass._data)
    return mass._packed


def tree_mass(st: State, pages: Pages, layer: int, queries: Queries, mass: Mass, ws: torch.Tensor, stream=None) -> None:
    """Adds the weights of ``tree_attention`` with the same queries (their ``lse`` as it wrote it) to ``mass``."""
    c, q, m = _c_pages(st, pages), _c_queries(st, pages, queries, True), _c_mass(st, pages, mass)
    _on(pages, ws)
    _check(lib().starkv_tree_mass(st.handle, c, layer, q, m, _ptr(ws), ws.numel(), _stream_on(pages, stream)))


def sink_mass(st: State, pages: Pages, layer: int, queries: Queries, n_sink: int, window: int, mass: Mass, ws: torch.Tensor,
              stream=None) -> None:
    """Adds the weights of ``sink_attention`` with the same queries (their ``lse`` as it wrote it) to ``mass``."""
    c, q, m = _c_pages(st, pages), _c_queries(st, pages, queries, True), _c_mass(st, pages, mass)
    _on(pages, ws)
    _check(lib().starkv_sink_mass(st.handle, c, layer, q, n_sink, window, m, _ptr(ws), ws.numel(), _stream_on(pages, stream)))


def pages_evict(st: State, pages: Pages, rows: Optional[torch.Tensor], seqs: Sequence[Seq], mass: Mass, ws: torch.Tensor,
                stream=None) -> None:
    """Every layer of ``rows[i]`` keeps the ``seqs[i].budget`` past tokens of greatest mass (written to ``seqs[i].idx``) and
    the window; their mass moves with them."""
    c, m = _c_pages(st, pages), _c_mass(st, pages, mass)
    _on(pages, rows, ws, *(t for s in seqs for t in (s.idx, s.meta, s.meta_out)))
    for i, s in enumerate(seqs):
        _check_kept(st.cfg, i, s)
    _check(lib().starkv_pages_evict(st.handle, c, _ids(rows, len(seqs), "rows"), _seq_array(seqs), len(seqs), m,
                                    _ptr(ws), ws.numel(), _stream_on(pages, stream)))


def make_bounds(st: State, pages: Pages) -> torch.Tensor:
    """Room for the bounds of every page: bf16 [n_layers][n_pages][G][2][d], least keys first."""
    return torch.empty((st.cfg.n_layers, pages.k.shape[1], st.cfg.n_kv_heads, 2, st.cfg.head_dim), dtype=torch.bfloat16,
                       device=pages.k.device)


def _c_bounds(st: State, pages: Pages, bounds: torch.Tensor) -> bytes:
    layers, n_pages, G, _, d = shape = (st.cfg.n_layers, pages.k.shape[1], st.cfg.n_kv_heads, 2, st.cfg.head_dim)
    strides = bounds.stride()
    if bounds.shape != shape or strides[2:] != (2 * d, d, 1):
        raise ValueError("bounds: [n_layers, n_pages, G, 2, d], a page of a layer contiguous")
    _expect(torch.bfloat16, bounds)
    _on(pages, bounds)
    # (an axis of one entry is never stepped along: its stride may be any)
    page = 2 * G * d
    return _BOUNDS.pack(bounds.data_ptr(), strides[0] if layers > 1 else page, strides[1] if n_pages > 1 else page)


def pages_bounds(st: State, pages: Pages, layer0: int, n_layers: int, bounds: torch.Tensor, T: int,
                 rows: Optional[torch.Tensor] = None, n_tokens: Optional[torch.Tensor] = None, stream=None) -> None:
    """Bounds of the pages that hold the last ``n_tokens[i]`` (at most ``T``; None: ``T``) tokens of ``rows[i]`` (None: of
    every row)."""
    c, b = _c_pages(st, pages), _c_bounds(st, pages, bounds)
    n = rows.numel() if rows is not None else n_tokens.numel() if n_tokens is not None else pages.table.shape[0]
    _on(pages, rows, n_tokens)
    _check(lib().starkv_pages_bounds(st.handle, c, layer0, n_layers, b, _ids(rows, n, "rows"), _ids(n_tokens, n, "n_tokens"), n, T,
                                     _stream_on(pages, stream)))


def sparse_workspace(st: State, pages: Pages, n: int, T: int, n_chosen: int) -> torch.Tensor:
    """Workspace for ``sparse_attention`` over at most ``n`` rows, ``T`` queries of each and ``n_chosen`` pages."""
    b = C.c_size_t()
    _check(lib().starkv_sparse_workspace_bytes(st.handle, _c_pages(st, pages), n, T, n_chosen, C.byref(b)))
    return torch.empty(int(b.value), dtype=torch.uint8, device=pages.k.device)


def sparse_attention(st: State, pages: Pages, layer: int, queries: Queries, bounds: torch.Tensor, n_first: int, n_last: int,
                     n_chosen: int, ws: torch.Tensor, chosen_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """Causal attention of each query over ``n_chosen`` pages per KV head: the first ``n_first``, the last ``n_last`` and
    the best of the others by their bounds (``chosen_out``, i32 [n][T][G][n_chosen]: their places in the row)."""
    c, q, b = _c_pages(st, pages), _c_queries(st, pages, queries), _c_bounds(st, pages, bounds)
    _on(pages, ws, chosen_out)
    if chosen_out is not None:
        _expect(torch.int32, chosen_out)
        n, T, _, _ = queries.q.shape
        if chosen_out.shape != (n, T, st.cfg.n_kv_heads, n_chosen):
            raise ValueError("chosen_out: [n, T, G, n_chosen]")
    _check(lib().starkv_sparse_attention(st.handle, c, layer, q, b, n_first, n_last, n_chosen, _ptr(chosen_out), _ptr(ws), ws.numel(),
                                         _stream_on(pages, stream)))
