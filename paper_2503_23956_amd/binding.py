"""ctypes binding of libaircache.so: same names as the C ABI, argument marshalling only.

Every step of the hot path runs in the HIP library; PyTorch only owns device memory and the
stream.  There is no CPU fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libaircache.so")

AIR_OK = 0
AIR_ERR_INVALID_ARG, AIR_ERR_SHAPE, AIR_ERR_WORKSPACE, AIR_ERR_STATE, AIR_ERR_HIP = 1, 2, 3, 4, 5
AIR_F32, AIR_BF16 = 0, 1
AIR_BUDGET_STRENGTH_SKEW, AIR_BUDGET_UNIFORM, AIR_BUDGET_STRENGTH, AIR_BUDGET_SKEW = 0, 1, 2, 3
AIR_WINDOW_TEXT, AIR_WINDOW_VISUAL = 0, 1
AIR_ROPE_HALF, AIR_ROPE_INTERLEAVED = 0, 1
AIR_ROPE_PLAIN, AIR_ROPE_LINEAR, AIR_ROPE_BY_PARTS = 0, 1, 2
_STATUS_NAMES = {0: "AIR_OK", 1: "AIR_ERR_INVALID_ARG", 2: "AIR_ERR_SHAPE", 3: "AIR_ERR_WORKSPACE",
                 4: "AIR_ERR_STATE", 5: "AIR_ERR_HIP"}


class AirError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class air_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "batch", "max_vis_len", "max_nonvis_len",
        "max_window", "max_decode_steps", "dtype", "budget_mode", "min_keep")] + [
        ("alpha", C.c_double), ("retention", C.c_double), ("window_kind", C.c_int32), ("device_steps", C.c_int32),
        ("cache_in_place", C.c_int32), ("causal_text", C.c_int32)]


class air_seq(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("seq_len", "vis_start", "vis_len", "win_start", "win_len")]


class air_layer(C.Structure):
    _fields_ = [("q_text", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p)]


class air_tuning(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("decode_splits", "decode_waves", "decode_tiles", "score_block_mb",
                                         "score_rows_kernel", "select_threads", "select_direct_max", "gather_wgs",
                                         "decode_order", "decode_halves", "budget_in_score")]


class air_strides(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("q_b", "q_h", "q_t", "kv_b", "kv_h", "kv_t")]


class air_rope_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "dtype", "batch", "n_tokens", "layout", "n_axes")] + [
        ("axis_pairs", C.c_int32 * 3), ("norm_eps", C.c_float), ("scale", C.c_float)]


class air_rope_tensor(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("weight", C.c_void_p)] + [
        (n, C.c_int64) for n in ("src_b", "src_h", "src_t", "dst_b", "dst_h", "dst_t")]


class air_prompt_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "dtype")] + [("scale", C.c_float)] + [
        (n, C.c_int64) for n in ("q_h", "q_t", "k_h", "k_t", "v_h", "v_t", "out_h", "out_t")]


class air_prompt_seq(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("q_off", "k_off", "v_off", "out_off")] + [("q_len", C.c_int32), ("kv_len", C.c_int32)]


class air_quant_cache(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "n_kv_heads", "capacity", "head_dim", "group", "dtype")] + [
        (n, C.c_void_p) for n in ("k_codes", "v_codes", "k_scales", "v_scales")]


class air_quant_rows(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p)] + [(n, C.c_int64) for n in ("k_b", "k_h", "k_t", "v_b", "v_h", "v_t")] + [
        ("n_tokens", C.c_int32)] + [(n, C.c_void_p) for n in ("lens", "counts", "positions", "first_positions", "weights")]


class air_quant_query(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_tokens", "causal", "max_len")] + [("scale", C.c_float), ("q", C.c_void_p), ("out", C.c_void_p)] + [
        (n, C.c_int64) for n in ("q_b", "q_h", "q_t", "out_b", "out_h", "out_t")] + [(n, C.c_void_p) for n in ("lens", "counts", "weights")]


AIR_MAX_PLANES = 8


class air_evict_plane(C.Structure):
    _fields_ = [("rows", C.c_void_p), ("b", C.c_int64), ("h", C.c_int64), ("t", C.c_int64), ("row_bytes", C.c_int32)]


class air_evict_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "n_heads", "capacity", "keep", "limit", "first", "recent", "n_planes")] + [
        ("planes", air_evict_plane * AIR_MAX_PLANES)]


EXPORTS = (
    "air_version", "air_workspace_bytes", "air_create", "air_destroy", "air_reset", "air_set_tuning", "air_score",
    "air_budget", "air_select_compact", "air_decode_attn", "air_decode_attn_static", "air_get_scores", "air_get_elite", "air_get_stats",
    "air_get_budgets", "air_set_budgets", "air_get_indices", "air_set_indices", "air_get_lengths", "air_get_cache",
    "air_last_error", "air_rope", "air_rope_frequencies", "air_prompt_workspace_bytes", "air_prompt_attn", "air_prompt_plan",
    "air_quant_append", "air_quant_read", "air_quant_workspace_bytes", "air_quant_attn", "air_evict_workspace_bytes", "air_evict",
)

_lib = None


def load_library(path: Optional[str] = None):
    """Load libaircache.so (built in-tree by paper_2503_23956_amd.build).  Raises if it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise FileNotFoundError(
            f"{p} not found: build it with `python -m paper_2503_23956_amd.build` (there is no CPU fallback)")
    # PyTorch ships its own HIP runtime (soname libamdhip64.so.7).  Import it first so that this
    # library binds to the same runtime instance that owns the tensors and streams it is handed.
    import torch  # noqa: F401

    lib = C.CDLL(p)
    vp, i32 = C.c_void_p, C.c_int32
    lib.air_version.restype = C.c_char_p
    lib.air_workspace_bytes.restype = C.c_size_t
    lib.air_workspace_bytes.argtypes = [C.POINTER(air_config)]
    lib.air_create.argtypes = [C.POINTER(air_config), vp, C.c_size_t, C.POINTER(vp)]
    lib.air_destroy.argtypes = [vp]
    lib.air_reset.argtypes = [vp]
    lib.air_score.argtypes = [vp, vp, i32, i32, C.POINTER(air_layer), C.POINTER(air_strides), C.POINTER(air_seq)]
    lib.air_budget.argtypes = [vp, vp]
    lib.air_select_compact.argtypes = [vp, vp, i32, i32, C.POINTER(air_layer), C.POINTER(air_strides)]
    lib.air_decode_attn.argtypes = [vp, vp, i32, i32, vp, vp, vp, vp]
    lib.air_decode_attn_static.argtypes = [vp, vp, i32, i32, vp, vp, vp, vp]
    lib.air_set_tuning.argtypes = [vp, C.POINTER(air_tuning)]
    lib.air_get_scores.argtypes = [vp, i32, vp]
    lib.air_get_elite.argtypes = [vp, i32, vp, vp]
    lib.air_get_stats.argtypes = [vp, vp, vp]
    lib.air_get_budgets.argtypes = [vp, vp]
    lib.air_set_budgets.argtypes = [vp, vp]
    lib.air_set_indices.argtypes = [vp, C.c_int32, vp]
    lib.air_get_indices.argtypes = [vp, i32, vp]
    lib.air_get_lengths.argtypes = [vp, vp]
    lib.air_get_cache.argtypes = [vp, i32, i32, i32, vp, vp, i32]
    lib.air_last_error.argtypes = [vp]
    lib.air_last_error.restype = C.c_char_p
    dbl = C.c_double
    lib.air_rope.argtypes = [vp, C.POINTER(air_rope_config)] + [C.POINTER(air_rope_tensor)] * 3 + [vp, vp]
    lib.air_rope_frequencies.argtypes = [i32, dbl, i32, dbl, i32, dbl, dbl, vp, C.POINTER(C.c_float)]
    lib.air_prompt_workspace_bytes.argtypes = [C.POINTER(air_prompt_config), C.POINTER(air_prompt_seq), i32]
    lib.air_prompt_workspace_bytes.restype = C.c_size_t
    lib.air_prompt_plan.argtypes = [C.POINTER(air_prompt_config), C.POINTER(air_prompt_seq), i32, C.POINTER(i32), C.POINTER(i32)]
    lib.air_prompt_attn.argtypes = [vp, C.POINTER(air_prompt_config), C.POINTER(air_prompt_seq), i32, vp, vp, vp, vp, vp, C.c_size_t]
    lib.air_quant_append.argtypes = [vp, C.POINTER(air_quant_cache), C.POINTER(air_quant_rows)]
    lib.air_quant_read.argtypes = [vp, C.POINTER(air_quant_cache), C.POINTER(air_quant_rows)]
    lib.air_quant_workspace_bytes.argtypes = [C.POINTER(air_quant_cache), C.POINTER(air_quant_query)]
    lib.air_quant_workspace_bytes.restype = C.c_size_t
    lib.air_quant_attn.argtypes = [vp, C.POINTER(air_quant_cache), C.POINTER(air_quant_query), C.POINTER(air_quant_rows), vp, C.c_size_t]
    lib.air_evict_workspace_bytes.argtypes = [C.POINTER(air_evict_config)]
    lib.air_evict_workspace_bytes.restype = C.c_size_t
    lib.air_evict.argtypes = [vp, C.POINTER(air_evict_config), vp, vp, vp, vp, vp, C.c_size_t]
    for name in EXPORTS:
        if name not in ("air_version", "air_workspace_bytes", "air_prompt_workspace_bytes", "air_quant_workspace_bytes",
                        "air_evict_workspace_bytes", "air_last_error"):
            getattr(lib, name).restype = C.c_int
    if path is None:
        _lib = lib
    return lib


def make_config(*, n_layers, n_q_heads, n_kv_heads, head_dim, batch, max_vis_len, max_nonvis_len, max_window,
                max_decode_steps, dtype, alpha=0.9, retention=0.1, budget_mode=AIR_BUDGET_STRENGTH_SKEW,
                min_keep=1, window_kind=AIR_WINDOW_TEXT, device_steps=0, cache_in_place=0, causal_text=0) -> air_config:
    return air_config(n_layers, n_q_heads, n_kv_heads, head_dim, batch, max_vis_len, max_nonvis_len, max_window,
                      max_decode_steps, dtype, budget_mode, min_keep, alpha, retention, window_kind, device_steps, cache_in_place,
                      causal_text)


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


class Prepared:
    """Marshalled arguments of a range of layers: air_layer[] / air_strides / air_seq[] plus the tensors they point to."""

    def __init__(self, layers, strides, seqs, n, keepalive):
        self.layers, self.strides, self.seqs, self.n, self._keepalive = layers, strides, seqs, n, keepalive


class AirCache:
    """One context: thin wrapper that keeps the workspace tensor alive and marshals arguments.

    Methods carry the names of the C entry points they call.
    """

    def __init__(self, cfg: air_config, device="cuda:0"):
        import torch

        self.lib = load_library()
        self.cfg = cfg
        self.torch = torch
        self.device = torch.device(device)
        nbytes = self.lib.air_workspace_bytes(C.byref(cfg))
        if nbytes == 0:
            raise AirError(AIR_ERR_SHAPE, "air_workspace_bytes: invalid configuration")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.workspace_bytes = nbytes
        h = C.c_void_p()
        st = self.lib.air_create(C.byref(cfg), self.workspace.data_ptr(), nbytes, C.byref(h))
        if st != AIR_OK:
            raise AirError(st, "air_create failed")
        self.handle = h
        self._seqs = None

    def close(self):
        if getattr(self, "handle", None):
            self.lib.air_destroy(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    # -- helpers ---------------------------------------------------------------------
    def _check(self, st: int):
        if st != AIR_OK:
            raise AirError(st, self.lib.air_last_error(self.handle).decode())

    def _stream(self) -> int:
        return int(self.torch.cuda.current_stream(self.device).cuda_stream)

    @staticmethod
    def _layers(q_text: Optional[Sequence], k: Sequence, v: Sequence):
        n = len(k)
        arr = (air_layer * n)()
        for i in range(n):
            arr[i].q_text = _ptr(q_text[i]) if q_text is not None else 0
            arr[i].k = _ptr(k[i])
            arr[i].v = _ptr(v[i])
        return arr

    @staticmethod
    def strides_of(q_text, k) -> air_strides:
        """Element strides of [B][H][T][d]-indexed tensors (any memory order with contiguous d)."""
        qs = q_text.stride() if q_text is not None else (0, 0, 0, 1)
        ks = k.stride()
        assert ks[3] == 1 and qs[3] == 1
        return air_strides(qs[0], qs[1], qs[2], ks[0], ks[1], ks[2])

    @staticmethod
    def seq_array(seqs) -> "C.Array":
        arr = (air_seq * len(seqs))()
        for i, s in enumerate(seqs):
            arr[i] = air_seq(s.seq_len, s.vis_start, s.vis_len, s.win_start, s.win_len)
        return arr

    # -- the four stages -------------------------------------------------------------
    def prepare(self, q_text: Optional[Sequence], k: Sequence, v: Sequence, seqs=None) -> "Prepared":
        """Marshal a set of layers once (descriptor arrays, strides, segments) for repeated stage calls."""
        return Prepared(self._layers(q_text, k, v), self.strides_of(q_text[0] if q_text is not None else None, k[0]),
                        self.seq_array(seqs) if seqs is not None else None, len(k), (q_text, k, v))

    def air_score(self, l0: int, l1: int, q_text=None, k=None, v=None, seqs=None, strides=None, prepared=None, stream=None):
        """prepared: result of prepare() for exactly the layers [l0, l1) (skips the per-call marshalling).
        stream (here and in the other stage calls): a raw HIP stream handle taken beforehand; default: torch's current stream."""
        p = prepared or self.prepare(q_text, k, v, seqs)
        st = strides or p.strides
        assert p.n == l1 - l0 and p.seqs is not None
        self._check(self.lib.air_score(self.handle, self._stream() if stream is None else stream, l0, l1, p.layers, C.byref(st),
                                       p.seqs))

    def air_budget(self, stream=None):
        self._check(self.lib.air_budget(self.handle, self._stream() if stream is None else stream))

    def air_reset(self):
        self._check(self.lib.air_reset(self.handle))

    def air_set_tuning(self, *, decode_splits=0, decode_waves=0, decode_tiles=0, score_block_mb=0, score_rows_kernel=0,
                       select_threads=0, select_direct_max=-1, gather_wgs=0, decode_order=0, decode_halves=0, budget_in_score=0):
        tn = air_tuning(decode_splits, decode_waves, decode_tiles, score_block_mb, score_rows_kernel, select_threads,
                        select_direct_max, gather_wgs, decode_order, decode_halves, budget_in_score)
        self._check(self.lib.air_set_tuning(self.handle, C.byref(tn)))

    def air_select_compact(self, l0: int, l1: int, k=None, v=None, strides=None, prepared=None, stream=None):
        p = prepared or self.prepare(None, k, v)
        st = strides or p.strides
        assert p.n == l1 - l0
        self._check(self.lib.air_select_compact(self.handle, self._stream() if stream is None else stream, l0, l1, p.layers,
                                                C.byref(st)))

    def air_decode_attn(self, l0: int, l1: int, q_new, k_new, v_new, out, stream=None):
        """Tensors, or raw device addresses (ints) when the caller has taken them beforehand."""
        if type(q_new) is not int:
            q_new, k_new, v_new, out = _ptr(q_new), _ptr(k_new), _ptr(v_new), _ptr(out)
        st = self.lib.air_decode_attn(self.handle, self._stream() if stream is None else stream, l0, l1, q_new, k_new, v_new, out)
        if st != AIR_OK:
            self._check(st)

    def air_decode_attn_static(self, l0: int, l1: int, q_new, k_new, v_new, out, stream=None):
        if type(q_new) is not int:
            q_new, k_new, v_new, out = _ptr(q_new), _ptr(k_new), _ptr(v_new), _ptr(out)
        st = self.lib.air_decode_attn_static(self.handle, self._stream() if stream is None else stream, l0, l1, q_new, k_new,
                                             v_new, out)
        if st != AIR_OK:
            self._check(st)

    # -- inspection ------------------------------------------------------------------
    def air_get_scores(self, l: int) -> np.ndarray:
        c = self.cfg
        out = np.empty((c.batch, c.n_kv_heads, c.max_vis_len), dtype=np.float32)
        self._check(self.lib.air_get_scores(self.handle, l, out.ctypes.data))
        return out

    def air_get_elite(self, l: int):
        c = self.cfg
        cnt = np.empty((c.batch, c.n_q_heads), dtype=np.int32)
        idx = np.empty((c.batch, c.n_q_heads, c.max_window), dtype=np.int32)
        self._check(self.lib.air_get_elite(self.handle, l, cnt.ctypes.data, idx.ctypes.data))
        return cnt, idx

    def air_get_stats(self):
        c = self.cfg
        s_t = np.empty((c.batch, c.n_layers), dtype=np.float64)
        s_k = np.empty((c.batch, c.n_layers), dtype=np.float64)
        self._check(self.lib.air_get_stats(self.handle, s_t.ctypes.data, s_k.ctypes.data))
        return s_t, s_k

    def air_get_budgets(self) -> np.ndarray:
        c = self.cfg
        out = np.empty((c.batch, c.n_layers), dtype=np.int32)
        self._check(self.lib.air_get_budgets(self.handle, out.ctypes.data))
        return out

    def air_set_budgets(self, budgets: np.ndarray):
        b = np.ascontiguousarray(budgets, dtype=np.int32)
        assert b.shape == (self.cfg.batch, self.cfg.n_layers)
        self._check(self.lib.air_set_budgets(self.handle, b.ctypes.data))

    def air_get_indices(self, l: int) -> np.ndarray:
        c = self.cfg
        out = np.empty((c.batch, c.n_kv_heads, c.max_vis_len), dtype=np.int32)
        self._check(self.lib.air_get_indices(self.handle, l, out.ctypes.data))
        return out

    def air_set_indices(self, l: int, indices: np.ndarray):
        c = self.cfg
        idx = np.ascontiguousarray(indices, dtype=np.int32)
        assert idx.shape == (c.batch, c.n_kv_heads, c.max_vis_len)
        self._check(self.lib.air_set_indices(self.handle, l, idx.ctypes.data))

    def air_get_lengths(self) -> np.ndarray:
        c = self.cfg
        out = np.empty((c.batch, c.n_layers), dtype=np.int32)
        self._check(self.lib.air_get_lengths(self.handle, out.ctypes.data))
        return out

    def air_get_cache(self, l: int, b: int, h: int, max_rows: int):
        """Rows of the compacted cache of (l, b, h) in the storage dtype (fp32 array or bf16 bit patterns)."""
        c = self.cfg
        dt = np.uint16 if c.dtype == AIR_BF16 else np.float32
        kk = np.zeros((max_rows, c.head_dim), dtype=dt)
        vv = np.zeros((max_rows, c.head_dim), dtype=dt)
        self._check(self.lib.air_get_cache(self.handle, l, b, h, kk.ctypes.data, vv.ctypes.data, max_rows))
        return kk, vv


# -- calls without a context: norm and rotation of queries and keys, attention over a prompt -----------------------------
def _refuse(msg: str):
    raise AirError(AIR_ERR_INVALID_ARG, msg)


def _dtype_of(t) -> int:
    import torch

    if t.dtype not in (torch.bfloat16, torch.float32):
        _refuse(f"tensors must be bfloat16 or float32, not {t.dtype}")
    return AIR_BF16 if t.dtype == torch.bfloat16 else AIR_F32


def _strides4(t):
    """Element strides (batch, head, token) of a tensor indexed [B][H][T][d]; an axis of one entry has none."""
    if t.dim() != 4 or (t.stride(3) != 1 and t.shape[3] > 1):
        _refuse("tensors must be indexed [B][H][T][d] with a contiguous last axis")
    return [t.stride(i) if t.shape[i] > 1 else 0 for i in range(3)]


class PreparedCall:
    """Marshalled arguments of one call without a context plus the tensors they point to; may be called any number of
    times (the tensors' contents may change between calls).  workspace_bytes: what an attention or eviction call needs, None for calls
    that take no workspace."""

    def __init__(self, fn, args, device, keepalive, workspace_bytes=None):
        import torch

        self.name = fn.__name__
        self.torch, self.fn, self.args, self.device, self.workspace_bytes, self._keepalive = torch, fn, args, device, workspace_bytes, keepalive
        self.on_gpu = device.type == "cuda"
        self.index = device.index if device.index is not None else 0
        # the current stream's handle without a stream object around it (0.1 us in place of 3), where torch offers it
        self.raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)

    def __call__(self, stream=None, workspace=None):
        """Enqueues the call with the tensors' device current; stream: a raw HIP stream handle, default torch's current one there.
        workspace (attention, eviction): a contiguous tensor of at least workspace_bytes on the tensors' device; default: one allocated for the call on
        torch's current stream, which is then the only stream the call may go to."""
        more = ()
        if workspace is not None:
            if self.workspace_bytes is None:
                _refuse(f"{self.name}: takes no workspace")
            if workspace.device != self.device or not workspace.is_contiguous():
                _refuse(f"{self.name}: the workspace must be contiguous, on the tensors' device")
            more = (workspace.data_ptr(), workspace.numel() * workspace.element_size())
        if not self.on_gpu:
            _refuse("tensors must be on a GPU")
        cuda = self.torch.cuda
        if cuda.current_device() != self.index:
            with cuda.device(self.index):
                return self(stream, workspace)
        if self.workspace_bytes == 0 and workspace is None:
            more = (0, 0)
        elif self.workspace_bytes and workspace is None:
            if stream is not None:
                _refuse(f"{self.name}: a call on a stream of its own needs its workspace")
            workspace = self.torch.empty(self.workspace_bytes, dtype=self.torch.uint8, device=self.device)
            more = (workspace.data_ptr(), self.workspace_bytes)
        st = self.fn(self.raw_stream(self.index) if stream is None else stream, *self.args, *more)
        if st != AIR_OK:
            raise AirError(st, load_library().air_last_error(None).decode())


def air_rope_frequencies(n_pairs: int, theta: float, scaling=AIR_ROPE_PLAIN, factor=1.0, original_len=0, slow_turns=1.0, fast_turns=32.0):
    """(frequencies as a float64 array [n_pairs], factor of the rotated elements): see include/aircache.h."""
    lib = load_library()
    out, scale = np.empty(max(0, n_pairs), dtype=np.float64), C.c_float(1.0)
    st = lib.air_rope_frequencies(n_pairs, theta, scaling, factor, original_len, slow_turns, fast_turns, out.ctypes.data, C.byref(scale))
    if st != AIR_OK:
        raise AirError(st, lib.air_last_error(None).decode())
    return out, scale.value


def prepare_rope(q=None, k=None, v=None, q_out=None, k_out=None, v_out=None, *, positions=None, freqs=None, axis_pairs=(),
                 layout=AIR_ROPE_HALF, q_weight=None, k_weight=None, eps=1e-6, scale=1.0) -> PreparedCall:
    """Tensors indexed [B][H][T][d], any memory order with contiguous d; an output left out means in place.  axis_pairs: pairs per
    position axis (one to three).  positions: int32 [axes][B][T] ([B][T] with one axis), negative = padding, left as it is;
    freqs: float64 [sum(axis_pairs)]; both contiguous on the tensors' device."""
    import torch

    given = [(x, x if o is None else o, w) for x, o, w in ((q, q_out, q_weight), (k, k_out, k_weight), (v, v_out, None))]
    first = next((x for x, _, _ in given if x is not None), None)
    if first is None:
        _refuse("air_rope: one of q, k, v is needed")
    first_dtype = _dtype_of(first)
    _strides4(first)
    B, T, d = first.shape[0], first.shape[2], first.shape[3]
    n_axes, pairs = max(1, len(axis_pairs)), sum(axis_pairs)
    if len(axis_pairs) > 3:
        _refuse("air_rope: at most three position axes")
    ts = []
    for x, o, w in given:
        if x is None:
            if o is not None or w is not None:
                _refuse("air_rope: an output or a weight without its tensor")
            ts.append(None)
            continue
        if x.dtype != first.dtype or o.dtype != first.dtype or x.shape != o.shape or (x.shape[0], x.shape[2], x.shape[3]) != (B, T, d):
            _refuse("air_rope: tensors must have one type, batch, length and head size, outputs their tensor's shape")
        if w is not None and (w.dtype != first.dtype or tuple(w.shape) != (d,) or not w.is_contiguous()):
            _refuse("air_rope: a weight must be a contiguous [head_dim] of the tensors' type")
        if x.device != first.device or o.device != first.device or (w is not None and w.device != first.device):
            _refuse("air_rope: tensors must be on one device")
        ts.append(air_rope_tensor(_ptr(x), _ptr(o), _ptr(w), *_strides4(x), *_strides4(o)))
    if k is not None and v is not None and k.shape[1] != v.shape[1]:
        _refuse("air_rope: keys and values must have the same heads")
    hkv = k.shape[1] if k is not None else v.shape[1] if v is not None else 0
    hq = q.shape[1] if q is not None else hkv
    if positions is not None:
        if positions.dtype != torch.int32 or not positions.is_contiguous() or positions.device != first.device or \
                tuple(positions.shape) not in ((n_axes, B, T),) + (((B, T),) if n_axes == 1 else ()):
            _refuse("air_rope: positions must be a contiguous int32 [axes][B][T] on the tensors' device")
    if freqs is not None and (freqs.dtype != torch.float64 or not freqs.is_contiguous() or freqs.numel() < pairs or
                              freqs.device != first.device):
        _refuse("air_rope: freqs must be a contiguous float64 [sum(axis_pairs)] on the tensors' device")
    cfg = air_rope_config(hq, hkv or hq, d, first_dtype, B, T, layout, n_axes, (C.c_int32 * 3)(*axis_pairs), eps, scale)
    args = (C.byref(cfg), *(None if t is None else C.byref(t) for t in ts), _ptr(positions), _ptr(freqs))
    return PreparedCall(load_library().air_rope, args, first.device, (given, positions, freqs))


def air_rope(*tensors, prepared: Optional[PreparedCall] = None, stream=None, **kw):
    """prepared: result of prepare_rope (skips the marshalling); else its arguments.  stream: a raw HIP stream handle, default torch's
    current stream on the tensors' device."""
    (prepared or prepare_rope(*tensors, **kw))(stream)


def prepare_prompt_attn(q, k, v, out, spans=None, scale=0.0) -> PreparedCall:
    """q, out [B][Hq][T][d], k, v [B][Hkv][S][d], any memory order with contiguous d.  spans: one (batch row, first query, queries, first
    key, keys) per sequence; default: every batch row over its full length."""
    dt = _dtype_of(q)
    sq, sk, sv, so = (_strides4(t) for t in (q, k, v, out))
    if any(t.dtype != q.dtype or t.device != q.device for t in (k, v, out)):
        _refuse("air_prompt_attn: tensors must have one type and device")
    if k.shape != v.shape or q.shape != out.shape or q.shape[0] != k.shape[0] or q.shape[3] != k.shape[3]:
        _refuse("air_prompt_attn: shapes of q and out, of k and v must agree")
    if spans is None:
        spans = [(b, 0, q.shape[2], 0, k.shape[2]) for b in range(q.shape[0])]
    arr = (air_prompt_seq * max(1, len(spans)))()
    for i, (b, q0, n, k0, m) in enumerate(spans):
        if min(q0, n, k0, m) < 0 or not 0 <= b < q.shape[0] or q0 + n > q.shape[2] or k0 + m > k.shape[2]:
            _refuse("air_prompt_attn: a span lies outside its tensors")
        arr[i] = air_prompt_seq(b * sq[0] + q0 * sq[2], b * sk[0] + k0 * sk[2], b * sv[0] + k0 * sv[2], b * so[0] + q0 * so[2], n, m)
    cfg = air_prompt_config(q.shape[1], k.shape[1], q.shape[3], dt, scale, sq[1], sq[2], sk[1], sk[2], sv[1], sv[2], so[1], so[2])
    args = (C.byref(cfg), arr, len(spans), _ptr(q), _ptr(k), _ptr(v), _ptr(out))
    lib = load_library()
    nbytes = lib.air_prompt_workspace_bytes(C.byref(cfg), arr, len(spans))
    return PreparedCall(lib.air_prompt_attn, args, q.device, (q, k, v, out), nbytes)


def air_prompt_attn(*tensors, prepared: Optional[PreparedCall] = None, workspace=None, stream=None, **kw):
    """prepared: result of prepare_prompt_attn (skips the marshalling); else its arguments.  workspace: a contiguous tensor of at least
    prepared.workspace_bytes on the tensors' device; default: one allocated for the call on torch's current stream, which is then the only
    stream the call may go to.  stream: a raw HIP stream handle, default torch's current stream on the tensors' device."""
    (prepared or prepare_prompt_attn(*tensors, **kw))(stream, workspace)


def air_prompt_plan(prepared: PreparedCall):
    """(rows of a tile, splits over the keys) with which a result of prepare_prompt_attn runs."""
    lib = load_library()
    rows, splits = C.c_int32(), C.c_int32()
    st = lib.air_prompt_plan(*prepared.args[:3], C.byref(rows), C.byref(splits))
    if st != AIR_OK:
        raise AirError(st, lib.air_last_error(None).decode())
    return rows.value, splits.value


# -- a cache that is generated into: 4-bit rows, attention over them, eviction by attention weight ------------------------
class QuantCache:
    """K and V of up to `capacity` slots per (sequence, KV head) in 4 bits; dtype: of the rows that go in, of queries and outputs.  The
    memory (`planes`: codes of K and V, scales of K and V, each [B][H][capacity][...]) is torch's; what it holds is counted by the
    caller, in an int32 tensor [B] on the same device that every call takes as `lens`."""

    def __init__(self, batch, n_kv_heads, capacity, head_dim, dtype=AIR_BF16, group=32, device="cuda:0"):
        import torch

        if head_dim not in (64, 128) or group not in (32, 64) or min(batch, n_kv_heads, capacity) < 1:
            raise AirError(AIR_ERR_SHAPE, "QuantCache: head_dim must be 64 or 128, group 32 or 64, sizes positive")
        self.batch, self.n_kv_heads, self.capacity, self.head_dim, self.dtype, self.group = batch, n_kv_heads, capacity, head_dim, dtype, group
        self.torch_dtype = torch.bfloat16 if dtype == AIR_BF16 else torch.float32
        self.device = torch.device(device)
        shape = (batch, n_kv_heads, capacity)
        codes = [torch.empty((*shape, head_dim // 2), dtype=torch.uint8, device=self.device) for _ in range(2)]
        scales = [torch.empty((*shape, 2 * head_dim // group), dtype=torch.bfloat16, device=self.device) for _ in range(2)]
        self.planes = (*codes, *scales)
        self.device = codes[0].device  # (with its index)
        self.struct = air_quant_cache(batch, n_kv_heads, capacity, head_dim, group, dtype, *(_ptr(p) for p in self.planes))


def _table(who, name, t, dtype, shape, device):
    """Address of an optional contiguous tensor of one type, shape and device."""
    if t is None:
        return 0
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != device:
        _refuse(f"{who}: {name} must be a contiguous {dtype} {list(shape)} on the tensors' device")
    return _ptr(t)


def _cache_tensor(who, name, cache, t, heads):
    """Strides of a tensor [B][heads][T][d] of the cache's type and device."""
    if t.dtype != cache.torch_dtype or t.device != cache.device:
        _refuse(f"{who}: {name} must have the cache's type and device")
    st = _strides4(t)
    if t.shape[0] != cache.batch or t.shape[3] != cache.head_dim or (heads is not None and t.shape[1] != heads):
        _refuse(f"{who}: {name} must be indexed [B][H][T][d] as the cache is")
    return st


def _quant_rows(who, cache, k, v, lens, counts, positions=None, first_positions=None, weights=None):
    import torch

    first = k if k is not None else v
    if first is None:
        _refuse(f"{who}: one of k and v is needed")
    st = [_cache_tensor(who, n, cache, t, cache.n_kv_heads) if t is not None else [0, 0, 0] for n, t in (("k", k), ("v", v))]
    if k is not None and v is not None and k.shape != v.shape:
        _refuse(f"{who}: k and v must have one shape")
    B, cells, dev = (cache.batch,), (cache.batch, cache.n_kv_heads, cache.capacity), cache.device
    return air_quant_rows(_ptr(k), _ptr(v), *st[0], *st[1], first.shape[2], _table(who, "lens", lens, torch.int32, B, dev),
                          _table(who, "counts", counts, torch.int32, B, dev), _table(who, "positions", positions, torch.int32, cells, dev),
                          _table(who, "first_positions", first_positions, torch.int32, B, dev),
                          _table(who, "weights", weights, torch.float32, cells, dev))


def prepare_quant_append(cache: QuantCache, k, v, *, lens=None, counts=None, positions=None, first_positions=None, weights=None) -> PreparedCall:
    """k, v [B][Hkv][T][d], any memory order with contiguous d.  lens, counts, first_positions: int32 [B]; positions: int32, weights:
    float32 [B][Hkv][capacity]; all on the cache's device.  Row t of sequence b goes to slot lens[b] + t, for t < counts[b]."""
    if k is None or v is None:
        _refuse("air_quant_append: k and v are needed")
    rows = _quant_rows("air_quant_append", cache, k, v, lens, counts, positions, first_positions, weights)
    return PreparedCall(load_library().air_quant_append, (C.byref(cache.struct), C.byref(rows)), cache.device,
                        (cache, k, v, lens, counts, positions, first_positions, weights))


def air_quant_append(*args, prepared: Optional[PreparedCall] = None, stream=None, **kw):
    """prepared: result of prepare_quant_append (skips the marshalling); else its arguments.  stream: a raw HIP stream handle, default
    torch's current stream on the cache's device."""
    (prepared or prepare_quant_append(*args, **kw))(stream)


def prepare_quant_read(cache: QuantCache, k=None, v=None, *, starts=None, counts=None) -> PreparedCall:
    """What slots starts[b] .. starts[b] + counts[b] - 1 stand for, into k and v [B][Hkv][T][d]; either may be left out."""
    rows = _quant_rows("air_quant_read", cache, k, v, starts, counts)
    return PreparedCall(load_library().air_quant_read, (C.byref(cache.struct), C.byref(rows)), cache.device, (cache, k, v, starts, counts))


def air_quant_read(*args, prepared: Optional[PreparedCall] = None, stream=None, **kw):
    """prepared: result of prepare_quant_read; else its arguments.  stream as in air_quant_append."""
    (prepared or prepare_quant_read(*args, **kw))(stream)


def prepare_quant_attn(cache: QuantCache, q, out, *, lens, counts=None, k=None, v=None, causal=True, scale=0.0, weights=None, positions=None,
                       first_positions=None, max_len=0) -> PreparedCall:
    """q, out [B][Hq][T][d] (out may be None: weights only); k, v [B][Hkv][T][d]: the queries' own rows, which go into the cache
    first (with positions, where given).  weights float32 [B][Hkv][capacity] grow by what every slot is attended to.  max_len: most slots a sequence
    will hold when the call runs (the launch's shape goes by it; 0: capacity)."""
    import torch

    who, B = "air_quant_attn", (cache.batch,)
    sq = _cache_tensor(who, "q", cache, q, None)
    so = _cache_tensor(who, "out", cache, out, q.shape[1]) if out is not None else [0, 0, 0]
    if out is not None and out.shape != q.shape:
        _refuse("air_quant_attn: shapes of q and out must agree")
    if lens is None:
        _refuse("air_quant_attn: lens are needed")
    if (k is None) != (v is None):
        _refuse("air_quant_attn: k and v go together")
    rows = None
    if k is not None:
        rows = _quant_rows(who, cache, k, v, lens, counts, positions, first_positions, weights)
    elif positions is not None or first_positions is not None:
        _refuse("air_quant_attn: positions without rows to append")
    query = air_quant_query(q.shape[1], q.shape[2], int(causal), max_len, scale, _ptr(q), _ptr(out), *sq, *so,
                            _table(who, "lens", lens, torch.int32, B, cache.device), _table(who, "counts", counts, torch.int32, B, cache.device),
                            _table(who, "weights", weights, torch.float32, (*B, cache.n_kv_heads, cache.capacity), cache.device))
    lib = load_library()
    nbytes = lib.air_quant_workspace_bytes(C.byref(cache.struct), C.byref(query))
    return PreparedCall(lib.air_quant_attn, (C.byref(cache.struct), C.byref(query), C.byref(rows) if rows is not None else None), cache.device,
                        (cache, q, out, lens, counts, k, v, weights, positions, first_positions), nbytes)


def air_quant_attn(*args, prepared: Optional[PreparedCall] = None, workspace=None, stream=None, **kw):
    """prepared: result of prepare_quant_attn; else its arguments.  workspace and stream as in air_prompt_attn."""
    (prepared or prepare_quant_attn(*args, **kw))(stream, workspace)


def prepare_evict(planes, weights, *, lens, lens_out, keep, limit=None, positions=None, first=0, recent=0) -> PreparedCall:
    """planes: tensors [B][H][capacity][n] whose rows belong to the slots (K and V as they are, or QuantCache.planes), any strides with a
    contiguous last axis.  weights float32, positions int32 [B][H][capacity]; lens, lens_out int32 [B].  limit: default keep."""
    import torch

    who = "air_evict"
    if weights is None or lens is None or lens_out is None:
        _refuse("air_evict: weights, lens and lens_out are needed")
    if weights.dim() != 3 or len(planes) > AIR_MAX_PLANES:
        _refuse(f"air_evict: weights must be [B][H][capacity], planes at most {AIR_MAX_PLANES}")
    B, H, cap = weights.shape
    arr = (air_evict_plane * AIR_MAX_PLANES)()
    for i, p in enumerate(planes):
        if p.device != weights.device or tuple(p.shape[:3]) != (B, H, cap):
            _refuse("air_evict: planes must be [B][H][capacity][n] on the weights' device")
        arr[i] = air_evict_plane(_ptr(p), *(s * p.element_size() for s in _strides4(p)), p.shape[3] * p.element_size())
    cfg = air_evict_config(B, H, cap, keep, keep if limit is None else limit, first, recent, len(planes), arr)
    args = (C.byref(cfg), _table(who, "weights", weights, torch.float32, (B, H, cap), weights.device),
            _table(who, "positions", positions, torch.int32, (B, H, cap), weights.device),
            _table(who, "lens", lens, torch.int32, (B,), weights.device), _table(who, "lens_out", lens_out, torch.int32, (B,), weights.device))
    lib = load_library()
    return PreparedCall(lib.air_evict, args, weights.device, (planes, weights, lens, lens_out, positions),
                        lib.air_evict_workspace_bytes(C.byref(cfg)))


def air_evict(*args, prepared: Optional[PreparedCall] = None, workspace=None, stream=None, **kw):
    """prepared: result of prepare_evict; else its arguments.  workspace and stream as in air_prompt_attn."""
    (prepared or prepare_evict(*args, **kw))(stream, workspace)
