"""Thin binding of libxsv.so (include/xsv.h): argument marshalling only.

Every step of the path runs inside the HIP library; this module turns torch tensors into the
pointer/stride structs of the C ABI and numpy arrays into host buffers.  There is no fallback: if
the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libxsv.so")

XSV_OK = 0
XSV_ERR_ARG, XSV_ERR_UNSUPPORTED, XSV_ERR_OOM, XSV_ERR_STATE, XSV_ERR_HIP = -1, -2, -3, -4, -5


class XsvError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {strerror(code)} ({code})")


class xsv_config(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
        ("tokens_per_frame", C.c_int32), ("n_special", C.c_int32), ("budget", C.c_int32),
        ("kv_bits", C.c_int32), ("group_size", C.c_int32), ("pool_size", C.c_int32), ("score_mode", C.c_int32),
        ("softmax_scale", C.c_float), ("max_frames", C.c_int32), ("value_mode", C.c_int32),
    ]


class xsv_tensor(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("stride_head", C.c_int64), ("stride_token", C.c_int64)]


NORMS = {"none": 0, "rms": 1, "layer": 2}


class xsv_rotate_config(C.Structure):
    _fields_ = [
        ("n", C.c_int32), ("heads_q", C.c_int32), ("heads_k", C.c_int32), ("norm", C.c_int32), ("axes", C.c_int32),
        ("interleaved", C.c_int32), ("eps", C.c_float), ("base", C.c_double), ("positions", C.c_void_p),
        ("q_weight", C.c_void_p), ("q_bias", C.c_void_p), ("k_weight", C.c_void_p), ("k_bias", C.c_void_p),
    ]


class xsv_seq_config(C.Structure):
    _fields_ = [
        ("heads", C.c_int32), ("kv_heads", C.c_int32), ("sequences", C.c_int32), ("rows_q", C.c_int32), ("rows_k", C.c_int32),
        ("longest_q", C.c_int32), ("longest_k", C.c_int32), ("q_begin", C.c_void_p), ("k_begin", C.c_void_p), ("causal", C.c_int32),
        ("softmax_scale", C.c_float),
    ]


# every symbol include/xsv.h declares
EXPORTS = (
    "xsv_create", "xsv_destroy", "xsv_reset", "xsv_dequant_attend", "xsv_frame_attend", "xsv_score_prune", "xsv_quantize",
    "xsv_step", "xsv_step_all_layers", "xsv_set_overlap", "xsv_join", "xsv_cache_len", "xsv_cache_export",
    "xsv_cache_import", "xsv_last_selection", "xsv_quantize_k", "xsv_quantize_v", "xsv_score", "xsv_score_noalloc",
    "xsv_topk_keep", "xsv_strerror", "xsv_norm_rotate", "xsv_norm_rotate_grad", "xsv_norm_rotate_grad_workspace",
    "xsv_seq_attend", "xsv_seq_attend_workspace", "xsv_seq_attend_grad", "xsv_seq_attend_grad_workspace", "xsv_query_attend",
)
# every symbol include/xsv_tune.h declares (launch tuning and measurement aids)
TUNE_EXPORTS = (
    "xsv_set_attend_splits", "xsv_set_attend_variant", "xsv_set_side_cus", "xsv_set_short_range", "xsv_set_frame_tile_cost",
    "xsv_set_pool_polls", "xsv_set_merge_looks",
    "xsv_last_attend_workgroups", "xsv_last_attend_merge", "xsv_settled_blocks", "xsv_set_attend_timing", "xsv_attend_times", "xsv_chain_times", "xsv_measure_peaks",
    "xsv_key_ranges", "xsv_line_partition", "xsv_step_plan",
)

_lib = None


def lib():
    """The loaded library; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2602_21780_amd/build.py "
                               "(or __graft_entry__.build()); there is no fallback path")
        L = C.CDLL(LIB_PATH)
        vp, i32 = C.c_void_p, C.c_int
        T = xsv_tensor
        L.xsv_create.argtypes = [C.POINTER(xsv_config), vp, C.POINTER(vp)]
        L.xsv_destroy.argtypes = [vp]
        L.xsv_reset.argtypes = [vp]
        L.xsv_join.argtypes = [vp]
        L.xsv_dequant_attend.argtypes = [vp, i32, T, T, T, vp]
        L.xsv_frame_attend.argtypes = [vp, T, T, T, vp]
        L.xsv_query_attend.argtypes = [vp, i32, T, i32, vp, vp]
        L.xsv_score_prune.argtypes = [vp, i32, T]
        L.xsv_quantize.argtypes = [vp, i32, T, T]
        L.xsv_step.argtypes = [vp, i32, T, T, T, vp]
        L.xsv_step_all_layers.argtypes = [vp, C.POINTER(T), C.POINTER(T), C.POINTER(T), C.POINTER(vp)]
        L.xsv_set_attend_splits.argtypes = [vp, i32, i32]
        L.xsv_set_attend_variant.argtypes = [vp, i32]
        L.xsv_set_overlap.argtypes = [vp, i32]
        L.xsv_set_side_cus.argtypes = [vp, i32]
        L.xsv_set_short_range.argtypes = [vp, i32]
        L.xsv_set_pool_polls.argtypes = [vp, i32]
        L.xsv_set_merge_looks.argtypes = [vp, i32]
        L.xsv_set_frame_tile_cost.argtypes = [vp, i32]
        L.xsv_last_attend_workgroups.argtypes = [vp, C.POINTER(C.c_int32)]
        L.xsv_last_attend_merge.argtypes = [vp, C.POINTER(C.c_int32)]
        L.xsv_set_attend_timing.argtypes = [vp, i32]
        L.xsv_settled_blocks.argtypes = [vp, i32, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.xsv_chain_times.argtypes = [vp, C.POINTER(C.c_int32), C.POINTER(C.c_float), C.POINTER(C.c_float)]
        L.xsv_attend_times.argtypes = [vp, C.POINTER(C.c_int32), C.POINTER(C.c_float), C.POINTER(C.c_float), C.POINTER(C.c_float)]
        L.xsv_cache_len.argtypes = [vp, i32, C.POINTER(C.c_int32)]
        L.xsv_cache_export.argtypes = [vp, i32] + [vp] * 10
        L.xsv_cache_import.argtypes = [vp, i32, C.c_int32, C.c_int32] + [vp] * 10
        L.xsv_last_selection.argtypes = [vp, i32, C.POINTER(C.c_int32), vp, C.POINTER(C.c_int32), vp]
        L.xsv_quantize_k.argtypes = [vp, vp, i32, i32, i32, i32, i32, vp, vp, vp]
        L.xsv_quantize_v.argtypes = [vp, vp, i32, i32, i32, i32, i32, vp, vp, vp]
        L.xsv_score.argtypes = [vp, T, vp, i32, i32, i32, i32, i32, i32, vp]
        L.xsv_score_noalloc.argtypes = [vp, T, vp, i32, i32, i32, i32, i32, i32, vp]
        L.xsv_topk_keep.argtypes = [vp, vp, i32, i32, i32, i32, vp]
        R = C.POINTER(xsv_rotate_config)
        L.xsv_norm_rotate.argtypes = [vp, R, T, T, T, T]
        L.xsv_norm_rotate_grad.argtypes = [vp, R, T, T, T, T, T, T, vp, vp, C.c_int64]
        L.xsv_norm_rotate_grad_workspace.argtypes = [R, C.POINTER(C.c_int64)]
        S = C.POINTER(xsv_seq_config)
        L.xsv_seq_attend.argtypes = [vp, S, T, T, T, T, vp, vp, C.c_int64]
        L.xsv_seq_attend_workspace.argtypes = [S, C.POINTER(C.c_int64)]
        L.xsv_seq_attend_grad.argtypes = [vp, S, T, T, T, T, vp, T, T, T, T, vp, C.c_int64]
        L.xsv_seq_attend_grad_workspace.argtypes = [S, C.POINTER(C.c_int64)]
        L.xsv_measure_peaks.argtypes = [vp, C.POINTER(C.c_float), C.POINTER(C.c_float)]
        L.xsv_strerror.argtypes = [i32]
        L.xsv_strerror.restype = C.c_char_p
        for name in EXPORTS + TUNE_EXPORTS:
            if name != "xsv_strerror":
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().xsv_strerror(code).decode()


def _check(code: int, what: str):
    if code != XSV_OK:
        raise XsvError(code, what)


def as_tensor(t: torch.Tensor) -> xsv_tensor:
    """bf16 device tensor [H][n][64], channel-contiguous → xsv_tensor (strides in elements)."""
    if t.dtype != torch.bfloat16 or t.dim() != 3 or t.stride(2) != 1 or not t.is_cuda:
        raise ValueError("expected a bf16 device tensor [H][n][d] with contiguous channels")
    return xsv_tensor(t.data_ptr(), t.stride(0), t.stride(1))


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _np_ptr(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


@dataclass
class CacheDump:
    T: int
    k_codes: np.ndarray | None
    k_scale: np.ndarray | None
    k_zero: np.ndarray | None
    v_codes: np.ndarray | None
    v_scale: np.ndarray | None
    v_zero: np.ndarray | None
    k_bf16: np.ndarray
    v_bf16: np.ndarray
    token_frame: np.ndarray
    token_index: np.ndarray


class Context:
    """Owner of an xsv_ctx.  Method names follow the C entry points.  Its calls run on `stream` (None: the one that is current when it is made),
    whatever the current one is then, and outputs that they make belong to that stream."""

    def __init__(self, n_layers, n_heads, head_dim, tokens_per_frame, n_special, budget, kv_bits, group_size,
                 pool_size=16, softmax_scale=0.0, max_frames=0, stream=None, score_mode=0, value_mode=0):
        self.cfg = xsv_config(n_layers, n_heads, head_dim, tokens_per_frame, n_special, budget, kv_bits, group_size,
                              pool_size, score_mode, softmax_scale, max_frames, value_mode)
        self._h = C.c_void_p()
        # (the library works on this stream whatever the current one is later, and so what a call allocates belongs to it)
        self._stream = torch.cuda.current_stream() if stream is None else stream
        _check(lib().xsv_create(C.byref(self.cfg), _stream_ptr(self._stream), C.byref(self._h)), "xsv_create")

    @classmethod
    def from_spec(cls, spec, stream=None, **over):
        kw = dict(n_layers=spec.n_layers, n_heads=spec.n_heads, head_dim=spec.head_dim,
                  tokens_per_frame=spec.tokens_per_frame, n_special=spec.n_special, budget=spec.budget,
                  kv_bits=spec.kv_bits, group_size=spec.group_size, pool_size=spec.pool_size,
                  max_frames=spec.frames)
        kw.update(over)
        return cls(stream=stream, **kw)

    def destroy(self):
        if self._h:
            lib().xsv_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def reset(self):
        _check(lib().xsv_reset(self._h), "xsv_reset")

    def set_attend_splits(self, per_layer_calls=0, batched_calls=0):
        _check(lib().xsv_set_attend_splits(self._h, per_layer_calls, batched_calls), "xsv_set_attend_splits")

    def set_attend_variant(self, variant):
        _check(lib().xsv_set_attend_variant(self._h, variant), "xsv_set_attend_variant")

    def set_overlap(self, mode):
        _check(lib().xsv_set_overlap(self._h, int(mode)), "xsv_set_overlap")

    def set_attend_timing(self, enabled):
        _check(lib().xsv_set_attend_timing(self._h, int(enabled)), "xsv_set_attend_timing")

    def attend_times(self):
        """(launches, attention-kernel span ms, merge-kernel span ms, span of an empty event pair ms), averages
        since the last call."""
        n, a, m, e = C.c_int32(), C.c_float(), C.c_float(), C.c_float()
        _check(lib().xsv_attend_times(self._h, C.byref(n), C.byref(a), C.byref(m), C.byref(e)), "xsv_attend_times")
        return n.value, a.value, m.value, e.value

    def chain_times(self):
        """(steps, score + select span ms, re-quantize span ms), averages since the last call."""
        n, a, b = C.c_int32(), C.c_float(), C.c_float()
        _check(lib().xsv_chain_times(self._h, C.byref(n), C.byref(a), C.byref(b)), "xsv_chain_times")
        return n.value, a.value, b.value

    def last_attend_workgroups(self) -> int:
        w = C.c_int32()
        _check(lib().xsv_last_attend_workgroups(self._h, C.byref(w)), "xsv_last_attend_workgroups")
        return w.value

    def last_attend_merges_inside(self) -> bool:
        inside = C.c_int32()
        _check(lib().xsv_last_attend_merge(self._h, C.byref(inside)), "xsv_last_attend_merge")
        return bool(inside.value)

    def settled_blocks(self, layer=0):
        """((head, block) pairs the re-quantization no longer touches, (head, block) pairs in the layer's cache)."""
        a, b = C.c_int32(), C.c_int32()
        _check(lib().xsv_settled_blocks(self._h, layer, C.byref(a), C.byref(b)), "xsv_settled_blocks")
        return a.value, b.value

    def join(self):
        _check(lib().xsv_join(self._h), "xsv_join")

    def set_short_range(self, percent):
        _check(lib().xsv_set_short_range(self._h, int(percent)), "xsv_set_short_range")

    def set_frame_tile_cost(self, percent):
        _check(lib().xsv_set_frame_tile_cost(self._h, int(percent)), "xsv_set_frame_tile_cost")

    def set_side_cus(self, compute_units):
        _check(lib().xsv_set_side_cus(self._h, int(compute_units)), "xsv_set_side_cus")

    def set_pool_polls(self, polls):
        _check(lib().xsv_set_pool_polls(self._h, int(polls)), "xsv_set_pool_polls")

    def set_merge_looks(self, looks):
        _check(lib().xsv_set_merge_looks(self._h, int(looks)), "xsv_set_merge_looks")

    def _out(self, q, out):
        if out is None:
            with _on(q.device, self._stream):
                out = torch.empty((self.cfg.n_heads, self.cfg.tokens_per_frame, self.cfg.head_dim), dtype=torch.bfloat16,
                                  device=q.device)
        return out

    def dequant_attend(self, layer, q, k_new, v_new, out=None):
        out = self._out(q, out)
        _check(lib().xsv_dequant_attend(self._h, layer, as_tensor(q), as_tensor(k_new), as_tensor(v_new), out.data_ptr()),
               "xsv_dequant_attend")
        return out

    def frame_attend(self, q, k, v, out=None):
        out = self._out(q, out)
        _check(lib().xsv_frame_attend(self._h, as_tensor(q), as_tensor(k), as_tensor(v), out.data_ptr()), "xsv_frame_attend")
        return out

    def query_attend(self, layer, q, out=None, lse=None):
        """xsv_query_attend: q [H][rows][64] over the layer's cache, on the context's stream.  Returns (out, lse)."""
        H, d = self.cfg.n_heads, self.cfg.head_dim
        tq = _tensor(q, "q", shape=(H, q.shape[1], d) if isinstance(q, torch.Tensor) and q.dim() == 3 else None)
        rows, dev = q.shape[1], q.device
        with _on(dev, self._stream):
            out = torch.empty((H, rows, d), dtype=torch.bfloat16, device=dev) if out is None else _plain(out, "out", torch.bfloat16, (H, rows, d), dev)
            lse = torch.empty((H, rows), dtype=torch.float32, device=dev) if lse is None else _plain(lse, "lse", torch.float32, (H, rows), dev)
            if rows:
                _check(lib().xsv_query_attend(self._h, layer, tq, rows, out.data_ptr(), lse.data_ptr()), "xsv_query_attend")
        return out, lse

    def score_prune(self, layer, q):
        _check(lib().xsv_score_prune(self._h, layer, as_tensor(q)), "xsv_score_prune")

    def quantize(self, layer, k_new, v_new):
        _check(lib().xsv_quantize(self._h, layer, as_tensor(k_new), as_tensor(v_new)), "xsv_quantize")

    def step(self, layer, q, k_new, v_new, out=None):
        out = self._out(q, out)
        _check(lib().xsv_step(self._h, layer, as_tensor(q), as_tensor(k_new), as_tensor(v_new), out.data_ptr()), "xsv_step")
        return out

    def pack_step(self, q, k_new, v_new, out):
        """Marshal one layer's tensors once, for repeated step_packed calls (the tensors must stay alive)."""
        return as_tensor(q), as_tensor(k_new), as_tensor(v_new), out.data_ptr()

    def step_packed(self, layer, packed):
        _check(lib().xsv_step(self._h, layer, *packed), "xsv_step")

    def pack_layers(self, q, k_new, v_new, out):
        """Marshal per-layer tensors ([L][H][n][d] or lists) once, for repeated step_all_layers calls."""
        L = self.cfg.n_layers
        arr = lambda ts: (xsv_tensor * L)(*[as_tensor(ts[l]) for l in range(L)])
        outs = (C.c_void_p * L)(*[out[l].data_ptr() for l in range(L)])
        return arr(q), arr(k_new), arr(v_new), outs

    def step_all_layers(self, q=None, k_new=None, v_new=None, out=None, packed=None):
        if packed is None:
            if out is None:
                with _on(q[0].device, self._stream):
                    out = torch.empty((self.cfg.n_layers, self.cfg.n_heads, self.cfg.tokens_per_frame, self.cfg.head_dim),
                                      dtype=torch.bfloat16, device=q[0].device)
            packed = self.pack_layers(q, k_new, v_new, out)
        _check(lib().xsv_step_all_layers(self._h, *packed), "xsv_step_all_layers")
        return out

    def cache_len(self, layer=0) -> int:
        T = C.c_int32()
        _check(lib().xsv_cache_len(self._h, layer, C.byref(T)), "xsv_cache_len")
        return T.value

    def cache_export(self, layer=0) -> CacheDump:
        H, d, G = self.cfg.n_heads, self.cfg.head_dim, self.cfg.group_size
        T = self.cache_len(layer)
        quant = self.cfg.kv_bits != 16
        ng = (T + G - 1) // G if quant else 0
        kc = np.zeros((H, T, d), np.uint8) if quant else None
        vc = np.zeros((H, T, d), np.uint8) if quant else None
        ks = np.zeros((H, ng, d), np.float32) if quant else None
        kz = np.zeros((H, ng, d), np.float32) if quant else None
        vs = np.zeros((H, T, d // G), np.float32) if quant else None
        vz = np.zeros((H, T, d // G), np.float32) if quant else None
        kb = np.zeros((H, T, d), np.uint16)
        vb = np.zeros((H, T, d), np.uint16)
        lead = (H,) if self.cfg.score_mode == 1 else ()     # one retained set per head, or one per layer
        tf = np.zeros(lead + (T,), np.int32)
        ti = np.zeros(lead + (T,), np.int32)
        _check(lib().xsv_cache_export(self._h, layer, _np_ptr(kc), _np_ptr(ks), _np_ptr(kz), _np_ptr(vc), _np_ptr(vs),
                                      _np_ptr(vz), _np_ptr(kb), _np_ptr(vb), _np_ptr(tf), _np_ptr(ti)), "xsv_cache_export")
        return CacheDump(T, kc, ks, kz, vc, vs, vz, kb, vb, tf, ti)

    def cache_import(self, layer, dump, frames_seen):
        """`dump`: any object with the fields of CacheDump (e.g. the oracle's export)."""
        c = lambda a, dt: None if a is None else np.ascontiguousarray(a, dt)
        quant = self.cfg.kv_bits != 16
        arrs = [c(dump.k_codes, np.uint8), c(dump.k_scale, np.float32), c(dump.k_zero, np.float32),
                c(dump.v_codes, np.uint8), c(dump.v_scale, np.float32), c(dump.v_zero, np.float32)] if quant else [None] * 6
        arrs += [None, None] if quant else [c(dump.k_bf16, np.uint16), c(dump.v_bf16, np.uint16)]
        arrs += [c(dump.token_frame, np.int32), c(dump.token_index, np.int32)]
        _check(lib().xsv_cache_import(self._h, layer, int(dump.T), int(frames_seen), *[_np_ptr(a) for a in arrs]),
               "xsv_cache_import")

    def last_selection(self, layer=0):
        ns, nk = C.c_int32(), C.c_int32()
        _check(lib().xsv_last_selection(self._h, layer, C.byref(ns), None, C.byref(nk), None), "xsv_last_selection")
        lead = (self.cfg.n_heads,) if self.cfg.score_mode == 1 else ()
        scores = np.zeros(lead + (ns.value,), np.float32)
        keep = np.zeros(lead + (nk.value,), np.int32)
        _check(lib().xsv_last_selection(self._h, layer, C.byref(ns), _np_ptr(scores), C.byref(nk), _np_ptr(keep)),
               "xsv_last_selection")
        return scores, keep


# ---- stateless entry points (device tensors in, device tensors out) ----------------------------------

def _quantize(fn, name, x, bits, G, stream):
    if x.dtype != torch.bfloat16 or not x.is_contiguous() or x.dim() != 3:
        raise ValueError("expected a contiguous bf16 device tensor [H][T][d]")
    H, T, d = x.shape
    codes = torch.empty((H, T, d), dtype=torch.uint8, device=x.device)
    shape = (H, (T + G - 1) // G, d) if name.endswith("_k") else (H, T, d // G)
    scale = torch.empty(shape, dtype=torch.float32, device=x.device)
    zero = torch.empty(shape, dtype=torch.float32, device=x.device)
    _check(fn(_stream_ptr(stream), x.data_ptr(), H, T, d, bits, G, codes.data_ptr(), scale.data_ptr(), zero.data_ptr()), name)
    return codes, scale, zero


def quantize_k(k, bits, G, stream=None):
    return _quantize(lib().xsv_quantize_k, "xsv_quantize_k", k, bits, G, stream)


def quantize_v(v, bits, G, stream=None):
    return _quantize(lib().xsv_quantize_v, "xsv_quantize_v", v, bits, G, stream)


def score(q, k_mid, n_special, pool_size, stream=None):
    H, n, d = q.shape
    P = k_mid.shape[1]
    if k_mid.dtype != torch.bfloat16 or not k_mid.is_contiguous():
        raise ValueError("k_mid must be a contiguous bf16 device tensor [H][P][d]")
    out = torch.empty(P, dtype=torch.float32, device=q.device)
    _check(lib().xsv_score(_stream_ptr(stream), as_tensor(q), k_mid.data_ptr(), H, n, n_special, P, d, pool_size,
                           out.data_ptr()), "xsv_score")
    return out


def score_noalloc(q, k_mid, n_special, pool_size, out, stream=None):
    """xsv_score_noalloc: asynchronous on the stream, writes the caller's `out` (float32 device tensor [P])."""
    H, n, d = q.shape
    P = k_mid.shape[1]
    if k_mid.dtype != torch.bfloat16 or not k_mid.is_contiguous():
        raise ValueError("k_mid must be a contiguous bf16 device tensor [H][P][d]")
    if out.dtype != torch.float32 or not out.is_contiguous() or out.numel() < P or not out.is_cuda:
        raise ValueError("out must be a contiguous float32 device tensor of at least P elements")
    _check(lib().xsv_score_noalloc(_stream_ptr(stream), as_tensor(q), k_mid.data_ptr(), H, n, n_special, P, d, pool_size,
                                   out.data_ptr()), "xsv_score_noalloc")
    return out


def topk_keep(scores, k, T_first, T_cur, stream=None):
    P = scores.numel()
    keep = torch.empty(T_first + k + T_cur, dtype=torch.int32, device=scores.device)
    _check(lib().xsv_topk_keep(_stream_ptr(stream), scores.data_ptr() if P else None, P, k, T_first, T_cur,
                               keep.data_ptr()), "xsv_topk_keep")
    return keep


# ---- operators around the step: asynchronous on the stream (default: the current one of the tensors' device) ------------

_NO_TENSOR = xsv_tensor(None, 0, 0)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _tensor(t, name, beside=None, shape=None, written=False):
    """xsv_tensor of a bf16 device tensor [heads][rows][64], after the checks that need the torch tensor; the library checks pointers, strides
    and sizes.  beside: a tensor of the call on whose device it has to be.  (Every torch attribute costs some 0.1 us: each is asked for once.)"""
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.bfloat16 or t.dim() != 3 or not t.is_cuda:
        raise ValueError(f"{name}: expected a bf16 device tensor [heads][tokens][64]")
    size = t.shape
    if shape is not None and size != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(size)}")
    heads, rows, channels = size
    sh, st, sc = t.stride()
    if channels != 64 or (sc != 1 and heads and rows):
        raise ValueError(f"{name}: expected 64 contiguous channels")
    if beside is not None and t.get_device() != beside.get_device():
        raise ValueError(f"all tensors of a call must be on one device: {name} on {t.device}, others on {beside.device}")
    if written and ((heads > 1 and sh == 0) or (rows > 1 and st == 0)):
        raise ValueError(f"{name}: an output must not be an expanded tensor")
    # (the strides of an axis of one entry mean nothing to the tensor and are free)
    return xsv_tensor(t.data_ptr(), 0 if heads == 1 else sh, 64 if rows == 1 else st)


def _plain(t, name, dtype, shape, device):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.shape != shape or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor {tuple(shape)} on {device}")
    return t


class _on:
    """For one call: the tensors' device is the current one, and what the call allocates belongs to the stream it runs on."""

    __slots__ = ("device", "guards")

    def __init__(self, device, stream):
        self.device, self.guards = device, ()
        if stream is not None:
            if stream.device != device:
                raise ValueError(f"stream of {stream.device}, tensors on {device}")
            if device.index != torch.cuda.current_device() or stream.cuda_stream != torch._C._cuda_getCurrentRawStream(device.index):
                self.guards = (torch.cuda.device(device), torch.cuda.stream(stream))
        elif device.index != torch.cuda.current_device():
            self.guards = (torch.cuda.device(device),)

    def __enter__(self):
        for g in self.guards:
            g.__enter__()
        # (the handle alone: a Stream object around it costs 1.8 us, and a call takes 15)
        return torch._C._cuda_getCurrentRawStream(self.device.index)

    def __exit__(self, *exc):
        for g in reversed(self.guards):
            g.__exit__(*exc)


def _output(out, name, x, new=torch.empty):
    """The caller's output tensor, checked, or a new one like x, and its xsv_tensor."""
    if out is None:
        out = new(x.shape, dtype=torch.bfloat16, device=x.device)
        return out, xsv_tensor(out.data_ptr(), out.stride(0), 64)
    return out, _tensor(out, name, x, x.shape, written=True)


def _workspace(size_of, cfg, device):
    """A call's workspace, of the size that the library asks for (None: it asks for none), and that size."""
    nbytes = C.c_int64()
    _check(size_of(C.byref(cfg), C.byref(nbytes)), size_of.__name__)
    n = nbytes.value
    return (torch.empty(n, dtype=torch.uint8, device=device) if n else None), n


def _rotate_config(q, k, norm, eps, q_weight, q_bias, k_weight, k_bias, positions, base, interleaved):
    if norm not in NORMS:
        raise ValueError(f"norm must be one of {sorted(NORMS)}")
    heads, n, _ = q.shape
    heads_k = 0
    if k is not None:
        heads_k, n_k, _ = k.shape
        if n_k != n:
            raise ValueError("q and k must have the same number of tokens")
    dev = q.device
    axes = 0
    if positions is not None:
        if positions.dim() == 1:
            positions = positions.view(n, 1) if positions.numel() == n else positions
        if positions.dim() != 2 or positions.shape[1] not in (1, 2):
            raise ValueError("positions: expected int32 [tokens] or [tokens][1 or 2]")
        axes = positions.shape[1]
        _plain(positions, "positions", torch.int32, (n, axes), dev)
    for name, w in (("q_weight", q_weight), ("q_bias", q_bias), ("k_weight", k_weight), ("k_bias", k_bias)):
        if w is not None:
            _plain(w, name, torch.float32, (64,), dev)
    return xsv_rotate_config(n, heads, heads_k, NORMS[norm], axes, int(bool(interleaved)), eps, base, _ptr(positions), _ptr(q_weight),
                             _ptr(q_bias), _ptr(k_weight), _ptr(k_bias))


def norm_rotate(q, k=None, *, norm="layer", eps=1e-5, q_weight=None, q_bias=None, k_weight=None, k_bias=None, positions=None,
                base=100.0, interleaved=False, out=None, stream=None):
    """xsv_norm_rotate: norm per head, weight and bias (fp32 [64]) and rotation by `positions` (int32 [tokens] or [tokens][1 or 2];
    None: no rotation) of queries and, unless None, keys.  Returns (q_out, k_out), contiguous unless `out` gives the two."""
    tq = _tensor(q, "q")
    tk = _NO_TENSOR if k is None else _tensor(k, "k", q)
    cfg = _rotate_config(q, k, norm, eps, q_weight, q_bias, k_weight, k_bias, positions, base, interleaved)
    q_out, k_out = out if out is not None else (None, None)
    with _on(q.device, stream) as s:
        q_out, tq_out = _output(q_out, "out[0]", q)
        k_out, tk_out = (None, _NO_TENSOR) if k is None else _output(k_out, "out[1]", k)
        _check(lib().xsv_norm_rotate(s, C.byref(cfg), tq, tk, tq_out, tk_out), "xsv_norm_rotate")
    return q_out, k_out


def norm_rotate_grad(dq_out, dk_out, q, k=None, *, norm="layer", eps=1e-5, q_weight=None, q_bias=None, k_weight=None, k_bias=None,
                     positions=None, base=100.0, interleaved=False, out=None, weight_grads=True, stream=None):
    """xsv_norm_rotate_grad: (dq, dk, gradients of q_weight, q_bias, k_weight, k_bias as fp32 [4][64]) from the gradients of the
    outputs of norm_rotate and what it was called with.  weight_grads=False leaves the last out (None)."""
    tq = _tensor(q, "q")
    tdq_out = _tensor(dq_out, "dq_out", q, q.shape)
    tk = tdk_out = _NO_TENSOR
    if k is not None:
        tk, tdk_out = _tensor(k, "k", q), _tensor(dk_out, "dk_out", q, k.shape)
    cfg = _rotate_config(q, k, norm, eps, q_weight, q_bias, k_weight, k_bias, positions, base, interleaved)
    dq, dk = out if out is not None else (None, None)
    sums, work, n_work = None, None, 0
    with _on(q.device, stream) as s:
        dq, tdq = _output(dq, "out[0]", q)
        dk, tdk = (None, _NO_TENSOR) if k is None else _output(dk, "out[1]", k)
        if weight_grads:
            sums = torch.empty((4, 64), dtype=torch.float32, device=q.device)
            work, n_work = _workspace(lib().xsv_norm_rotate_grad_workspace, cfg, q.device)
        _check(lib().xsv_norm_rotate_grad(s, C.byref(cfg), tq, tk, tdq_out, tdk_out, tdq, tdk, _ptr(sums), _ptr(work), n_work),
               "xsv_norm_rotate_grad")
    return dq, dk, sums


def _seq_config(q, k, q_begin, k_begin, longest_q, longest_k, causal, softmax_scale):
    if k_begin is None:
        k_begin = q_begin
    n = q_begin.numel() - 1 if isinstance(q_begin, torch.Tensor) else -1
    if n < 0:
        raise ValueError("q_begin: expected int32 [sequences + 1]")
    for name, t in (("q_begin", q_begin), ("k_begin", k_begin)):
        _plain(t, name, torch.int32, (n + 1,), q.device)
    (heads, rows_q, _), (kv_heads, rows_k, _) = q.shape, k.shape
    longest_q = rows_q if longest_q is None else longest_q
    longest_k = rows_k if longest_k is None else longest_k
    # (ctypes cuts integers down to 32 bits, and rounds a scale to fp32: to 0, which would ask for the usual one)
    if max(longest_q, longest_k, causal) >= 1 << 31 or min(longest_q, longest_k, causal) < -(1 << 31) or 0.0 < abs(softmax_scale) < 1e-40:
        raise ValueError("longest_q, longest_k and causal must fit 32 bits, softmax_scale fp32")
    return xsv_seq_config(heads, kv_heads, n, rows_q, rows_k, longest_q, longest_k, _ptr(q_begin), _ptr(k_begin), causal, softmax_scale)


def seq_attend(q, k, v, q_begin, k_begin=None, *, longest_q=None, longest_k=None, causal=0, softmax_scale=0.0, out=None, lse=None, stream=None):
    """xsv_seq_attend: attention of q [heads][rows][64] over k, v [kv_heads][rows][64] inside the sequences that the int32 device tensors
    q_begin and k_begin (None: the same) bound.  longest_q / longest_k, the lengths of the longest, size the launch (None: all rows).
    Returns (out, lse); tensors that it makes hold zeros in rows of no sequence."""
    tq, tk = _tensor(q, "q"), _tensor(k, "k", q)
    tv = _tensor(v, "v", q, k.shape)
    cfg = _seq_config(q, k, q_begin, k_begin, longest_q, longest_k, causal, softmax_scale)
    with _on(q.device, stream) as s:
        out, t_out = _output(out, "out", q, torch.zeros)
        if lse is None:
            lse = torch.zeros(q.shape[:2], dtype=torch.float32, device=q.device)
        else:
            _plain(lse, "lse", torch.float32, q.shape[:2], q.device)
        work, n_work = _workspace(lib().xsv_seq_attend_workspace, cfg, q.device)
        _check(lib().xsv_seq_attend(s, C.byref(cfg), tq, tk, tv, t_out, lse.data_ptr(), _ptr(work), n_work), "xsv_seq_attend")
    return out, lse


def seq_attend_grad(dout, q, k, v, out, lse, q_begin, k_begin=None, *, longest_q=None, longest_k=None, causal=0, softmax_scale=0.0, grads=None,
                    stream=None):
    """xsv_seq_attend_grad: (dq, dk, dv) from the gradient of seq_attend's out, what it was called with and what it returned.  `grads`
    gives the three tensors to write; those that it makes hold zeros in rows of no sequence."""
    tq, tk = _tensor(q, "q"), _tensor(k, "k", q)
    tv, tdout, t_out = _tensor(v, "v", q, k.shape), _tensor(dout, "dout", q, q.shape), _tensor(out, "out", q, q.shape)
    cfg = _seq_config(q, k, q_begin, k_begin, longest_q, longest_k, causal, softmax_scale)
    _plain(lse, "lse", torch.float32, q.shape[:2], q.device)
    dq, dk, dv = grads if grads is not None else (None, None, None)
    with _on(q.device, stream) as s:
        (dq, tdq), (dk, tdk) = _output(dq, "grads[0]", q, torch.zeros), _output(dk, "grads[1]", k, torch.zeros)
        dv, tdv = _output(dv, "grads[2]", v, torch.zeros)
        work, n_work = _workspace(lib().xsv_seq_attend_grad_workspace, cfg, q.device)
        _check(lib().xsv_seq_attend_grad(s, C.byref(cfg), tq, tk, tv, t_out, lse.data_ptr(), tdout, tdq, tdk, tdv, _ptr(work), n_work),
               "xsv_seq_attend_grad")
    return dq, dk, dv


def key_ranges(cache_tiles, frame_tiles, ranges, last_percent=100, frame_tile_cost=95):
    """xsv_key_ranges (host only): the tile index at which each of `ranges` key ranges begins, plus the total."""
    begin = (C.c_int32 * (ranges + 1))()
    _check(lib().xsv_key_ranges(cache_tiles, frame_tiles, ranges, last_percent, frame_tile_cost, begin), "xsv_key_ranges")
    return list(begin)


def measure_peaks(stream=None):
    """(bf16 MFMA loop TFLOP/s, streaming copy GB/s) of the current device."""
    a, b = C.c_float(), C.c_float()
    _check(lib().xsv_measure_peaks(_stream_ptr(stream), C.byref(a), C.byref(b)), "xsv_measure_peaks")
    return a.value, b.value
