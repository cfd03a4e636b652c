"""ctypes binding of libfdkv (argument marshalling only).

Each function mirrors one entry point of ``include/fdkv.h`` and takes torch
tensors for device buffers (their ``data_ptr()`` is passed) and numpy arrays
for host buffers.  Work is queued on the current torch stream.  Nothing here
computes any part of the method; a missing library raises ``RuntimeError``.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Sequence

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libfdkv.so")
_lib = None

SHARED, RESIDUAL, EXACT = 0, 1, 2
F32, BF16, BF16_E4M3 = 0, 1, 2   # cache types (fdkv_dtype)

STATUS = {0: "FDKV_OK", -1: "FDKV_E_INVALID_ARG", -2: "FDKV_E_UNSUPPORTED", -3: "FDKV_E_WORKSPACE",
          -4: "FDKV_E_BUDGET", -5: "FDKV_E_HIP"}

SYMBOLS = ("fdkv_status_string", "fdkv_last_error", "fdkv_blocks", "fdkv_layout", "fdkv_route",
           "fdkv_probe_workspace", "fdkv_probe", "fdkv_compress", "fdkv_decode_workspace", "fdkv_decode_attn",
           "fdkv_append", "fdkv_decode_spans_workspace", "fdkv_decode_spans", "fdkv_decode_static_scratch_bytes",
           "fdkv_decode_attn_static", "fdkv_decode_partial", "fdkv_decode_combine", "fdkv_selection_bytes",
           "fdkv_check_conversions", "fdkv_rope_append",
           "fdkv_key_bounds", "fdkv_block_select_workspace", "fdkv_block_select", "fdkv_decode_parts_workspace",
           "fdkv_decode_parts")
PAIRS, MIXED, QUADS = 0, 1, 2    # block schedules (fdkv_schedule)
RES_CHANNELS, RES_TOKENS = 0, 1  # residual kinds (fdkv_residual)
PART_OWN, PART_BLOCKS, PART_SHARED = 0, 1, 2  # parts of a decode step (fdkv_part_kind)
BLOCK_TOKENS = 64                # tokens of a block of sparse decode (FDKV_BLOCK_TOKENS)
MAX_SELECTED, MAX_SELECT_UNITS = 1 << 24, 65535  # of fdkv_block_select: n_sel, and batch x Hkv


class FdkvError(RuntimeError):
    def __init__(self, status: int, where: str):
        lib = load()
        msg = lib.fdkv_status_string(status).decode()
        if status == -5 or (status == -3 and "static" in where):
            msg += ": " + lib.fdkv_last_error().decode()
        super().__init__(f"{where}: {STATUS.get(status, status)} ({msg})")
        self.status = status


class Dims(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("topk", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("schedule", ctypes.c_int32), ("residual", ctypes.c_int32), ("res_ppm", ctypes.c_int32),
                ("n_rates", ctypes.c_int32), ("rates_ppm", ctypes.c_int32 * 8)]

    @property
    def n_err(self) -> int:
        """Columns of the probe's loss array: E_S, then E_R at each candidate fraction."""
        return 1 + (self.n_rates if self.residual == RES_TOKENS and self.n_rates else 1)


class Span(ctypes.Structure):
    _fields_ = [("seq_lens", ctypes.c_void_p), ("max_seq_len", ctypes.c_int32), ("modes", ctypes.c_void_p),
                ("seg_offsets", ctypes.c_void_p), ("cache", ctypes.c_void_p)]


class Tail(ctypes.Structure):
    _fields_ = [("lens", ctypes.c_void_p), ("cap", ctypes.c_int32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p)]


class Part(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("max_seq_len", ctypes.c_int32), ("n_sel", ctypes.c_int32),
                ("seq_lens", ctypes.c_void_p), ("modes", ctypes.c_void_p), ("seg_offsets", ctypes.c_void_p),
                ("cache", ctypes.c_void_p), ("blocks", ctypes.c_void_p), ("counts", ctypes.c_void_p)]


class Rope(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("n_axes", ctypes.c_int32),
                ("inv_freq", ctypes.c_void_p), ("pos", ctypes.c_void_p), ("axis", ctypes.c_uint8 * 64)]


def dims(n_layers, n_kv_heads, n_q_heads, head_dim, topk, dtype, schedule=PAIRS, residual=RES_CHANNELS,
         res_ppm=0, res_rates=()) -> Dims:
    """``res_rates``: routed candidate fractions (ppm) of token-level sets, at most 8."""
    dt = {"f32": F32, "bf16": BF16, "bf16_e4m3": BF16_E4M3}.get(dtype, dtype)
    rates = list(res_rates) + [0] * (8 - len(res_rates))
    return Dims(n_layers, n_kv_heads, n_q_heads, head_dim, topk, dt, schedule, residual, res_ppm, len(res_rates),
                (ctypes.c_int32 * 8)(*rates))


def load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is not built; run __graft_entry__.build() first")
    lib = ctypes.CDLL(_LIB_PATH)
    P, I32, I64, U64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t
    DP = ctypes.POINTER(Dims)
    lib.fdkv_status_string.restype = ctypes.c_char_p
    lib.fdkv_status_string.argtypes = [I32]
    lib.fdkv_last_error.restype = ctypes.c_char_p
    lib.fdkv_last_error.argtypes = []
    lib.fdkv_blocks.restype = I32
    lib.fdkv_blocks.argtypes = [DP, P, P, P]
    lib.fdkv_layout.restype = I32
    lib.fdkv_layout.argtypes = [DP, I32, P, P, P, P]
    lib.fdkv_route.restype = I32
    lib.fdkv_route.argtypes = [DP, I32, P, ctypes.c_double, U64, P, P]
    lib.fdkv_probe_workspace.restype = I32
    lib.fdkv_probe_workspace.argtypes = [DP, I32, I32, P]
    lib.fdkv_probe.restype = I32
    lib.fdkv_probe.argtypes = [DP, I32, P, P, I32, P, P, P, SZ, P, P]
    lib.fdkv_compress.restype = I32
    lib.fdkv_compress.argtypes = [DP, I32, P, P, P, P, P, P, P, P]
    lib.fdkv_selection_bytes.restype = I32
    lib.fdkv_selection_bytes.argtypes = [DP, I32, P]
    lib.fdkv_check_conversions.restype = I32
    lib.fdkv_check_conversions.argtypes = [P, P]
    lib.fdkv_decode_workspace.restype = I32
    lib.fdkv_decode_workspace.argtypes = [DP, I32, I32, P]
    lib.fdkv_decode_attn.restype = I32
    lib.fdkv_decode_attn.argtypes = [DP, I32, P, I32, P, P, P, I32, P, P, ctypes.c_float, P, SZ, P]
    lib.fdkv_decode_static_scratch_bytes.restype = SZ
    lib.fdkv_decode_static_scratch_bytes.argtypes = []
    lib.fdkv_decode_attn_static.restype = I32
    lib.fdkv_decode_attn_static.argtypes = [DP, I32, P, I32, P, P, P, I32, P, P, ctypes.c_float, P]
    lib.fdkv_decode_partial.restype = I32
    lib.fdkv_decode_partial.argtypes = [DP, I32, P, I32, P, P, P, I32, P, ctypes.c_float, P, SZ, P]
    lib.fdkv_decode_combine.restype = I32
    lib.fdkv_decode_combine.argtypes = [DP, I32, I32, P, P, SZ, P]
    lib.fdkv_append.restype = I32
    lib.fdkv_append.argtypes = [DP, I32, P, I32, P, P, P, P, P]
    lib.fdkv_decode_spans_workspace.restype = I32
    lib.fdkv_decode_spans_workspace.argtypes = [DP, I32, I32, P, I32, P]
    lib.fdkv_decode_spans.restype = I32
    lib.fdkv_decode_spans.argtypes = [DP, I32, I32, P, P, I32, P, P, ctypes.c_float, P, SZ, P]
    lib.fdkv_rope_append.restype = I32
    lib.fdkv_rope_append.argtypes = [DP, I32, P, P, I64, P, I64, P, I64, P, P, ctypes.c_float, P, I32, P, P, I32, P, P, P]
    lib.fdkv_key_bounds.restype = I32
    lib.fdkv_key_bounds.argtypes = [DP, I32, P, P, I32, P]
    lib.fdkv_block_select_workspace.restype = I32
    lib.fdkv_block_select_workspace.argtypes = [DP, I32, I32, P]
    lib.fdkv_block_select.restype = I32
    lib.fdkv_block_select.argtypes = [DP, I32, P, I32, P, P, I32, I32, I32, P, P, P, SZ, P]
    lib.fdkv_decode_parts_workspace.restype = I32
    lib.fdkv_decode_parts_workspace.argtypes = [DP, I32, I32, P, I32, P]
    lib.fdkv_decode_parts.restype = I32
    lib.fdkv_decode_parts.argtypes = [DP, I32, I32, P, P, I32, P, P, ctypes.c_float, P, SZ, P]
    _lib = lib
    return lib


def _check(st: int, where: str):
    if st != 0:
        raise FdkvError(st, where)


def _np_ptr(a: np.ndarray):
    return a.ctypes.data_as(ctypes.c_void_p)


def _dev(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        # the handle of torch's current stream, without the Stream object around it
        # (0.3 us instead of 2.9 us, which counts on calls of some 10 us)
        import torch
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return ctypes.c_void_p(int(stream.cuda_stream))


@functools.lru_cache(maxsize=256)
def _array_type(element, n: int):
    """The ctypes array type, kept: made anew for each call it costs about 15 us."""
    return element * n


def _ptr_array(tensors: Sequence) -> ctypes.Array:
    return _array_type(ctypes.c_void_p, len(tensors))(*[_dev(t) for t in tensors])


# ----------------------------------------------------------------- host entry points
def blocks(d: Dims):
    """``(first_layer [n_blocks] int32, block_size [n_blocks] int32)`` of the schedule."""
    lib = load()
    n = ctypes.c_int32(0)
    _check(lib.fdkv_blocks(ctypes.byref(d), ctypes.byref(n), None, None), "fdkv_blocks")
    first = np.zeros(n.value, dtype=np.int32)
    size = np.zeros(n.value, dtype=np.int32)
    _check(lib.fdkv_blocks(ctypes.byref(d), ctypes.byref(n), _np_ptr(first), _np_ptr(size)), "fdkv_blocks")
    return first, size


def layout(d: Dims, seq_lens, modes):
    """``(seg_offsets [batch][n_blocks][Hkv] uint64, total_bytes)`` for host ``modes``."""
    lib = load()
    sl = np.ascontiguousarray(seq_lens, dtype=np.int32)
    m = np.ascontiguousarray(modes, dtype=np.uint8)
    off = np.zeros(m.shape, dtype=np.uint64)
    total = ctypes.c_uint64(0)
    _check(lib.fdkv_layout(ctypes.byref(d), int(sl.size), _np_ptr(sl), _np_ptr(m), _np_ptr(off),
                           ctypes.byref(total)), "fdkv_layout")
    return off, int(total.value)


def route(d: Dims, seq_len: int, errors, lam: float = 0.0, budget_bytes: int = 0, allow_infeasible=False):
    """``(modes [n_blocks][Hkv] uint8, lambda_used, status)`` from host ``errors [n_blocks][Hkv][n_err]``
    (the mode bytes carry the routed fraction index of residual units in bits 2-4)."""
    lib = load()
    e = np.ascontiguousarray(errors, dtype=np.float32)
    modes = np.zeros(e.shape[:-1], dtype=np.uint8)
    lam_out = ctypes.c_double(0.0)
    st = lib.fdkv_route(ctypes.byref(d), int(seq_len), _np_ptr(e), float(lam), int(budget_bytes),
                        _np_ptr(modes), ctypes.byref(lam_out))
    if not (st == 0 or (st == -4 and allow_infeasible)):
        _check(st, "fdkv_route")
    return modes, float(lam_out.value), st


def probe_workspace(d: Dims, seq_len: int, n_probe: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load().fdkv_probe_workspace(ctypes.byref(d), int(seq_len), int(n_probe), ctypes.byref(n)),
           "fdkv_probe_workspace")
    return int(n.value)


def selection_bytes(d: Dims, seq_len: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load().fdkv_selection_bytes(ctypes.byref(d), int(seq_len), ctypes.byref(n)), "fdkv_selection_bytes")
    return int(n.value)


def check_conversions(stream=None) -> tuple:
    """Mismatches of the device E4M3 encoder and bf16 rounding against their integer
    definitions over every non-NaN fp32 bit pattern (fdkv_check_conversions)."""
    out = (ctypes.c_uint64 * 2)()
    _check(load().fdkv_check_conversions(out, _stream(stream)), "fdkv_check_conversions")
    return int(out[0]), int(out[1])


def decode_workspace(d: Dims, batch: int, max_seq_len: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load().fdkv_decode_workspace(ctypes.byref(d), int(batch), int(max_seq_len), ctypes.byref(n)),
           "fdkv_decode_workspace")
    return int(n.value)


# ----------------------------------------------------------------- device entry points
def probe(d: Dims, seq_len: int, k_layers: Sequence, qp_layers: Sequence, n_probe: int, errors_out, ws,
          stream=None, token_scores=None, k_select=None):
    """Queue fdkv_probe; ``k_layers``/``qp_layers`` are per-layer device tensors;
    ``token_scores`` (token-level residual set) receives s_t ``[n_blocks][Hkv][T]``;
    ``k_select`` (``selection_bytes`` bytes) the K selections for compress to reuse."""
    _check(load().fdkv_probe(ctypes.byref(d), int(seq_len), _ptr_array(k_layers), _ptr_array(qp_layers),
                             int(n_probe), _dev(errors_out), _dev(token_scores), _dev(ws),
                             int(ws.numel() * ws.element_size()), _dev(k_select), _stream(stream)), "fdkv_probe")


def compress(d: Dims, seq_len: int, k_layers: Sequence, v_layers: Sequence, modes, seg_offsets, cache,
             stream=None, token_scores=None, k_select=None):
    """Queue fdkv_compress for one sequence (``modes``/``seg_offsets`` device tensors; ``token_scores``
    from the probe when residual heads hold a token-level set; ``k_select`` the probe's K selections
    of the same keys, or None to select in the pass)."""
    _check(load().fdkv_compress(ctypes.byref(d), int(seq_len), _ptr_array(k_layers), _ptr_array(v_layers),
                                _dev(modes), _dev(seg_offsets), _dev(token_scores), _dev(k_select), _dev(cache),
                                _stream(stream)), "fdkv_compress")


def decode_attn(d: Dims, batch: int, seq_lens, max_seq_len: int, modes, seg_offsets, cache, layer: int, q, out,
                sm_scale: float, ws, stream=None):
    """Queue fdkv_decode_attn for one layer."""
    _check(load().fdkv_decode_attn(ctypes.byref(d), int(batch), _dev(seq_lens), int(max_seq_len), _dev(modes),
                                   _dev(seg_offsets), _dev(cache), int(layer), _dev(q), _dev(out),
                                   ctypes.c_float(sm_scale), _dev(ws), int(ws.numel() * ws.element_size()),
                                   _stream(stream)), "fdkv_decode_attn")


def decode_partial(d: Dims, batch: int, seq_lens, max_seq_len: int, modes, seg_offsets, cache, layer: int, q,
                   sm_scale: float, ws, stream=None):
    """Queue fdkv_decode_partial: the split-K records of one layer into ``ws``."""
    _check(load().fdkv_decode_partial(ctypes.byref(d), int(batch), _dev(seq_lens), int(max_seq_len), _dev(modes),
                                      _dev(seg_offsets), _dev(cache), int(layer), _dev(q), ctypes.c_float(sm_scale),
                                      _dev(ws), int(ws.numel() * ws.element_size()), _stream(stream)),
           "fdkv_decode_partial")


def decode_combine(d: Dims, batch: int, n_chunks: int, out, ws, stream=None):
    """Queue fdkv_decode_combine: merge ``n_chunks`` records per (sequence, query head) of ``ws`` into ``out``."""
    _check(load().fdkv_decode_combine(ctypes.byref(d), int(batch), int(n_chunks), _dev(out), _dev(ws),
                                      int(ws.numel() * ws.element_size()), _stream(stream)), "fdkv_decode_combine")


def decode_static_scratch_bytes() -> int:
    """Bytes of the static device scratch behind fdkv_decode_attn_static."""
    return int(load().fdkv_decode_static_scratch_bytes())


def decode_attn_static(d: Dims, batch: int, seq_lens, max_seq_len: int, modes, seg_offsets, cache, layer: int, q,
                       out, sm_scale: float, stream=None):
    """Queue fdkv_decode_attn_static for one layer (no workspace: the library's static scratch)."""
    _check(load().fdkv_decode_attn_static(ctypes.byref(d), int(batch), _dev(seq_lens), int(max_seq_len), _dev(modes),
                                          _dev(seg_offsets), _dev(cache), int(layer), _dev(q), _dev(out),
                                          ctypes.c_float(sm_scale), _stream(stream)), "fdkv_decode_attn_static")


def decode_attn_raw(d: Dims, batch: int, seq_lens_ptr: int, max_seq_len: int, modes_ptr: int, offs_ptr: int,
                    cache_ptr: int, layer: int, q_ptr: int, out_ptr: int, sm_scale: float, ws_ptr: int,
                    ws_bytes: int, stream_ptr: int) -> int:
    """Same call with raw integer pointers (for tight timing loops); returns the status."""
    return load().fdkv_decode_attn(ctypes.byref(d), batch, seq_lens_ptr, max_seq_len, modes_ptr, offs_ptr,
                                   cache_ptr, layer, q_ptr, out_ptr, ctypes.c_float(sm_scale), ws_ptr, ws_bytes,
                                   ctypes.c_void_p(stream_ptr))


# ----------------------------------------------------------------- generation: spans and the exact tail
def append(d: Dims, batch: int, pos, cap: int, k_new, v_new, tail_k, tail_v, stream=None):
    """Queue fdkv_append: row ``pos[s]`` of the layer's tail gets the new K / V rows."""
    _check(load().fdkv_append(ctypes.byref(d), int(batch), _dev(pos), int(cap), _dev(k_new), _dev(v_new),
                              _dev(tail_k), _dev(tail_v), _stream(stream)), "fdkv_append")


def decode_spans_workspace(d: Dims, batch: int, max_seq_lens, tail_cap: int) -> int:
    m = np.ascontiguousarray(max_seq_lens, dtype=np.int32)
    n = ctypes.c_size_t(0)
    _check(load().fdkv_decode_spans_workspace(ctypes.byref(d), int(batch), int(m.size), _np_ptr(m),
                                              int(tail_cap), ctypes.byref(n)), "fdkv_decode_spans_workspace")
    return int(n.value)


def decode_spans(d: Dims, batch: int, spans: Sequence[Span], tail, layer: int, q, out, sm_scale: float, ws,
                 stream=None):
    """Queue fdkv_decode_spans; ``spans`` are ``Span`` descriptors, ``tail`` a ``Tail`` or None."""
    arr = _array_type(Span, max(len(spans), 1))(*spans)
    _check(load().fdkv_decode_spans(ctypes.byref(d), int(batch), len(spans), ctypes.cast(arr, ctypes.c_void_p),
                                    None if tail is None else ctypes.byref(tail), int(layer), _dev(q), _dev(out),
                                    ctypes.c_float(sm_scale), _dev(ws), int(ws.numel() * ws.element_size()),
                                    _stream(stream)), "fdkv_decode_spans")


# ----------------------------------------------------------------- a step's rows: norm, rotation, cache
@functools.lru_cache(maxsize=None)
def _element(dtype: int):
    """The torch type of inputs, queries and outputs."""
    import torch
    return torch.float32 if dtype == F32 else torch.bfloat16


def _operands(what: str, element, tensors, numbers=(), ws=None):
    """Refuses operands that a kernel would misread: ``tensors`` (each with the values that it holds at least) of another
    element type, ``numbers`` that are not int32, any that is not contiguous, too short or on another device than the
    current one, and a workspace ``ws`` with gaps or on another device (its size is the library's to check)."""
    import torch
    here = torch.cuda.current_device()
    for t, n in tensors:
        if t.dtype is not element or t.get_device() != here or t.numel() < n or not t.is_contiguous():
            raise ValueError(f"{what}: {t.dtype} {list(t.shape)} on {t.device}, not {n} contiguous {element} on cuda:{here}")
    if ws is not None and (ws.get_device() != here or not ws.is_contiguous()):
        raise ValueError(f"{what}: a workspace on {ws.device}, strides {ws.stride()}, not contiguous on cuda:{here}")
    if numbers:
        _operands(what, torch.int32, numbers)


@functools.lru_cache(maxsize=256)
def _n_blocks(n_layers: int, schedule: int) -> int:
    """Blocks of layers of a schedule."""
    return len(blocks(dims(n_layers, 1, 1, 64, 0, "f32", schedule))[0])


def rope(rot_dim: int, inv_freq, pos, axis: Sequence[int] = (), interleaved: bool = False) -> Rope:
    """Rotary positions: ``inv_freq`` device float64 ``[rot_dim / 2]``, ``pos`` device int32 ``[n_tokens]``
    or ``[n_axes][n_tokens]``, ``axis`` the axis that each pair follows (default: axis 0).  The descriptor
    keeps both tensors."""
    import torch
    n_axes = 1 if pos.dim() == 1 else int(pos.shape[0])
    if inv_freq.dtype != torch.float64 or pos.dtype != torch.int32 or pos.dim() > 2:
        raise ValueError("rope: inv_freq is float64, pos int32 [n_tokens] or [n_axes][n_tokens]")
    if inv_freq.get_device() != pos.get_device():
        raise ValueError("rope: inv_freq and pos lie on one device")
    if inv_freq.numel() < rot_dim // 2 or not inv_freq.is_contiguous() or not pos.is_contiguous():
        raise ValueError("rope: inv_freq holds rot_dim / 2 values; both tensors are contiguous")
    if len(axis) not in (0, rot_dim // 2) or rot_dim > 128:
        raise ValueError("rope: one axis for each of the rot_dim / 2 pairs")
    if len(axis) and not (min(axis) >= 0 and max(axis) < n_axes):
        raise ValueError(f"rope: an axis of a pair is 0 .. {n_axes - 1}, a row of pos")
    r = Rope(int(rot_dim), int(interleaved), n_axes, _dev(inv_freq), _dev(pos), (ctypes.c_uint8 * 64)(*axis))
    r.tensors = (inv_freq, pos)
    r.n_tokens, r.device = int(pos.shape[-1]), pos.get_device()
    return r


def rope_append(d: Dims, rope: Rope, q, k, v, q_out, seqs, rows, k_out, v_out, q_norm=None, k_norm=None,
                eps: float = 1e-6, stream=None):
    """Queue fdkv_rope_append: ``q [n][Hq][d]``, ``k`` / ``v [n][Hkv][d]`` (views of one fused projection, say),
    ``k_out`` / ``v_out [batch][Hkv][cap][d]``; ``seqs`` None: token i is of sequence i."""
    # (checks without loops and calls of their own, which would cost a call of 10 us two more)
    import torch
    hd, hkv = d.head_dim, d.n_kv_heads
    n, hq, _ = heads = q.shape
    kv = k.shape
    qs, q1, q2 = q.stride()
    ks, k1, k2 = k.stride()
    vs, v1, v2 = v.stride()
    if heads != (n, d.n_q_heads, hd) or kv != (n, hkv, hd) or v.shape != kv or not q2 == k2 == v2 == 1 or \
            (q1 != hd and hq > 1) or (hkv > 1 and not k1 == v1 == hd):
        raise ValueError("rope_append: q is [n][Hq][d], k and v [n][Hkv][d], contiguous but for their token strides")
    batch, kh, cap, kd = cache = k_out.shape
    if q_out.shape != heads or kh != hkv or kd != hd or v_out.shape != cache or \
            not (q_out.is_contiguous() and k_out.is_contiguous() and v_out.is_contiguous()):
        raise ValueError("rope_append: q_out is [n][Hq][d], k_out and v_out [batch][Hkv][cap][d], all contiguous")
    e, i32, at = _element(d.dtype), torch.int32, torch.cuda.current_device()
    if not (e is q.dtype is k.dtype is v.dtype is q_out.dtype is k_out.dtype is v_out.dtype) or \
            not (at == q.get_device() == k.get_device() == v.get_device() == q_out.get_device() == k_out.get_device() ==
                 v_out.get_device() == rows.get_device()):
        raise ValueError(f"rope_append: q, k, v and the outputs are {e}, all on the current device (cuda:{at})")
    if rows.dtype is not i32 or rows.shape != (n,) or not rows.is_contiguous() or \
            (rope.rot_dim and (rope.n_tokens != n or rope.device != at)) or \
            (seqs is not None and (seqs.dtype is not i32 or seqs.shape != (n,) or not seqs.is_contiguous() or
                                   seqs.get_device() != at)):
        raise ValueError(f"rope_append: rows and seqs are contiguous int32 [n] on cuda:{at}, the positions of n tokens")
    if q_norm is not None or k_norm is not None:
        _operands("rope_append", e, [(t, hd) for t in (q_norm, k_norm) if t is not None])
    st = (_lib or load()).fdkv_rope_append(
        ctypes.byref(d), n, ctypes.byref(rope), q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs,
        q_norm.data_ptr() if q_norm is not None else 0, k_norm.data_ptr() if k_norm is not None else 0, eps,
        q_out.data_ptr(), batch, seqs.data_ptr() if seqs is not None else 0, rows.data_ptr(), cap, k_out.data_ptr(),
        v_out.data_ptr(), torch._C._cuda_getCurrentRawStream(at) if stream is None else stream.cuda_stream)
    if st:
        _check(st, "fdkv_rope_append")


# ----------------------------------------------------------------- sparse decode: the index and the selection
def key_bounds(d: Dims, seq_len: int, k_layers: Sequence, bounds_layers: Sequence, blocks_cap: int, stream=None):
    """Queue fdkv_key_bounds: per layer ``k [Hkv][T][d]`` -> ``bounds [Hkv][blocks_cap][2][d]``."""
    if len(k_layers) != d.n_layers or len(bounds_layers) != d.n_layers:
        raise ValueError("key_bounds: one tensor of keys and one of bounds for every layer")
    # (a tensor's checks and its address in one pass, as a call takes some 10 us)
    import torch
    e, at, row = _element(d.dtype), torch.cuda.current_device(), d.n_kv_heads * d.head_dim
    nk, nb = int(seq_len) * row, int(blocks_cap) * 2 * row
    k = [t.data_ptr() for t in k_layers
         if t.dtype is e and t.get_device() == at and t.is_contiguous() and t.numel() >= nk]
    b = [t.data_ptr() for t in bounds_layers
         if t.dtype is e and t.get_device() == at and t.is_contiguous() and t.numel() >= nb]
    if len(k) != len(k_layers) or len(b) != len(bounds_layers):
        raise ValueError(f"key_bounds: keys and bounds are contiguous {e} on cuda:{at}, {nk} and {nb} values a layer")
    pointers = _array_type(ctypes.c_void_p, d.n_layers)
    _check((_lib or load()).fdkv_key_bounds(ctypes.byref(d), int(seq_len), pointers(*k), pointers(*b), int(blocks_cap),
                                            torch._C._cuda_getCurrentRawStream(at) if stream is None else
                                            stream.cuda_stream), "fdkv_key_bounds")


def block_select_workspace(d: Dims, batch: int, max_seq_len: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load().fdkv_block_select_workspace(ctypes.byref(d), int(batch), int(max_seq_len), ctypes.byref(n)),
           "fdkv_block_select_workspace")
    return int(n.value)


def block_select(d: Dims, batch: int, seq_lens, max_seq_len: int, bounds, q, n_first: int, n_last: int, n_sel: int,
                 blocks_out, counts_out, ws, stream=None):
    """Queue fdkv_block_select for one layer: ``blocks_out [batch][Hkv][n_sel]``, ``counts_out [batch][Hkv]`` int32."""
    units = int(batch) * d.n_kv_heads
    _operands("block_select", _element(d.dtype),
              ((bounds, units * -(-int(max_seq_len) // BLOCK_TOKENS) * 2 * d.head_dim), (q, int(batch) * d.n_q_heads * d.head_dim)),
              ((seq_lens, int(batch)), (blocks_out, units * int(n_sel)), (counts_out, units)), ws)
    _check(load().fdkv_block_select(ctypes.byref(d), int(batch), _dev(seq_lens), int(max_seq_len), _dev(bounds),
                                    _dev(q), int(n_first), int(n_last), int(n_sel), _dev(blocks_out),
                                    _dev(counts_out), _dev(ws), int(ws.numel() * ws.element_size()),
                                    _stream(stream)), "fdkv_block_select")


# ----------------------------------------------------------------- decode over parts
def part(kind: int, seq_lens, max_seq_len: int, modes, seg_offsets, cache, blocks=None, counts=None,
         n_sel: int = 0) -> Part:
    """A part of a decode step (PART_OWN, PART_BLOCKS or PART_SHARED); the descriptor keeps its tensors."""
    import torch
    for t, types in ((seq_lens, (torch.int32,)), (blocks, (torch.int32,)), (counts, (torch.int32,)), (modes, (torch.uint8, torch.int8)),
                     (seg_offsets, (torch.int64, torch.uint64)), (cache, (cache.dtype,))):
        if t is not None and (t.dtype not in types or not t.is_contiguous() or t.get_device() != cache.get_device()):
            raise ValueError(f"part: {t.dtype} {list(t.shape)} on {t.device}, not contiguous {types[0]} on the cache's device")
    p = Part(int(kind), int(max_seq_len), int(n_sel), _dev(seq_lens), _dev(modes), _dev(seg_offsets), _dev(cache),
             _dev(blocks), _dev(counts))
    p.tensors = (seq_lens, modes, seg_offsets, cache, blocks, counts)
    p.device, p.fits = cache.get_device(), None
    return p


def _fits(p: Part, batch: int, hkv: int, n_layers: int, schedule: int, device: int):
    """Refuses a part whose tensors are shorter than a call would read them, or on another device.  (A descriptor of plain
    addresses says nothing of what lies there.)"""
    seqs = 1 if p.kind == PART_SHARED else int(batch)
    units, chosen = seqs * hkv * _n_blocks(n_layers, schedule), seqs * hkv if p.kind == PART_BLOCKS else 0
    held = tuple(0 if t is None else t.numel() for i, t in enumerate(p.tensors) if i != 3)
    need = (seqs, units, units, chosen * p.n_sel, chosen)
    if any(h < m for h, m in zip(held, need)):
        raise ValueError(f"decode_parts: a part of {seqs} sequences takes {need} lengths, modes, offsets, blocks and counts; "
                         f"it has {held}")
    if p.device != device:
        raise ValueError("decode_parts: a part lies on another device than the queries")


def decode_parts_workspace(d: Dims, batch: int, parts: Sequence[Part], tail_cap: int) -> int:
    n = ctypes.c_size_t(0)
    arr = _array_type(Part, max(len(parts), 1))(*parts)
    _check(load().fdkv_decode_parts_workspace(ctypes.byref(d), int(batch), len(parts), ctypes.cast(arr, ctypes.c_void_p),
                                              int(tail_cap), ctypes.byref(n)), "fdkv_decode_parts_workspace")
    return int(n.value)


def decode_parts(d: Dims, batch: int, parts: Sequence[Part], tail, layer: int, q, out, sm_scale: float, ws,
                 stream=None):
    """Queue fdkv_decode_parts for one layer; ``parts`` are ``Part`` descriptors, ``tail`` a ``Tail`` or None."""
    n, call = int(batch) * d.n_q_heads * d.head_dim, (batch, d.n_kv_heads, d.n_layers, d.schedule)
    for p in parts:
        # (once for a descriptor and a kind of call, which some layers and steps repeat)
        if getattr(p, "device", None) is not None and p.fits != (call, p.kind, p.n_sel, q.get_device()):
            _fits(p, *call, q.get_device())
            p.fits = (call, p.kind, p.n_sel, q.get_device())
    _operands("decode_parts", _element(d.dtype), ((q, n), (out, n)), (), ws)
    arr = _array_type(Part, max(len(parts), 1))(*parts)
    _check(load().fdkv_decode_parts(ctypes.byref(d), int(batch), len(parts), ctypes.cast(arr, ctypes.c_void_p),
                                    None if tail is None else ctypes.byref(tail), int(layer), _dev(q), _dev(out),
                                    ctypes.c_float(sm_scale), _dev(ws), int(ws.numel() * ws.element_size()),
                                    _stream(stream)), "fdkv_decode_parts")
