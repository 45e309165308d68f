"""The verification step around the accept test: cache plan, rotary positions, attention over the paged cache, the logits'
adjustments.  Thin ctypes wrappers of ``ciar_cache_plan``, ``ciar_rotary``, ``ciar_paged_attention`` and
``ciar_adjust_logits`` (``include/ciar.h`` has their formulas and rules): checks of types and shapes, output tensors, the call.

A step of a serving loop, all of it enqueued without waiting for the GPU::

    o = cache_plan(lengths, new, held, ring, ring_state, table, tokens, page_size=16, kept=accept_len)
    rotary(q, k, o["positions"], inv_freq, v=v, k_cache=kc, v_cache=vc, slots=o["slots"])
    a = paged_attention(q, kc, vc, table, o["cu_new"], o["kv_len"], max_new, max_len)
    y = adjust_logits(logits, params, history=..., drafted=ids, allowed=..., allowed_row=...)
    verify(draft, y["logits"], ids, u_accept, u_resample, params)
"""
from __future__ import annotations

import ctypes
import math

import torch

from .binding import CIAR_BF16, CIAR_F32, Params, _check, _ptr, _stream, lib

ATOM = 16                                                         # tokens of one head that lie together in the cache


class _RotaryParams(ctypes.Structure):
    """Mirror of ``struct ciar_rotary_params``."""
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in (
        "dtype", "q_heads", "kv_heads", "head_dim", "rotary_dim", "interleaved", "inverse")] + [
        ("magnitude", ctypes.c_double), ("page_size", ctypes.c_int32), ("reserved", ctypes.c_int32)] + [
        (n, ctypes.c_int64) for n in ("cache_pages", "q_stride", "q_head_stride", "k_stride", "k_head_stride", "v_stride",
                                      "v_head_stride", "q_out_stride", "q_out_head_stride", "k_out_stride",
                                      "k_out_head_stride")]


class _AttentionParams(ctypes.Structure):
    """Mirror of ``struct ciar_attention_params``."""
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in (
        "q_heads", "kv_heads", "head_dim", "page_size", "table_width", "max_new", "max_len")] + [
        ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)] + [
        (n, ctypes.c_int64) for n in ("table_stride", "cache_pages", "q_stride", "q_head_stride", "out_stride",
                                      "out_head_stride")]


class _Adjustments(ctypes.Structure):
    """Mirror of ``struct ciar_adjustments``."""
    _fields_ = [("struct_size", ctypes.c_uint32), ("mask_rows", ctypes.c_int32)] + [
        (n, ctypes.c_int64 if n in ("history_len", "bias_len", "allowed_stride") else ctypes.c_void_p) for n in (
            "history_start", "history", "history_len", "prompt_len", "drafted", "repetition", "presence", "frequency",
            "bias_start", "bias_ids", "bias_values", "bias_len", "allowed", "allowed_stride", "allowed_row")]


_ROTARY_SIZE, _ATTENTION_SIZE = ctypes.sizeof(_RotaryParams), ctypes.sizeof(_AttentionParams)
_ADJUST_SIZE = ctypes.sizeof(_Adjustments)
_I32, _I64, _F32, _F64, _U8, _BF16 = torch.int32, torch.int64, torch.float32, torch.float64, torch.uint8, torch.bfloat16


def _list(t, name: str, dtype, n: int):
    """A contiguous list of ``n`` values on the GPU."""
    if t.dtype is not dtype or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} entries, got {t.dtype} {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError("all tensors must live on the GPU")
    return t.data_ptr()


def _any_list(t, name: str, dtype):
    if t is None:
        return None
    return _list(t, name, dtype, t.numel())


def _table(t, name: str):
    """An int32 matrix with unit stride along its rows."""
    if t.dtype is not _I32 or t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{name} must be a 2-D int32 tensor with unit stride along its rows")
    if not t.is_cuda:
        raise ValueError("all tensors must live on the GPU")
    return t.data_ptr()


def _row_stride(t) -> int:
    """Elements between rows (a single row's stride means nothing: its length)."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _heads(t, name: str, dtype, T: int, D: int):
    """A [T, heads, D] tensor whose heads' dimensions are consecutive."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 3 or t.shape[0] != T or t.shape[2] != D or (t.stride(2) != 1 and D > 1):
        raise ValueError(f"{name} must be [{T}, heads, {D}] with unit stride along the last dimension, got {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError("all tensors must live on the GPU")
    return t.data_ptr()


def cache_shapes(pages: int, kv_heads: int, head_dim: int, page_size: int):
    """Shapes of the bfloat16 key and value caches."""
    atoms = page_size // ATOM
    return (pages, kv_heads, atoms, head_dim // 8, ATOM, 8), (pages, kv_heads, atoms, 2, head_dim, 8)


def _cache(k_cache, v_cache):
    """Checks the two caches; returns (pages, kv_heads, page_size, head_dim)."""
    s = k_cache.shape
    if k_cache.dtype is not _BF16 or v_cache.dtype is not _BF16:
        raise TypeError("k_cache and v_cache must be bfloat16")
    if len(s) != 6 or s[4] != ATOM or s[5] != 8 or v_cache.shape != (s[0], s[1], s[2], 2, 8 * s[3], 8):
        raise ValueError("k_cache must be [pages, kv_heads, page_size / 16, head_dim / 8, 16, 8] and v_cache "
                         f"[pages, kv_heads, page_size / 16, 2, head_dim, 8], got {tuple(s)} and {tuple(v_cache.shape)}")
    if not (k_cache.is_contiguous() and v_cache.is_contiguous()):
        raise ValueError("k_cache and v_cache must be contiguous")
    if not (k_cache.is_cuda and v_cache.is_cuda):
        raise ValueError("all tensors must live on the GPU")
    return s[0], s[1], s[2] * ATOM, s[3] * 8


def cache_plan(lengths, new, held, ring, ring_state, table, tokens: int, *, page_size: int, kept=None, stream=None,
               out: dict | None = None) -> dict:
    """``ciar_cache_plan``: pages, slots and positions of the next new tokens of every request; ``table`` and ``ring`` are
    updated in place.  ``lengths``, ``new``, ``held``, ``kept`` int32 [R], ``ring`` int32 [pages], ``ring_state`` int64 [2],
    ``table`` int32 [R, width]; ``tokens``: places for new tokens in this step.  Returns lengths, kv_len, held int32 [R],
    cu_new int32 [R + 1], granted uint8 [R], ring_state int64 [2] and slots, positions, requests int32 [tokens]; ``out`` may
    carry preallocated tensors under the same names."""
    R, tokens = lengths.shape[0], int(tokens)
    ins = (_list(lengths, "lengths", _I32, R), None if kept is None else _list(kept, "kept", _I32, R),
           _list(new, "new", _I32, R), _list(held, "held", _I32, R))
    rp, sp = _any_list(ring, "ring", _I32), _list(ring_state, "ring_state", _I64, 2)
    tp = _table(table, "table")
    if table.shape[0] != R:
        raise ValueError(f"table must have {R} rows, got {table.shape[0]}")
    o, ptrs = dict(out) if out else {}, []
    for name, dtype, n in (("lengths", _I32, R), ("kv_len", _I32, R), ("cu_new", _I32, R + 1), ("held", _I32, R),
                           ("granted", _U8, R), ("ring_state", _I64, 2), ("slots", _I32, tokens),
                           ("positions", _I32, tokens), ("requests", _I32, tokens)):
        t = o.get(name)
        if t is None:
            t = o[name] = torch.empty(n, dtype=dtype, device=lengths.device)
        ptrs.append(_list(t, f"out[{name!r}]", dtype, n))
    _check(lib().ciar_cache_plan(*ins, R, rp, ring.numel(), sp, tp, table.shape[1], _row_stride(table), int(page_size), tokens,
                                 *ptrs, _stream(stream)))
    return o


def rotary(q, k, positions, inv_freq, *, layout: str = "half", inverse: bool = False, magnitude: float = 1.0, v=None,
           k_cache=None, v_cache=None, slots=None, stream=None, out: dict | None = None) -> dict:
    """``ciar_rotary``: ``q`` [T, heads, D] and ``k`` [T, kv_heads, D] (float32 or bfloat16, any strides between tokens and
    heads) turned by ``positions`` int32 [T] times ``inv_freq`` float64 [n / 2], the first n dimensions of a head.  ``layout``:
    "half" pairs dimension p with p + n / 2, "interleaved" 2 p with 2 p + 1.  ``inverse`` turns back, which is the gradient:
    of the turned tensors' gradients it makes those of q and k.  With ``v``, ``k_cache``, ``v_cache`` and ``slots`` int32 [T]
    (bfloat16) the turned keys and the values go into the cache.  Returns q, and k without a cache; ``out`` may carry them."""
    if layout not in ("half", "interleaved"):
        raise ValueError(f"layout must be 'half' or 'interleaved', got {layout!r}")
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q and k must be [T, heads, D]")
    dtype, (T, Hq, D), Hk = q.dtype, q.shape, k.shape[1]
    if dtype is not _BF16 and dtype is not _F32:
        raise TypeError(f"q must be float32 or bfloat16, got {dtype}")
    qp, kp, vp = _heads(q, "q", dtype, T, D), _heads(k, "k", dtype, T, D), None
    o = dict(out) if out else {}
    qo = o.get("q")
    if qo is None:
        qo = o["q"] = torch.empty((T, Hq, D), dtype=dtype, device=q.device)
    qop, kop, kcp, vcp, slp = _heads(qo, "out['q']", dtype, T, D), None, None, None, None
    if qo.shape[1] != Hq:
        raise ValueError(f"out['q'] must have {Hq} heads")
    pages = page = 0
    vs, ks = (0, 0, 0), (0, 0, 0)
    if k_cache is not None or v_cache is not None or slots is not None:
        if k_cache is None or v_cache is None or slots is None or v is None:
            raise ValueError("v, k_cache, v_cache and slots go together")
        if o.pop("k", None) is not None:
            raise ValueError("out['k'] is not written where a cache is given")
        pages, heads, page, dim = _cache(k_cache, v_cache)
        if heads != Hk or dim != D:
            raise ValueError(f"the cache has {heads} heads of {dim}, k has {Hk} of {D}")
        vp, slp = _heads(v, "v", dtype, T, D), _list(slots, "slots", _I32, T)
        if v.shape[1] != Hk:
            raise ValueError(f"v must have {Hk} heads")
        kcp, vcp, vs = k_cache.data_ptr(), v_cache.data_ptr(), v.stride()
    else:
        if v is not None:
            raise ValueError("v is given without a cache")
        ko = o.get("k")
        if ko is None:
            ko = o["k"] = torch.empty((T, Hk, D), dtype=dtype, device=q.device)
        kop, ks = _heads(ko, "out['k']", dtype, T, D), ko.stride()
        if ko.shape[1] != Hk:
            raise ValueError(f"out['k'] must have {Hk} heads")
    pp, fp = _list(positions, "positions", _I32, T), _any_list(inv_freq, "inv_freq", _F64)
    a, b, c = q.stride(), k.stride(), qo.stride()
    cp = _RotaryParams(_ROTARY_SIZE, CIAR_F32 if dtype is _F32 else CIAR_BF16, Hq, Hk, D, 2 * inv_freq.shape[0],
                       1 if layout == "interleaved" else 0, 1 if inverse else 0, magnitude, page, 0, pages, a[0], a[1], b[0], b[1],
                       vs[0], vs[1], c[0], c[1], ks[0], ks[1])
    _check(lib().ciar_rotary(qp, kp, vp, pp, fp, T, ctypes.byref(cp), qop, kop, kcp, vcp, slp, _stream(stream)))
    return o


def paged_attention(q, k_cache, v_cache, table, cu_new, kv_len, max_new: int, max_len: int, *, scale: float | None = None,
                    stream=None, out: dict | None = None, workspace=None) -> dict:
    """``ciar_paged_attention``: the new tokens ``q`` [T, heads, D] (bfloat16) of R requests over the cache.  ``table`` int32
    [R, width], ``cu_new`` int32 [R + 1], ``kv_len`` int32 [R]; no request has more than ``max_new`` new tokens and
    ``max_len`` tokens in the cache.  ``scale`` defaults to 1 / sqrt(D).  Returns out [T, heads, D] bfloat16 and lse
    [T, heads] float32; ``out`` may carry them."""
    pages, Hk, page, D = _cache(k_cache, v_cache)
    if q.dim() != 3:
        raise ValueError("q must be [T, heads, D]")
    T, Hq, R = q.shape[0], q.shape[1], table.shape[0]
    qp, tp = _heads(q, "q", _BF16, T, D), _table(table, "table")
    cu, kl = _list(cu_new, "cu_new", _I32, R + 1), _list(kv_len, "kv_len", _I32, R)
    o = dict(out) if out else {}
    y, lse = o.get("out"), o.get("lse")
    if y is None:
        y = o["out"] = torch.empty((T, Hq, D), dtype=_BF16, device=q.device)
    if lse is None:
        lse = o["lse"] = torch.empty((T, Hq), dtype=_F32, device=q.device)
    yp = _heads(y, "out['out']", _BF16, T, D)
    if y.shape[1] != Hq or lse.shape != (T, Hq) or lse.dtype is not _F32 or not lse.is_contiguous() or not lse.is_cuda:
        raise ValueError(f"out['out'] must be [{T}, {Hq}, {D}] and out['lse'] a contiguous float32 [{T}, {Hq}] on the GPU")
    a, b = q.stride(), y.stride()
    cp = _AttentionParams(_ATTENTION_SIZE, Hq, Hk, D, page, table.shape[1], int(max_new), int(max_len),
                          1.0 / math.sqrt(D) if scale is None else scale, 0, _row_stride(table), pages, a[0], a[1], b[0], b[1])
    ref, L = ctypes.byref(cp), lib()
    wp, wsb = None, 0
    if workspace is None:
        wsb = L.ciar_attention_workspace_bytes(R, T, ref)
        if wsb:
            workspace = torch.empty(wsb, dtype=_U8, device=q.device)
            wp = workspace.data_ptr()
    else:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the GPU")
        wp, wsb = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(L.ciar_paged_attention(qp, k_cache.data_ptr(), v_cache.data_ptr(), tp, cu, kl, R, T, ref, yp, lse.data_ptr(), wp, wsb,
                                  _stream(stream)))
    return o


def attention_workspace_bytes(q, k_cache, table, max_new: int, max_len: int) -> int:
    """Bytes of workspace ``paged_attention`` asks for (0: none)."""
    s = k_cache.shape
    cp = _AttentionParams(_ATTENTION_SIZE, q.shape[1], s[1], 8 * s[3], ATOM * s[2], table.shape[1], int(max_new), int(max_len),
                          1.0, 0, _row_stride(table), s[0], 0, 0, 0, 0)
    return int(lib().ciar_attention_workspace_bytes(table.shape[0], q.shape[0], ctypes.byref(cp)))


def adjust_logits(logits, params: Params, *, history_start=None, history=None, prompt_len=None, drafted=None, repetition=None,
                  presence=None, frequency=None, bias_start=None, bias_ids=None, bias_values=None, allowed=None,
                  allowed_row=None, vocab: int | None = None, stream=None, out: dict | None = None, workspace=None) -> dict:
    """``ciar_adjust_logits``: penalties, biases and grammar masks on the rows of ``logits``, ``params.window`` rows to a request.
    ``history`` int32 with ``history_start`` int64 [W + 1] (its offsets), ``prompt_len`` int32 [W], ``drafted`` int32 [N],
    ``repetition`` / ``presence`` / ``frequency`` float32 [W]; ``bias_ids`` int32 ascending and ``bias_values`` float32 with
    ``bias_start`` int64 [W + 1]; ``allowed`` int32 [masks, words] bits with ``allowed_row`` int32 [N] (negative: no mask).  Each
    group may be left out.  Returns logits (``out["logits"]`` may be ``logits`` itself) and left int32 [N], the finite logits left
    in each row."""
    cp = params.to_c(logits, vocab)
    if not logits.is_cuda:
        raise ValueError("all tensors must live on the GPU")
    N = logits.shape[0]
    K = cp.window
    W = (N + K - 1) // K if K > 0 else 0
    o = dict(out) if out else {}
    y, left = o.get("logits"), o.get("left")
    if y is None:
        # (rows laid out like the input's: a padded row stays readable and aligned)
        y = o["logits"] = torch.empty((N, cp.row_stride), dtype=logits.dtype, device=logits.device)[:, :cp.vocab]
    elif y.dtype is not logits.dtype or y.dim() != 2 or y.shape[0] != N or y.shape[1] < cp.vocab or y.stride(1) != 1 or not y.is_cuda:
        raise ValueError("out['logits'] must match logits in dtype and rows, with unit stride along the vocabulary")
    if left is None:
        left = o["left"] = torch.empty(N, dtype=_I32, device=logits.device)
    lp = _list(left, "out['left']", _I32, N)

    def per(t, name, dtype, n):
        return None if t is None else _list(t, name, dtype, n)

    a = _Adjustments(_ADJUST_SIZE, 0, per(history_start, "history_start", _I64, W + 1), _any_list(history, "history", _I32),
                     0 if history is None else history.numel(), per(prompt_len, "prompt_len", _I32, W),
                     per(drafted, "drafted", _I32, N), per(repetition, "repetition", _F32, W), per(presence, "presence", _F32, W),
                     per(frequency, "frequency", _F32, W), per(bias_start, "bias_start", _I64, W + 1),
                     _any_list(bias_ids, "bias_ids", _I32), _any_list(bias_values, "bias_values", _F32),
                     0 if bias_ids is None else bias_ids.numel(), None, 0, per(allowed_row, "allowed_row", _I32, N))
    if bias_ids is not None and bias_values is not None and bias_values.shape[0] != bias_ids.shape[0]:
        raise ValueError("bias_ids and bias_values must have the same number of entries")
    if allowed is not None:
        a.allowed, a.mask_rows, a.allowed_stride = _table(allowed, "allowed"), allowed.shape[0], _row_stride(allowed)
        if allowed.shape[1] * 32 < cp.vocab:
            raise ValueError(f"allowed must have {(cp.vocab + 31) // 32} words a row, got {allowed.shape[1]}")
    wp, wsb = None, 0
    if workspace is None:
        wsb = (8 * N + 255) // 256 * 256
        workspace = torch.empty(wsb, dtype=_U8, device=logits.device)
        wp = workspace.data_ptr()
    else:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the GPU")
        wp, wsb = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(lib().ciar_adjust_logits(logits.data_ptr(), N, ctypes.byref(cp), ctypes.byref(a), y.data_ptr(),
                                    max(y.stride(0), cp.vocab) if N <= 1 else y.stride(0), lp, wp, wsb, _stream(stream)))
    return o


def adjust_workspace_bytes(N: int) -> int:
    """Bytes of workspace ``adjust_logits`` asks for."""
    return (8 * int(N) + 255) // 256 * 256
