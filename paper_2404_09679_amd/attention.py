"""Attention over a user's history (antdt.h: antdt_rotary, antdt_cache_*, antdt_cross_attention*) on torch tensors, with the conventions of
tokens.py: torch's current stream, results in `out` (or the other named outputs) where given, nothing registered with autograd.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from .binding import RotarySpec, lib
from .tokens import _DTYPES, _bytes, _check, _current_device, _stream, _vector, _workspace


class Rotary:
    """Rotary positions of a head's first `dim` columns: pair i turns by base^(-2 i / dim) radians a position.  For a context `factor` times as long
    as the `original` one pairs are slowed by the factor: all of them, or, with `low` and `high`, fully those of fewer than `low` turns in the
    original context, not at all those of more than `high`.  What is turned is multiplied by `magnitude`.  `turns`: the frequencies, on `device`."""

    def __init__(self, dim: int, base: float = 10000.0, interleaved: bool = False, factor: float = 1.0, original: float = 0.0, low: float = 0.0,
                 high: float = 0.0, magnitude: float = 1.0, device="cuda"):
        turns = (C.c_uint64 * max(dim // 2, 1))()
        _check(lib.antdt_rotary_turns(dim, base, factor, original, low, high, turns))
        self.dim, self.interleaved, self.magnitude = dim, bool(interleaved), magnitude
        self.turns = torch.tensor([t for t in turns], dtype=torch.int64, device=device)      # (below 2^62)
        self._spec = RotarySpec(dim, int(self.interleaved), magnitude, self.turns.data_ptr())
        self._ref = C.byref(self._spec)

    def _on(self, device: int):
        """The spec for a call on `device`, which reads the frequencies."""
        if self.turns.get_device() != device:
            raise ValueError(f"Rotary: on {self.turns.device}, the operands on device {device}")
        return self._ref


def _first(t: torch.Tensor, name: str, dims: int):
    """(shape, strides but the columns', dtype, device) of a call's first heads."""
    shape, s, device = t.shape, t.stride(), t.get_device()
    if len(shape) != dims or t.dtype not in _DTYPES or device < 0 or (s[-1] != 1 and shape[-1] > 1):
        raise ValueError(f"{name}: {dims} dimensions of float32 or bfloat16 on the device, columns neighbours, not {tuple(shape)} (strides {s}) "
                         f"of {t.dtype} on {t.device}")
    return shape, s[:-1], t.dtype, device


def _heads(t: torch.Tensor, name: str, shape: Tuple[int, ...], dtype: torch.dtype, device: int) -> Tuple[int, ...]:
    """Strides of another heads argument but its columns', after the checks that the C boundary cannot make."""
    s = t.stride()
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or (s[-1] != 1 and shape[-1] > 1):
        raise ValueError(f"{name}: heads of neighbouring columns, {tuple(shape)} of {dtype} on device {device}, not {tuple(t.shape)} "
                         f"(strides {s}) of {t.dtype} on {t.device}")
    return s[:-1]


def _new(shape: Tuple[int, ...], like: torch.Tensor, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    return like.new_empty(shape, dtype=dtype)


def _lengths(t: Optional[torch.Tensor], name: str, n: int, device: int) -> Optional[int]:
    return None if t is None else _vector(t, name, n, torch.int32, device)


def _scale(scale: Optional[float], D: int) -> float:
    return max(D, 1) ** -0.5 if scale is None else scale


def _turned(x: torch.Tensor, positions: torch.Tensor, rotary: Rotary, inverse: int, out: Optional[torch.Tensor]) -> torch.Tensor:
    shape, ldx, dt, dev = _first(x, "x", 3)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return _turned(x, positions, rotary, inverse, out)
    N, H, D = shape
    if out is None:
        out = _new(shape, x)
    ldy = _heads(out, "out", shape, dt, dev)
    _check(lib.antdt_rotary(x.data_ptr(), *ldx, N, H, D, _DTYPES[dt], _vector(positions, "positions", N, torch.int32, dev), rotary._on(dev),
                            inverse, out.data_ptr(), *ldy, _stream(dev)))
    return out


def rotary(x: torch.Tensor, positions: torch.Tensor, rotary: Rotary, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [N, H, D] turned by its rows' positions (int32 [N]).  `out` may be x."""
    return _turned(x, positions, rotary, 0, out)


def rotary_gradient(dy: torch.Tensor, positions: torch.Tensor, rotary: Rotary, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of rotary's x from that of its result.  `out` may be dy."""
    return _turned(dy, positions, rotary, 1, out)


def _cache(k_cache: torch.Tensor, v_cache: torch.Tensor, dtype: torch.dtype, device: int):
    """(shape, strides) of the two caches."""
    shape, s, dt, dev = _first(k_cache, "k_cache", 4)
    if dt is not dtype or dev != device:
        raise ValueError(f"k_cache: {dt} on device {dev}, the tokens {dtype} on device {device}")
    if _heads(v_cache, "v_cache", shape, dtype, device) != s:
        raise ValueError("k_cache and v_cache: one layout")
    return shape, s


def _table(table: torch.Tensor, device: int) -> Tuple[int, int, int]:
    """(sequences, columns, leading dimension) of a cache's table."""
    shape, s = table.shape, table.stride()
    if len(shape) != 2 or table.dtype is not torch.int32 or table.get_device() != device or (s[1] != 1 and shape[1] > 1):
        raise ValueError(f"table: int32 [sequences, pages of one], neighbours in a row, on device {device}")
    B, W = shape
    return B, W, s[0] if B > 1 else W


def cache_append(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
                 offsets: Optional[torch.Tensor] = None, rotary: Optional[Rotary] = None, q: Optional[torch.Tensor] = None,
                 q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """New tokens' k and v [N, heads, D] to the caches [pages, page size, heads, D], k turned by its positions.  Tokens offsets[b] .. offsets[b + 1] - 1 (or
    token b) are the last ones of sequence b, whose lengths[b] counts them in and whose pages are table[b].  Returns the queries `q` [N, q heads, D] of the
    same tokens turned likewise (to `q_out`, which may be q), None without."""
    shape, ldk, dt, dev = _first(k, "k", 3)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return cache_append(k, v, k_cache, v_cache, table, lengths, offsets, rotary, q, q_out)
    N, H, D = shape
    ldv = _heads(v, "v", shape, dt, dev)
    (pages, page, CH, CD), ldc = _cache(k_cache, v_cache, dt, dev)
    if (CH, CD) != (H, D):
        raise ValueError(f"k_cache: heads {CH} x {CD}, k has {H} x {D}")
    B, W, ldt = _table(table, dev)
    HQ, ldq, ldo, qp, op = 0, (0, 0), (0, 0), None, None
    if q is not None:
        HQ = q.shape[1] if len(q.shape) == 3 else 0
        ldq = _heads(q, "q", (N, HQ, D), dt, dev)
        if q_out is None:
            q_out = _new((N, HQ, D), q)
        ldo = _heads(q_out, "q_out", (N, HQ, D), dt, dev)
        qp, op = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out: without q")
    _check(lib.antdt_cache_append(qp, *ldq, op, *ldo, k.data_ptr(), *ldk, v.data_ptr(), *ldv, N, HQ, H, D, _DTYPES[dt],
                                  None if rotary is None else rotary._on(dev), k_cache.data_ptr(), v_cache.data_ptr(), *ldc, pages, page,
                                  table.data_ptr(), ldt, B, W, _vector(lengths, "lengths", B, torch.int32, dev),
                                  _lengths(offsets, "offsets", B + 1, dev), _stream(dev)))
    return q_out


def cache_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
                    scale: Optional[float] = None, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """softmax(scale q k^T) v of one token of each sequence, q [B, q heads, D], over the lengths[b] tokens that the caches hold of it
    (see cache_append).  scale: D^-1/2 unless given."""
    shape, ldq, dt, dev = _first(q, "q", 3)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return cache_attention(q, k_cache, v_cache, table, lengths, scale, out, workspace)
    B, HQ, D = shape
    (pages, page, H, CD), ldc = _cache(k_cache, v_cache, dt, dev)
    TB, W, ldt = _table(table, dev)
    if CD != D or TB != B:
        raise ValueError(f"q: {B} sequences of heads of {D}, the cache has {TB} of {CD}")
    if out is None:
        out = _new(shape, q)
    ldo = _heads(out, "out", shape, dt, dev)
    held, ws, n = _workspace(workspace, _bytes("antdt_cache_attention_bytes", B, HQ, H, D, _DTYPES[dt]), q)
    _check(lib.antdt_cache_attention(q.data_ptr(), *ldq, k_cache.data_ptr(), v_cache.data_ptr(), *ldc, pages, page, table.data_ptr(), ldt, B, W,
                                     _vector(lengths, "lengths", B, torch.int32, dev), HQ, H, D, _DTYPES[dt],
                                     _scale(scale, D), out.data_ptr(), *ldo, ws, n, _stream(dev)))
    return out


def cross_attention_stats(q: torch.Tensor) -> torch.Tensor:
    """A buffer (fp32 [B, heads, S]) for what cross_attention leaves to cross_attention_backward, for queries [B, S, heads, D]."""
    _first(q, "q", 4)
    B, S, H, _ = q.shape
    return _new((B, H, S), q, torch.float32)


def _stats(stats: torch.Tensor, B: int, S: int, H: int, device: int) -> int:
    if stats.shape != (B, H, S) or stats.dtype is not torch.float32 or stats.get_device() != device or not stats.is_contiguous():
        raise ValueError("stats: the buffer of cross_attention_stats")
    return stats.data_ptr()


def _sides(q: torch.Tensor, k: torch.Tensor):
    """(shape of the queries and of the keys, their strides, dtype, device)."""
    qs, ldq, dt, dev = _first(q, "q", 4)
    ks = k.shape
    if len(ks) != 4 or ks[0] != qs[0] or ks[3] != qs[3]:
        raise ValueError(f"k: shape {tuple(ks)}, expected ({qs[0]}, keys, heads, {qs[3]})")
    return qs, ks, ldq, _heads(k, "k", ks, dt, dev), dt, dev


def cross_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_lengths: Optional[torch.Tensor] = None,
                    k_lengths: Optional[torch.Tensor] = None, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                    stats: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """softmax(scale q k^T) v of queries [B, S, q heads, D] over keys and values [B, T, heads, D].  q_lengths and k_lengths (int32 [B]): rows that an
    entry has; queries behind them have zeros.  scale: D^-1/2 unless given.  `stats` (see cross_attention_stats) is filled for cross_attention_backward."""
    qs, ks, ldq, ldk, dt, dev = _sides(q, k)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return cross_attention(q, k, v, q_lengths, k_lengths, scale, out, stats, workspace)
    (B, S, HQ, D), (_, T, H, _) = qs, ks
    ldv = _heads(v, "v", ks, dt, dev)
    if out is None:
        out = _new(qs, q)
    ldo = _heads(out, "out", qs, dt, dev)
    held, ws, n = _workspace(workspace, _bytes("antdt_cross_attention_bytes", B, S, T, HQ, H, D, _DTYPES[dt]), q)
    _check(lib.antdt_cross_attention(q.data_ptr(), *ldq, k.data_ptr(), *ldk, v.data_ptr(), *ldv, B, S, T, HQ, H, D, _DTYPES[dt],
                                     _lengths(q_lengths, "q_lengths", B, dev), _lengths(k_lengths, "k_lengths", B, dev),
                                     _scale(scale, D), out.data_ptr(), *ldo,
                                     None if stats is None else _stats(stats, B, S, HQ, dev), ws, n, _stream(dev)))
    return out


def cross_attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, stats: torch.Tensor,
                             q_lengths: Optional[torch.Tensor] = None, k_lengths: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                             dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None, dv: Optional[torch.Tensor] = None,
                             workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dq, dk, dv) of cross_attention from the gradient of its result; the other arguments as it was given and left them.  In bf16 the gradients
    of the scores, operands of the products, are rounded to bf16 too."""
    qs, ks, ldq, ldk, dt, dev = _sides(q, k)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return cross_attention_backward(dout, q, k, v, out, stats, q_lengths, k_lengths, scale, dq, dk, dv, workspace)
    (B, S, HQ, D), (_, T, H, _) = qs, ks
    ldv, ldo, ldg = _heads(v, "v", ks, dt, dev), _heads(out, "out", qs, dt, dev), _heads(dout, "dout", qs, dt, dev)
    dq = _new(qs, q) if dq is None else dq
    dk = _new(ks, q) if dk is None else dk
    dv = _new(ks, q) if dv is None else dv
    lddq, lddk, lddv = _heads(dq, "dq", qs, dt, dev), _heads(dk, "dk", ks, dt, dev), _heads(dv, "dv", ks, dt, dev)
    held, ws, n = _workspace(workspace, _bytes("antdt_cross_attention_backward_bytes", B, S, T, HQ, H, D, _DTYPES[dt]), q)
    _check(lib.antdt_cross_attention_backward(dout.data_ptr(), *ldg, q.data_ptr(), *ldq, k.data_ptr(), *ldk, v.data_ptr(), *ldv, out.data_ptr(),
                                              *ldo, _stats(stats, B, S, HQ, dev), B, S, T, HQ, H, D, _DTYPES[dt],
                                              _lengths(q_lengths, "q_lengths", B, dev), _lengths(k_lengths, "k_lengths", B, dev),
                                              _scale(scale, D), dq.data_ptr(), *lddq, dk.data_ptr(), *lddk, dv.data_ptr(),
                                              *lddv, ws, n, _stream(dev)))
    return dq, dk, dv
