"""Operators on sequences of tokens (antdt.h: antdt_token_*, antdt_gated_*, antdt_dropout) on torch tensors.

Every call works on torch's current stream.  Results go to `out` (or the other named outputs) where
given, else to new tensors; a workspace that is not given comes from torch's allocator.  Nothing here is registered
with autograd: a backward pass is a call of its own.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Tuple

import torch

from .binding import BF16, F32, AntdtError, DropoutSpec, _stream, lib

ACTS = {"silu": 0, "gelu": 1, "relu": 2, "sigmoid": 3}
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


class Dropout:
    """One dropout of a training step: the probability, the seed, which of the step's dropouts it is (`call`) and, for
    captured graphs, a device tensor (int64, one element) that is added to the seed when the kernel runs."""

    def __init__(self, p: float, seed: int, call: int = 0, step: Optional[torch.Tensor] = None):
        if step is not None and (step.dtype != torch.int64 or step.numel() != 1 or not step.is_cuda):
            raise ValueError("Dropout: step is one int64 on the device")
        self.p, self.seed, self.call, self.step = p, seed, call, step
        self._spec = DropoutSpec(p, call & 0xFFFFFFFF, seed & 0xFFFFFFFFFFFFFFFF,
                                 None if step is None else step.data_ptr())
        self._ref = C.byref(self._spec)


def _check(rc: int):
    if rc:
        raise AntdtError(rc, lib.antdt_last_error(None).decode())


def _rows(t: torch.Tensor, name: str, rows: Optional[int] = None, cols: Optional[int] = None,
          dtype: Optional[torch.dtype] = None, device: Optional[torch.device] = None) -> int:
    """Leading dimension of a matrix argument, after the checks that the C boundary cannot make."""
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name}: a matrix on the device")
    if t.dtype not in _DTYPES or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name}: dtype {t.dtype}")
    r, c = t.shape
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected ({rows}, {cols})")
    if device is not None and t.device != device:
        raise ValueError(f"{name}: on {t.device}, expected {device}")
    s0, s1 = t.stride()
    if s1 != 1 and c > 1:
        raise ValueError(f"{name}: columns of a row must be neighbours")
    return s0 if r > 1 else max(s0, c)


def _vector(t: torch.Tensor, name: str, n: int, dtype: torch.dtype, device: torch.device) -> int:
    if t.dtype != dtype or t.device != device or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous elements of {dtype} on {device}")
    return t.data_ptr()


def _workspace(workspace: Optional[torch.Tensor], nbytes: int, device: torch.device) -> Tuple[Optional[int], int]:
    """(address, bytes) of the caller's workspace, or of a new one; torch's blocks start at multiples of 512 bytes."""
    if workspace is None:
        if nbytes == 0:
            return None, 0
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    elif workspace.device != device or not workspace.is_contiguous():
        raise ValueError("workspace: contiguous, on the operands' device")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _bytes(call, *args) -> int:
    size = C.c_size_t()
    _check(call(*args, C.byref(size)))
    return size.value


def dropout(x: torch.Tensor, drop: Dropout, residual: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """residual + dropout(x), or dropout(x).  `out` may be x or residual.  The gradient of x is dropout(gradient, drop)."""
    ldx = _rows(x, "x")
    rows, cols = x.shape
    if out is None:
        out = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
    ldr = _rows(residual, "residual", rows, cols, x.dtype, x.device) if residual is not None else 0
    ldo = _rows(out, "out", rows, cols, x.dtype, x.device)
    _check(lib.antdt_dropout(x.data_ptr(), ldx, None if residual is None else residual.data_ptr(), ldr, rows, cols,
                             _DTYPES[x.dtype], drop._ref, out.data_ptr(), ldo, _stream()))
    return out


def token_lookup(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, dropout: Optional[Dropout] = None,
                 out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """scale * dropout(table[tokens]); tokens outside the table are padding and give zeros."""
    ldt = _rows(table, "table")
    (V, D), N = table.shape, tokens.numel()
    tp = _vector(tokens, "tokens", N, torch.int32, table.device)
    if out is None:
        out = torch.empty((N, D), dtype=out_dtype or table.dtype, device=table.device)
    ldo = _rows(out, "out", N, D, out_dtype, table.device)
    _check(lib.antdt_token_lookup(table.data_ptr(), ldt, V, D, _DTYPES[table.dtype], tp, N, scale,
                                  None if dropout is None else dropout._ref, out.data_ptr(), ldo, _DTYPES[out.dtype],
                                  _stream()))
    return out


def token_gradient(dy: torch.Tensor, tokens: torch.Tensor, rows: int, scale: float = 1.0,
                   dropout: Optional[Dropout] = None, out: Optional[torch.Tensor] = None, accumulate: bool = False,
                   workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient (fp32 [rows, D]) of the table of token_lookup from that of its output.  With `accumulate` the sums are
    added to `out`, whose other rows are not touched."""
    ldd = _rows(dy, "dy")
    N, D = dy.shape
    tp = _vector(tokens, "tokens", N, torch.int32, dy.device)
    if out is None:
        if accumulate:
            raise ValueError("token_gradient: accumulate needs out")
        out = torch.empty((rows, D), dtype=torch.float32, device=dy.device)
    ldg = _rows(out, "out", rows, D, torch.float32, dy.device)
    ws, n = _workspace(workspace, _bytes(lib.antdt_token_gradient_bytes, N, rows, D), dy.device)
    _check(lib.antdt_token_gradient(dy.data_ptr(), ldd, _DTYPES[dy.dtype], tp, N, scale,
                                    None if dropout is None else dropout._ref, out.data_ptr(), ldg, rows, D,
                                    1 if accumulate else 0, ws, n, _stream()))
    return out


def gated_saved(x: torch.Tensor, wg: torch.Tensor) -> torch.Tensor:
    """A buffer for what gated_forward leaves to gated_backward."""
    n = _bytes(lib.antdt_gated_saved_bytes, x.shape[0], wg.shape[1], _DTYPES[x.dtype])
    return torch.empty(n, dtype=torch.uint8, device=x.device)


def _saved(saved: torch.Tensor, N: int, H: int, x: torch.Tensor) -> int:
    if saved.device != x.device or not saved.is_contiguous() or (
            saved.numel() * saved.element_size() < _bytes(lib.antdt_gated_saved_bytes, N, H, _DTYPES[x.dtype])):
        raise ValueError("saved: the buffer of gated_saved")
    return saved.data_ptr()


def gated_forward(x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, act: str = "silu",
                  out: Optional[torch.Tensor] = None, saved: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """act(x Wg) * (x Wu), weights [in, out].  `saved` (see gated_saved) is filled for gated_backward."""
    if act not in ACTS:
        raise ValueError(f"act: one of {', '.join(ACTS)}")
    ldx = _rows(x, "x")
    (N, K), dev, dt = x.shape, x.device, x.dtype
    H = wg.shape[-1]
    ldw = _rows(wg, "wg", K, H, dt, dev)
    if _rows(wu, "wu", K, H, dt, dev) != ldw:
        raise ValueError("wg and wu: one leading dimension")
    if out is None:
        out = torch.empty((N, H), dtype=dt, device=dev)
    ldh = _rows(out, "out", N, H, dt, dev)
    ws, n = _workspace(workspace, _bytes(lib.antdt_gated_forward_bytes, N, K, H, _DTYPES[dt]), dev)
    _check(lib.antdt_gated_forward(x.data_ptr(), ldx, wg.data_ptr(), wu.data_ptr(), ldw, N, K, H, _DTYPES[dt], ACTS[act],
                                   out.data_ptr(), ldh, None if saved is None else _saved(saved, N, H, x), ws, n,
                                   _stream()))
    return out


def gated_backward(dh: torch.Tensor, x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, saved: torch.Tensor,
                   dx: Optional[torch.Tensor] = None, dwg: Optional[torch.Tensor] = None,
                   dwu: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """(dx, dwg, dwu) of gated_forward from the gradient of its result."""
    ldx = _rows(x, "x")
    (N, K), dev, dt = x.shape, x.device, x.dtype
    H = wg.shape[-1]
    ldw = _rows(wg, "wg", K, H, dt, dev)
    if _rows(wu, "wu", K, H, dt, dev) != ldw:
        raise ValueError("wg and wu: one leading dimension")
    ldd = _rows(dh, "dh", N, H, dt, dev)
    dx = torch.empty((N, K), dtype=dt, device=dev) if dx is None else dx
    dwg = torch.empty((K, H), dtype=dt, device=dev) if dwg is None else dwg
    dwu = torch.empty((K, H), dtype=dt, device=dev) if dwu is None else dwu
    lddx, lddw = _rows(dx, "dx", N, K, dt, dev), _rows(dwg, "dwg", K, H, dt, dev)
    if _rows(dwu, "dwu", K, H, dt, dev) != lddw:
        raise ValueError("dwg and dwu: one leading dimension")
    ws, n = _workspace(workspace, _bytes(lib.antdt_gated_backward_bytes, N, K, H, _DTYPES[dt]), dev)
    _check(lib.antdt_gated_backward(dh.data_ptr(), ldd, x.data_ptr(), ldx, wg.data_ptr(), wu.data_ptr(), ldw, N, K, H,
                                    _DTYPES[dt], _saved(saved, N, H, x), dx.data_ptr(), lddx, dwg.data_ptr(),
                                    dwu.data_ptr(), lddw, ws, n, _stream()))
    return dx, dwg, dwu


class LogProbs(NamedTuple):
    logp: Optional[torch.Tensor]       # fp32 [N], None without tokens
    entropy: torch.Tensor              # fp32 [N]
    stats: torch.Tensor                # fp32 [N, 4], for token_logprobs_gradient
    top_logp: Optional[torch.Tensor]   # fp32 [N, top], descending
    top_index: Optional[torch.Tensor]  # int32 [N, top]


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top: int = 0,
                   workspace: Optional[torch.Tensor] = None) -> LogProbs:
    """Log probabilities of `tokens` under softmax(logits), the rows' entropies and their `top` largest log
    probabilities with their columns."""
    ld = _rows(logits, "logits")
    (N, V), dev = logits.shape, logits.device
    tp = None if tokens is None else _vector(tokens, "tokens", N, torch.int32, dev)
    # one allocation: stats first, they are read 16 bytes at a time
    buf = torch.empty(N * (6 + 2 * max(top, 0)), dtype=torch.float32, device=dev)
    stats, logp, entropy = buf[:4 * N].view(N, 4), buf[4 * N:5 * N], buf[5 * N:6 * N]
    tops = (buf[6 * N:(6 + top) * N].view(N, top), buf[(6 + top) * N:].view(torch.int32).view(N, top)) if top > 0 else (None, None)
    ws, n = _workspace(workspace, _bytes(lib.antdt_token_logprobs_bytes, N, V, top), dev)
    _check(lib.antdt_token_logprobs(logits.data_ptr(), ld, N, V, _DTYPES[logits.dtype], tp,
                                    None if tp is None else logp.data_ptr(), entropy.data_ptr(), stats.data_ptr(), top,
                                    None if top == 0 else tops[0].data_ptr(), None if top == 0 else tops[1].data_ptr(),
                                    ws, n, _stream()))
    return LogProbs(None if tp is None else logp, entropy, stats, *tops)


def token_logprobs_gradient(logits: torch.Tensor, tokens: Optional[torch.Tensor], stats: torch.Tensor,
                            d_logp: Optional[torch.Tensor], d_entropy: Optional[torch.Tensor] = None,
                            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of the logits from those of token_logprobs' logp and entropy.  `out` may be the logits themselves."""
    ld = _rows(logits, "logits")
    (N, V), dev = logits.shape, logits.device
    if stats.dtype != torch.float32 or tuple(stats.shape) != (N, 4) or not stats.is_contiguous() or stats.device != dev:
        raise ValueError("stats: as token_logprobs left them")
    if out is None:
        out = torch.empty((N, V), dtype=logits.dtype, device=dev)
    ldd = _rows(out, "out", N, V, logits.dtype, dev)
    _check(lib.antdt_token_logprobs_gradient(
        logits.data_ptr(), ld, N, V, _DTYPES[logits.dtype],
        None if tokens is None else _vector(tokens, "tokens", N, torch.int32, dev), stats.data_ptr(),
        None if d_logp is None else _vector(d_logp, "d_logp", N, torch.float32, dev),
        None if d_entropy is None else _vector(d_entropy, "d_entropy", N, torch.float32, dev), out.data_ptr(), ldd,
        _stream()))
    return out
