"""Operators on sequences of tokens (antdt.h: antdt_token_*, antdt_gated_*, antdt_dropout) on torch tensors.

Every call works on torch's current stream.  Results go to `out` (or the other named outputs) where
given, else to new tensors; a workspace that is not given comes from torch's allocator.  Nothing here is registered
with autograd: a backward pass is a call of its own, results do not require a gradient whatever the operands do, and what
is written through `out` (and the other named outputs) does not count as an in-place change of that tensor.
"""
from __future__ import annotations

import ctypes as C
from functools import lru_cache
from typing import NamedTuple, Optional, Tuple

import torch

from .binding import BF16, F32, AntdtError, DropoutSpec, _raw_stream, lib

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

    def _on(self, device: int):
        """The spec, with a step, for a call on `device`, which reads it."""
        if self.step.get_device() != device:
            raise ValueError(f"Dropout: step is on {self.step.device}, the operands on device {device}")
        return self._ref


def _check(rc: int):
    if rc:
        raise AntdtError(rc, lib.antdt_last_error(None).decode())


# Handle of torch's current stream of a device.  Its default stream has the same handle on every device, and kernels on it
# go to the current one: a call whose operands are on another makes that the current one first.
_stream = _raw_stream or (lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _rows(t: torch.Tensor, name: str, rows: int, cols: int, dtype: torch.dtype, device: int) -> int:
    """Leading dimension of a matrix argument (a single row's stride means nothing), after the checks that the C boundary
    cannot make."""
    s, shape = t.stride(), t.shape
    if len(s) != 2 or shape[0] != rows or shape[1] != cols:
        raise ValueError(f"{name}: shape {tuple(shape)}, expected ({rows}, {cols})")
    if t.dtype is not dtype:
        raise ValueError(f"{name}: {t.dtype}, expected {dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name}: on {t.device}, expected device {device}")
    if s[1] != 1 and cols > 1:
        raise ValueError(f"{name}: columns of a row must be neighbours")
    return s[0] if rows > 1 else cols


def _matrix(t: torch.Tensor, name: str) -> Tuple[int, int, int, int]:
    """(rows, columns, leading dimension, device) of a call's first matrix."""
    shape, s = t.shape, t.stride()
    if len(shape) != 2 or t.dtype not in _DTYPES:
        raise ValueError(f"{name}: a matrix of float32 or bfloat16, not {tuple(shape)} of {t.dtype}")
    device = t.get_device()
    if device < 0:
        raise ValueError(f"{name}: not on the device")
    rows, cols = shape
    if s[1] != 1 and cols > 1:
        raise ValueError(f"{name}: columns of a row must be neighbours")
    return rows, cols, s[0] if rows > 1 else cols, device


def _vector(t: torch.Tensor, name: str, n: int, dtype: torch.dtype, device: int) -> int:
    shape = t.shape
    if len(shape) != 1 or shape[0] != n or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous elements of {dtype} on device {device}")
    return t.data_ptr()


def _new(shape: Tuple[int, ...], dtype: torch.dtype, like: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor (empty_strided costs about half of empty)."""
    return torch.empty_strided(shape, (shape[1], 1) if len(shape) == 2 else (1,), dtype=dtype, device=like.device)


def _workspace(workspace: Optional[torch.Tensor], nbytes: int,
               like: torch.Tensor) -> Tuple[Optional[torch.Tensor], Optional[int], int]:
    """(tensor, address, bytes) of the caller's workspace, or of a new one; torch's blocks start at multiples of 512 bytes.
    The caller holds on to the tensor until the kernels are enqueued: from then on torch's allocator hands a block that
    is given back on in the order of the stream, before that to any thread."""
    if workspace is None:
        if nbytes == 0:
            return None, None, 0
        workspace = _new((nbytes,), torch.uint8, like)
    elif workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError("workspace: contiguous, on the operands' device")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


@lru_cache(maxsize=4096)
def _bytes(call: str, *sizes: int) -> int:
    n = C.c_size_t()
    _check(getattr(lib, call)(*sizes, C.byref(n)))
    return n.value


def dropout(x: torch.Tensor, drop: Dropout, residual: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """residual + dropout(x), or dropout(x).  `out` may be x or residual.  The gradient of x is dropout(gradient, drop)."""
    rows, cols, ldx, dev = _matrix(x, "x")
    if dev != _current_device():
        with torch.cuda.device(dev):
            return dropout(x, drop, residual, out)
    dt = x.dtype
    if out is None:
        out = _new((rows, cols), dt, x)
    ldr, rp = 0, None
    if residual is not None:
        ldr, rp = _rows(residual, "residual", rows, cols, dt, dev), residual.data_ptr()
    ldo = _rows(out, "out", rows, cols, dt, dev)
    spec = drop._ref if drop.step is None else drop._on(dev)
    _check(lib.antdt_dropout(x.data_ptr(), ldx, rp, ldr, rows, cols, _DTYPES[dt], spec, out.data_ptr(), ldo,
                             _stream(dev)))
    return out


def token_lookup(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, dropout: Optional[Dropout] = None,
                 out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """scale * dropout(table[tokens]); tokens outside the table are padding and give zeros."""
    V, D, ldt, dev = _matrix(table, "table")
    if dev != _current_device():
        with torch.cuda.device(dev):
            return token_lookup(table, tokens, scale, dropout, out, out_dtype)
    N = tokens.numel()
    tp = _vector(tokens, "tokens", N, torch.int32, dev)
    if out is None:
        out = _new((N, D), out_dtype or table.dtype, table)
    odt = out.dtype if out_dtype is None else out_dtype
    if odt not in _DTYPES:
        raise ValueError(f"out: {odt}")
    ldo = _rows(out, "out", N, D, odt, dev)
    spec = None if dropout is None else dropout._ref if dropout.step is None else dropout._on(dev)
    _check(lib.antdt_token_lookup(table.data_ptr(), ldt, V, D, _DTYPES[table.dtype], tp, N, scale, spec, out.data_ptr(),
                                  ldo, _DTYPES[odt], _stream(dev)))
    return out


def token_gradient(dy: torch.Tensor, tokens: torch.Tensor, rows: int, scale: float = 1.0,
                   dropout: Optional[Dropout] = None, out: Optional[torch.Tensor] = None, accumulate: bool = False,
                   workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient (fp32 [rows, D]) of the table of token_lookup from that of its output.  With `accumulate` the sums are
    added to `out`, whose other rows are not touched."""
    N, D, ldd, dev = _matrix(dy, "dy")
    if dev != _current_device():
        with torch.cuda.device(dev):
            return token_gradient(dy, tokens, rows, scale, dropout, out, accumulate, workspace)
    tp = _vector(tokens, "tokens", N, torch.int32, dev)
    if out is None:
        if accumulate:
            raise ValueError("token_gradient: accumulate needs out")
        out = _new((rows, D), torch.float32, dy)
    ldg = _rows(out, "out", rows, D, torch.float32, dev)
    held, ws, n = _workspace(workspace, _bytes("antdt_token_gradient_bytes", N, rows, D), dy)
    spec = None if dropout is None else dropout._ref if dropout.step is None else dropout._on(dev)
    _check(lib.antdt_token_gradient(dy.data_ptr(), ldd, _DTYPES[dy.dtype], tp, N, scale, spec, out.data_ptr(), ldg,
                                    rows, D, 1 if accumulate else 0, ws, n, _stream(dev)))
    return out


def _width(w: torch.Tensor) -> int:
    """Columns of what should be a matrix, to check it by."""
    return w.shape[1] if len(w.shape) == 2 else 0


def gated_saved(x: torch.Tensor, wg: torch.Tensor) -> torch.Tensor:
    """A buffer for what gated_forward leaves to gated_backward."""
    N, K, _, dev = _matrix(x, "x")
    H = _width(wg)
    _rows(wg, "wg", K, H, x.dtype, dev)
    return _new((_bytes("antdt_gated_saved_bytes", N, H, _DTYPES[x.dtype]),), torch.uint8, x)


def _saved(saved: torch.Tensor, N: int, H: int, dtype: torch.dtype, device: int) -> int:
    if saved.get_device() != device or not saved.is_contiguous() or (
            saved.numel() * saved.element_size() < _bytes("antdt_gated_saved_bytes", N, H, _DTYPES[dtype])):
        raise ValueError("saved: the buffer of gated_saved")
    return saved.data_ptr()


def _weights(wg: torch.Tensor, wu: torch.Tensor, K: int, dt: torch.dtype, dev: int) -> Tuple[int, int]:
    """(H, leading dimension) of the two weight matrices."""
    H = _width(wg)
    ldw = _rows(wg, "wg", K, H, dt, dev)
    if _rows(wu, "wu", K, H, dt, dev) != ldw:
        raise ValueError("wg and wu: one leading dimension")
    return H, ldw


def gated_forward(x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, act: str = "silu",
                  out: Optional[torch.Tensor] = None, saved: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """act(x Wg) * (x Wu), weights [in, out].  `saved` (see gated_saved) is filled for gated_backward."""
    if act not in ACTS:
        raise ValueError(f"act: one of {', '.join(ACTS)}")
    N, K, ldx, dev = _matrix(x, "x")
    if dev != _current_device():
        with torch.cuda.device(dev):
            return gated_forward(x, wg, wu, act, out, saved, workspace)
    dt = x.dtype
    H, ldw = _weights(wg, wu, K, dt, dev)
    if out is None:
        out = _new((N, H), dt, x)
    ldh = _rows(out, "out", N, H, dt, dev)
    held, ws, n = _workspace(workspace, _bytes("antdt_gated_forward_bytes", N, K, H, _DTYPES[dt]), x)
    _check(lib.antdt_gated_forward(x.data_ptr(), ldx, wg.data_ptr(), wu.data_ptr(), ldw, N, K, H, _DTYPES[dt],
                                   ACTS[act], out.data_ptr(), ldh,
                                   None if saved is None else _saved(saved, N, H, dt, dev), ws, n, _stream(dev)))
    return out


def gated_backward(dh: torch.Tensor, x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, saved: torch.Tensor,
                   dx: Optional[torch.Tensor] = None, dwg: Optional[torch.Tensor] = None,
                   dwu: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """(dx, dwg, dwu) of gated_forward from the gradient of its result.  In bf16 the gradients of both projections, operands of
    the products, are rounded to bf16 too."""
    N, K, ldx, dev = _matrix(x, "x")
    if dev != _current_device():
        with torch.cuda.device(dev):
            return gated_backward(dh, x, wg, wu, saved, dx, dwg, dwu, workspace)
    dt = x.dtype
    H, ldw = _weights(wg, wu, K, dt, dev)
    ldd = _rows(dh, "dh", N, H, dt, dev)
    dx = _new((N, K), dt, x) if dx is None else dx
    dwg = _new((K, H), dt, x) if dwg is None else dwg
    dwu = _new((K, H), dt, x) if dwu is None else dwu
    lddx, lddw = _rows(dx, "dx", N, K, dt, dev), _rows(dwg, "dwg", K, H, dt, dev)
    if _rows(dwu, "dwu", K, H, dt, dev) != lddw:
        raise ValueError("dwg and dwu: one leading dimension")
    held, ws, n = _workspace(workspace, _bytes("antdt_gated_backward_bytes", N, K, H, _DTYPES[dt]), x)
    _check(lib.antdt_gated_backward(dh.data_ptr(), ldd, x.data_ptr(), ldx, wg.data_ptr(), wu.data_ptr(), ldw, N, K, H,
                                    _DTYPES[dt], _saved(saved, N, H, dt, dev), dx.data_ptr(), lddx, dwg.data_ptr(),
                                    dwu.data_ptr(), lddw, ws, n, _stream(dev)))
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
    N, V, ld, dev = _matrix(logits, "logits")
    if dev != _current_device():
        with torch.cuda.device(dev):
            return token_logprobs(logits, tokens, top, workspace)
    n = _bytes("antdt_token_logprobs_bytes", N, V, top)
    f32, given, k = torch.float32, tokens is not None, top if top > 0 else 0
    tp = _vector(tokens, "tokens", N, torch.int32, dev) if given else None
    # One block of memory for all results and, behind them, the workspace: an allocation costs as much as two views.
    words = [4 * N, N, N if given else 0, k * N, k * N]
    front = (sum(words) + 63) // 64 * 64
    own = workspace is None
    buf = _new((front + (n // 4 if own else 0),), f32, logits)
    held, ws, n = (buf, buf.data_ptr() + 4 * front, n) if own else _workspace(workspace, n, logits)
    stats, entropy, logp, top_logp, top_index, _ = torch.unsafe_split_with_sizes(buf, words + [buf.shape[0] - sum(words)])
    at = buf.data_ptr()
    sp, ep, lp = at, at + 16 * N, at + 20 * N
    tl = at + 4 * (words[0] + words[1] + words[2])
    ti = tl + 4 * k * N
    stats, logp = stats.view(N, 4), logp if given else None
    if k:
        top_logp, top_index = top_logp.view(N, k), top_index.view(torch.int32).view(N, k)
    else:
        top_logp = top_index = None
    _check(lib.antdt_token_logprobs(logits.data_ptr(), ld, N, V, _DTYPES[logits.dtype], tp, lp if given else None, ep,
                                    sp, top, tl, ti, ws, n, _stream(dev)))
    return LogProbs(logp, entropy, stats, top_logp, top_index)


def token_logprobs_gradient(logits: torch.Tensor, tokens: Optional[torch.Tensor], stats: torch.Tensor,
                            d_logp: Optional[torch.Tensor], d_entropy: Optional[torch.Tensor] = None,
                            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of the logits from those of token_logprobs' logp and entropy.  `out` may be the logits themselves."""
    N, V, ld, dev = _matrix(logits, "logits")
    if dev != _current_device():
        with torch.cuda.device(dev):
            return token_logprobs_gradient(logits, tokens, stats, d_logp, d_entropy, out)
    dt, f32 = logits.dtype, torch.float32
    if _rows(stats, "stats", N, 4, f32, dev) != 4:
        raise ValueError("stats: as token_logprobs left them")
    if out is None:
        out = _new((N, V), dt, logits)
    ldd = _rows(out, "out", N, V, dt, dev)
    tp = None if tokens is None else _vector(tokens, "tokens", N, torch.int32, dev)
    dl = None if d_logp is None else _vector(d_logp, "d_logp", N, f32, dev)
    dh = None if d_entropy is None else _vector(d_entropy, "d_entropy", N, f32, dev)
    _check(lib.antdt_token_logprobs_gradient(logits.data_ptr(), ld, N, V, _DTYPES[dt], tp, stats.data_ptr(), dl, dh,
                                             out.data_ptr(), ldd, _stream(dev)))
    return out
