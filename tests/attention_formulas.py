"""Rotary positions and attention in float64 on the host, written from their definitions, and bounds on the rounding of their fp32
evaluation.  u = 2^-24; HALF: half a unit in the last place of a type relative to the value."""
import numpy as np

from token_formulas import HALF, U32 as U  # noqa: F401


def angles(positions, turns):
    """Radians [N, pairs], |a| <= pi, of whole positions and 64-bit fractions of a turn, in Python's integers."""
    out = np.zeros((len(positions), len(turns)))
    for n, p in enumerate(positions):
        for i, t in enumerate(turns):
            x = int(p) * int(t) % 2 ** 64
            out[n, i] = (x - 2 ** 64 if x >= 2 ** 63 else x) / 2 ** 64 * 2 * np.pi
    return out


def rotate(x, positions, turns, interleaved, magnitude, inverse=False):
    """x [N, H, D] turned, and a bound on its evaluation before the result is rounded: cosine and sine are off by 3 u and their product with the
    magnitude rounds (4 u), two products and a sum of the results by 3 u of their size."""
    a = angles(positions, turns)[:, None, :]
    c, s = magnitude * np.cos(a), magnitude * np.sin(a) * (-1 if inverse else 1)
    h = len(turns)
    i, j = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
    y, e = x.copy(), np.zeros_like(x)
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    e[..., i] = e[..., j] = 7 * U * abs(magnitude) * (np.abs(x[..., i]) + np.abs(x[..., j]))
    return y, e


def attend(q, k, v, scale, half):
    """Of one head, q [S, D], k, v [T, D]: the result with a bound, p, and a relative bound on p.

    A score is a sum of D products, off by (D + 2) u of the sum of their magnitudes, times a scale that is rounded twice; the exponential's argument
    is a difference of two such numbers (4 u of the largest), itself good to 4 u.  The weights' errors count in numerator and denominator; the
    weights are rounded to the operands' type (half), the sums over T keys add (T + 8) u."""
    S, T = len(q), len(k)
    if T == 0:
        return dict(out=np.zeros_like(q), e=np.zeros_like(q), p=np.zeros((S, 0)), rel=np.zeros((S, 1)), L=np.full((S, 1), np.inf))
    with np.errstate(invalid="ignore", over="ignore"):
        z = scale * (q @ k.T)
        mag = scale * (np.abs(q) @ np.abs(k).T)
    there = z > -np.inf
    top = np.where(there, z, -np.inf).max(1, keepdims=True)
    none = top == -np.inf
    top = np.where(none, 0, top)
    w = np.where(there, np.exp(np.where(there, z - top, 0)), 0.0)
    l = w.sum(1, keepdims=True)
    p = w / np.where(none, 1, l)
    dz = np.where(there & (p > 0), (q.shape[1] + 6) * U * np.where(np.isfinite(mag), mag, 0) + 4 * U * (np.abs(np.where(there, z, 0)) + np.abs(top)), 0).max(1, keepdims=True)
    rel = np.expm1(dz) + 4 * U
    L = np.where(none, np.inf, (top + np.log(np.where(none, 1, l))) / np.log(2))
    out = p @ v
    e = (2 * rel + half + (T + 8) * U) * (p @ np.abs(v))
    return dict(out=out, e=e, p=p, rel=rel, L=L)


def attend_gradients(q, k, v, g, scale, f, half, stored):
    """(dq, dk, dv), each with a bound before it is rounded.  f: of attend; half: of the operands' type; stored: half a unit of the type that the
    result was kept in, which the backward pass reads."""
    S, T, D = len(q), len(k), q.shape[1]
    if T == 0 or S == 0:
        return [(np.zeros_like(x), np.zeros_like(x)) for x in (q, k, v)]
    p, a = f["p"], np.abs
    Lf = np.where(np.isfinite(f["L"]), f["L"], 0)
    rel = 2 * f["rel"] + 4 * U + 2 * U * a(Lf)
    dp, delta = g @ v.T, (g * f["out"]).sum(1, keepdims=True)
    eo = f["e"] + stored * (a(f["out"]) + f["e"])
    ed = (D + 2) * U * (a(g) @ a(v).T) + (a(g) * eo).sum(1, keepdims=True) + (D + 2) * U * (a(g) * (a(f["out"]) + eo)).sum(1, keepdims=True)
    dz = p * (dp - delta)
    ez = p * ed * (1 + rel) + a(dz) * (rel + 3 * U)
    ez = ez + half * (a(dz) + ez)
    ep = p * (rel + half * (1 + rel))
    dq, dk, dv = scale * (dz @ k), scale * (dz.T @ q), p.T @ g
    eq = scale * (ez @ a(k) + (T + 4) * U * ((a(dz) + ez) @ a(k)))
    ek = scale * (ez.T @ a(q) + (S + 4) * U * ((a(dz) + ez).T @ a(q)))
    ev = ep.T @ a(g) + (S + 4) * U * ((p + ep).T @ a(g))
    return [(dq, eq), (dk, ek), (dv, ev)]
