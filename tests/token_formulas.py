"""The operators on sequences of tokens in float64 on the host, written from their definitions, and bounds on the
rounding of their fp32 evaluation.  Half a unit in the last place of a type relative to the value: HALF."""
import math

import numpy as np

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
U32 = 2.0 ** -24

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85


def philox(counter, key):
    """Philox4x32-10 of one counter (four words) in Python's integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = M0 * c[0], M1 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + W0) & 0xFFFFFFFF, (k[1] + W1) & 0xFFFFFFFF]
    return c


def lots(rows, cols, seed, call):
    """16-bit lots [rows, cols] of a dropout."""
    m = np.uint64(0xFFFFFFFF)
    groups = (cols + 7) // 8
    r = np.repeat(np.arange(rows, dtype=np.uint64), groups)
    c = [np.tile(np.arange(groups, dtype=np.uint64), rows), r & m, r >> np.uint64(32), np.full(r.shape, call, np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        a, b = np.uint64(M0) * c[0], np.uint64(M1) * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & m, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & m]
        k0, k1 = (k0 + W0) & 0xFFFFFFFF, (k1 + W1) & 0xFFFFFFFF
    w = np.stack(c, 1)
    return np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 2).reshape(rows, groups * 8)[:, :cols].astype(np.int64)


def keep(rows, cols, p, seed, call):
    """Factors of a dropout."""
    t = int(math.floor(float(np.float32(p)) * 65536 + 0.5))
    if t == 0:
        return np.ones((rows, cols))
    if t == 65536:
        return np.zeros((rows, cols))
    return (lots(rows, cols, seed, call) >= t) * (65536.0 / (65536 - t))


def lookup(table, tokens, scale, m):
    there = (tokens >= 0) & (tokens < table.shape[0])
    out = np.zeros((tokens.size, table.shape[1]))
    out[there] = table[tokens[there]] * m[there] * scale
    return out


def table_gradient(dy, tokens, rows, scale, m):
    """The gradient, and for every element the sum of its terms' magnitudes and how many there are."""
    there = (tokens >= 0) & (tokens < rows)
    d = dy[there] * m[there] * scale
    g, mag, n = np.zeros((rows, dy.shape[1])), np.zeros((rows, dy.shape[1])), np.zeros(rows)
    np.add.at(g, tokens[there], d)
    np.add.at(mag, tokens[there], np.abs(d))
    np.add.at(n, tokens[there], 1)
    return g, mag, n


_erf = np.vectorize(math.erf, otypes=[np.float64])


def activation(act, g):
    if act == "silu":
        s = 1 / (1 + np.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if act == "gelu":
        c = 0.5 * (1 + _erf(g / math.sqrt(2)))
        return g * c, c + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if act == "relu":
        return np.maximum(g, 0), (g > 0) * 1.0
    s = 1 / (1 + np.exp(-g))
    return s, s * (1 - s)


def gated(x, wg, wu, act, half):
    """h, and a bound on the error of an evaluation with fp32 sums and the result rounded once.

    A sum of K products in any order is off by at most K u times the sum of the magnitudes (u = 2^-24; the products of
    fp32 operands round as well).  All activations here have slopes below 1.2 and change their slope by less than 1 per
    unit; their evaluation is taken to be off by 8 + |g| units (an exponential of an argument rounded before)."""
    K = x.shape[1]
    g, u = x @ wg, x @ wu
    p, r = activation(act, g)
    eg, eu = (K + 2) * U32 * (np.abs(x) @ np.abs(wg)), (K + 2) * U32 * (np.abs(x) @ np.abs(wu))
    jump = (act == "relu") * (np.abs(g) <= eg)           # the slope may go either way there
    ep = 1.2 * eg + (8 + np.abs(g)) * U32 * (np.abs(p) + np.abs(g) * (act == "gelu"))
    er = 1.0 * eg * (act != "relu") + (8 + np.abs(g)) * 2 * U32 * (1 + np.abs(g)) + jump
    eh = ep * (np.abs(u) + eu) + np.abs(p) * eu + 2 * U32 * np.abs(p * u)
    return dict(g=g, u=u, p=p, r=r, ep=ep, er=er, eu=eu, h=p * u, eh=eh + half * (np.abs(p * u) + eh))


def gated_gradients(x, wg, wu, dh, f, half):
    """(dx, dwg, dwu) and bounds: dg and du are rounded to the operands' type, then products and sums as above."""
    dg, du = dh * f["u"] * f["r"], dh * f["p"]
    adh = np.abs(dh)
    eg = adh * (f["er"] * (np.abs(f["u"]) + f["eu"]) + np.abs(f["r"]) * f["eu"]) + 3 * U32 * np.abs(dg)
    eu = adh * f["ep"] + 2 * U32 * np.abs(du)
    eg, eu = eg + half * (np.abs(dg) + eg), eu + half * (np.abs(du) + eu)

    def product(parts):
        v = sum(a @ b for a, ea, b in parts)
        n = sum(a.shape[1] for a, ea, b in parts)
        e = sum(ea @ np.abs(b) + (n + 2) * U32 * ((np.abs(a) + ea) @ np.abs(b)) for a, ea, b in parts)
        return v, e + half * (np.abs(v) + e)

    def product_left(a, d, ed):
        v = a.T @ d
        e = np.abs(a).T @ ed + (a.shape[0] + 2) * U32 * (np.abs(a).T @ (np.abs(d) + ed))
        return v, e + half * (np.abs(v) + e)

    return product([(dg, eg, wg.T), (du, eu, wu.T)]), product_left(x, dg, eg), product_left(x, du, eu)


def logprobs(x, tokens, top):
    """logp, entropy, largest and log sum, top values and columns, all log probabilities."""
    N, V = x.shape
    m = x.max(1, keepdims=True)
    empty = (m == -np.inf)[:, 0]
    base = np.where(m == -np.inf, 0.0, m)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.exp(x - base)
        s = e.sum(1, keepdims=True)
        lp = np.where(empty[:, None], -np.inf, (x - base) - np.log(s))
        p = np.where(empty[:, None], 0.0, e / s)
        h = -np.where(p > 0, p * lp, 0.0).sum(1)
    there = (tokens >= 0) & (tokens < V)
    logp = np.zeros(N)
    logp[there] = lp[np.flatnonzero(there), tokens[there]]
    order = np.argsort(-x, axis=1, kind="stable")[:, :top]
    return dict(logp=logp, entropy=h, lp=lp, p=p, empty=empty, there=there, log_s=np.log(np.maximum(s[:, 0], 1e-300)),
                top_logp=np.take_along_axis(lp, order, 1), top_index=order, depth=V / 256 + 64)


def logprobs_gradient(f, tokens, a, b):
    """d_logits, and a bound on the error of an fp32 evaluation (before it is rounded to its type)."""
    N, V = f["p"].shape
    hot = np.zeros((N, V))
    rows = np.flatnonzero(f["there"] & ~f["empty"])
    hot[rows, tokens[rows]] = 1
    a = np.where(f["there"], a, 0.0)[:, None]
    b = b[:, None]
    lp = np.where(f["p"] > 0, f["lp"], 0.0)
    h = f["entropy"][:, None]
    d = a * (hot - f["p"]) - b * f["p"] * (lp + h)
    rel = U32 * (f["depth"] + 4 * np.abs(lp))          # of p, and of log p + H absolutely
    e = np.abs(a) * (f["p"] * rel + 2 * U32) + np.abs(b) * f["p"] * (rel * (np.abs(lp) + np.abs(h) + 4)) + 4 * U32 * np.abs(d)
    return d, np.where(f["empty"][:, None], 0.0, e)
