"""The operators on sequences of tokens, as cases that can be timed and compared.

A case is one pass through one of them:

  lookup    rows of a table for a sequence of tokens, scaled, with dropout; when `train`, also the table's
            gradient from the gradient of the output
  dropout   dropout of a matrix, the mask formed from a counter, optionally added to a residual
  gated     h = act(x Wg) * (x Wu); when `train`, also the gradients of x, Wg and Wu from that of h
  logprobs  log probabilities of given tokens under rows of logits, with the entropy of each row and its `top`
            largest alternatives; when `train`, also the gradient of the logits

Where `own` is false, run() computes them from elementary torch operations in fp32.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------- the cases
def _lookup(dtype, rows, dim, tokens, train, p, zipf=1.1):
    return dict(op="lookup", dtype=dtype, rows=rows, dim=dim, tokens=tokens, train=train, p=p, zipf=zipf)


def _dropout(dtype, rows, cols, p, residual):
    return dict(op="dropout", dtype=dtype, rows=rows, cols=cols, p=p, residual=residual)


def _gated(dtype, tokens, width, hidden, act, train):
    return dict(op="gated", dtype=dtype, tokens=tokens, width=width, hidden=hidden, act=act, train=train)


def _logprobs(dtype, tokens, vocab, top, train, masked=False, entropy_grad=False):
    return dict(op="logprobs", dtype=dtype, tokens=tokens, vocab=vocab, top=top, train=train, masked=masked,
                entropy_grad=entropy_grad)


def listed():
    return [
        # answering: the last few items of one user's history, a table of the ranking model's size
        dict(name="lookup-serve", **_lookup("f32", 1_000_000, 32, 16, False, 0.0)),
        # a training batch of histories, frequent items far ahead of the others
        dict(name="lookup-train", **_lookup("bf16", 200_000, 256, 131_072, True, 0.1)),
        # a small fp32 model of odd width
        dict(name="lookup-train-odd", **_lookup("f32", 50_021, 100, 3001, True, 0.25, 1.05)),
        # dropout of a small layer's output
        dict(name="dropout-small", **_dropout("f32", 64, 250, 0.5, False)),
        # the residual branch of a large batch
        dict(name="dropout-residual", **_dropout("bf16", 65_536, 1024, 0.1, True)),
        # answering token by token
        dict(name="gated-token", **_gated("bf16", 1, 1024, 4096, "silu", False)),
        # a ragged training batch of a narrow block
        dict(name="gated-ragged", **_gated("bf16", 777, 520, 1400, "gelu", True)),
        # a large training batch of a wide block
        dict(name="gated-train", **_gated("bf16", 8192, 2048, 5632, "silu", True)),
        # fp32 throughout
        dict(name="gated-fp32", **_gated("f32", 1000, 512, 1024, "silu", True)),
        # the best items for one user, every row of a table a candidate
        dict(name="logprobs-answer", **_logprobs("f32", 1, 1_000_000, 10, False)),
        # the loss over a vocabulary and its gradient
        dict(name="logprobs-train", **_logprobs("bf16", 4096, 50_000, 0, True)),
        # a policy's log probabilities with an entropy bonus, items that are not allowed masked out
        dict(name="logprobs-masked", **_logprobs("f32", 257, 10_007, 5, True, True, True)),
    ]


def draw(rng):
    """One more case: an operator with its sizes and options drawn over the range of the listed ones."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["lookup", "dropout", "gated", "gated", "logprobs"])
    dtype = rng.choice(["f32", "bf16"])
    train = rng.random() < 0.6
    if op == "lookup":
        dim = rng.choice([16, 32, 64, 128, 256, log_int(9, 300)])
        return _lookup(dtype, log_int(1000, min(1_000_000, 51_200_000 // dim)), dim,
                       log_int(1, min(131_072, 33_554_432 // dim)), train, rng.choice([0.0, 0.1, 0.3]),
                       rng.choice([1.05, 1.1, 1.2]))
    if op == "dropout":
        cols = log_int(10, 4096)
        return _dropout(dtype, log_int(1, min(65_536, 67_108_864 // cols)), cols, rng.choice([0.05, 0.1, 0.5]),
                        rng.random() < 0.5)
    if op == "gated":
        width, hidden = 8 * log_int(8, 256), 8 * log_int(16, 704)
        most = 8192 if dtype == "bf16" else 1024
        return _gated(dtype, log_int(1, most), width, hidden, rng.choice(["silu", "gelu", "relu", "sigmoid"]), train)
    vocab = log_int(100, 1_000_000)
    return _logprobs(dtype, log_int(1, max(1, min(4096, 200_000_000 // vocab))), vocab, rng.choice([0, 1, 5, 10, 32]), train,
                     rng.random() < 0.4, rng.random() < 0.4)


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "lookup":
        N, D, V = case["tokens"], case["dim"], case["rows"]
        b = 4 * N + 2 * N * D * es
        if case["train"]:
            b += N * D * es + V * D * 4
        return {"bytes": b, "flops": N * D * (3 if case["train"] else 1)}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * es * (3 if case["residual"] else 2), "flops": 2 * n}
    if case["op"] == "gated":
        N, K, H = case["tokens"], case["width"], case["hidden"]
        b, f = (N * K + 2 * K * H + N * H) * es, 4 * N * K * H
        if case["train"]:
            b, f = b + (N * H + N * K + 2 * K * H) * es, 3 * f
        return {"bytes": b, "flops": f}
    N, V = case["tokens"], case["vocab"]
    b, f = N * V * es, 4 * N * V
    if case["train"]:
        b, f = 3 * b, 2 * f
    return {"bytes": b + N * (12 + 8 * case["top"]), "flops": f}


# ---------------------------------------------------------------------------- inputs
def _zipf_tokens(case, gen):
    """Tokens whose frequency falls with a power of the row's rank, ranks scattered over the rows; one in a hundred is
    padding."""
    V, N = case["rows"], case["tokens"]
    w = torch.arange(1, V + 1, device=DEV, dtype=torch.float64).pow(-case["zipf"])
    cdf = torch.cumsum(w, 0)
    u = torch.rand(N, device=DEV, dtype=torch.float64, generator=gen) * cdf[-1]
    rank = torch.searchsorted(cdf, u).clamp(max=V - 1)
    place = torch.randperm(V, device=DEV, generator=gen)
    t = place[rank].to(torch.int32)
    return torch.where(torch.rand(N, device=DEV, generator=gen) < 0.01, torch.full_like(t, -1), t)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device=DEV, generator=gen).mul_(std)

    s = dict(case=case, seed=seed)
    if case["op"] == "lookup":
        V, D, N = case["rows"], case["dim"], case["tokens"]
        s["table"] = ((torch.rand(V, D, device=DEV, generator=gen) * 2 - 1) * 0.05).to(dt)
        s["tokens"] = _zipf_tokens(case, gen)
        s["scale"] = math.sqrt(D)
        s["out"] = torch.empty(N, D, device=DEV, dtype=dt)
        if case["train"]:
            s["dy"] = normal(N, D, std=1e-2).to(dt)
            s["grad"] = torch.empty(V, D, device=DEV)
    elif case["op"] == "dropout":
        R, C = case["rows"], case["cols"]
        s["x"] = normal(R, C).to(dt)
        s["residual"] = normal(R, C).to(dt) if case["residual"] else None
        s["out"] = torch.empty(R, C, device=DEV, dtype=dt)
    elif case["op"] == "gated":
        N, K, H = case["tokens"], case["width"], case["hidden"]
        s["x"] = normal(N, K).to(dt)
        s["wg"], s["wu"] = normal(K, H, std=K ** -0.5).to(dt), normal(K, H, std=K ** -0.5).to(dt)
        s["h"] = torch.empty(N, H, device=DEV, dtype=dt)
        if case["train"]:
            s["dh"] = normal(N, H, std=1e-2).to(dt)
            s["dx"], s["dwg"], s["dwu"] = (torch.empty_like(s[k]) for k in ("x", "wg", "wu"))
    else:
        N, V = case["tokens"], case["vocab"]
        x = normal(N, V, std=2.0)
        t = torch.randint(0, V, (N,), device=DEV, generator=gen)
        x.scatter_add_(1, t[:, None], normal(N, 1).abs() * 4)   # the given token is often a likely one
        if case["masked"]:
            x.masked_fill_(torch.rand(N, V, device=DEV, generator=gen) < 0.3, -math.inf)
            if N > 3:
                x[N // 2] = -math.inf                            # nothing is allowed there
        t = torch.where(torch.rand(N, device=DEV, generator=gen) < 0.02, torch.full_like(t, -1), t)
        s["logits"], s["tokens"] = x.to(dt), t.to(torch.int32)
        if case["train"]:
            s["d_logp"] = normal(N, std=1.0 / N)
            s["d_entropy"] = normal(N, std=0.1 / N) if case["entropy_grad"] else None
            s["d_logits"] = torch.empty(N, V, device=DEV, dtype=dt)
    return s


# ---------------------------------------------------------------------------- plain forms
CALL = 3          # which of a step's dropouts it is


def _kept(rows, cols, p, seed):
    """Factors of the dropout, fp32 [rows, cols]: 0 or 65536 / (65536 - t), t = round(65536 p), where column c of row r is
    dropped when 16-bit lot c % 8 of Philox4x32-10 (counter (c / 8, r, r >> 32, call), key seed) is below t."""
    t = int(math.floor(p * 65536 + 0.5))
    if t == 0:
        return torch.ones(rows, cols, device=DEV)
    low = 0xFFFFFFFF
    r = torch.arange(rows, device=DEV)[:, None]
    c0 = torch.arange((cols + 7) // 8, device=DEV)[None, :].expand(rows, -1)
    c1, c2, c3 = (r & low).expand_as(c0), (r >> 32).expand_as(c0), torch.full_like(c0, CALL)
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    lots = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], dim=2)
    lots = lots.reshape(rows, -1)[:, :cols]
    return torch.where(lots >= t, 65536.0 / (65536 - t), 0.0).float()


def _act(name, g):
    """act(g) and its derivative."""
    if name == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    if name == "relu":
        return g.clamp(min=0), (g > 0).to(g.dtype)
    s = 1 / (1 + torch.exp(-g))
    return s, s * (1 - s)


def _plain_lookup(s, case):
    t = s["tokens"].long()
    there = ((t >= 0) & (t < case["rows"]))[:, None]
    m = _kept(case["tokens"], case["dim"], case["p"], s["seed"]) * s["scale"]
    row = t.clamp(0, case["rows"] - 1)
    out = {"out": torch.where(there, s["table"][row].float() * m, 0.0).to(s["table"].dtype)}
    if case["train"]:
        d = torch.where(there, s["dy"].float() * m, 0.0)
        out["grad"] = torch.zeros(case["rows"], case["dim"], device=DEV).index_add_(0, row, d)
    return out


def _plain_dropout(s, case):
    y = s["x"].float() * _kept(case["rows"], case["cols"], case["p"], s["seed"])
    if case["residual"]:
        y = s["residual"].float() + y
    return y.to(s["x"].dtype)


def _plain_gated(s, case):
    dt = s["x"].dtype
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    g, u = x @ wg, x @ wu
    a, da = _act(case["act"], g)
    out = {"h": (a * u).to(dt)}
    if case["train"]:
        dh = s["dh"].float()
        dg, du = dh * u * da, dh * a
        out |= {"dx": (dg @ wg.t() + du @ wu.t()).to(dt), "dwg": (x.t() @ dg).to(dt), "dwu": (x.t() @ du).to(dt)}
    return out


def _plain_logprobs(s, case):
    x = s["logits"].float()
    t = s["tokens"].long()
    given = (t >= 0) & (t < case["vocab"])
    m = x.amax(1, keepdim=True)
    d = x - torch.where(m == -math.inf, 0.0, m)             # rows without an allowed item: everything stays -inf
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    some = total > 0
    h = torch.where(some, log_total - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total, 0.0)
    logp = torch.where(some, d - log_total, -math.inf)
    out = {"logp": torch.where(given, logp.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0), "entropy": h[:, 0]}
    if case["top"]:
        # one whole number that orders by value, then by the lower index
        bits = (x + 0.0).view(torch.int32).long()
        key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF) - 1) * (1 << 32) + (
            (1 << 32) - 1 - torch.arange(case["vocab"], device=DEV))
        index = ((1 << 32) - 1) - (key.topk(case["top"], dim=1).values & 0xFFFFFFFF)
        out |= {"top_logp": logp.gather(1, index), "top_index": index.to(torch.int32)}
    if case["train"]:
        a = torch.where(given, s["d_logp"], 0.0)[:, None]
        p = torch.where(some, e / total, 0.0)
        dx = -a * p
        if case["entropy_grad"]:
            dx = dx - s["d_entropy"][:, None] * torch.where(p > 0, p * (logp + h), 0.0)
        some_given = torch.where(given[:, None] & some, a, 0.0)
        out["d_logits"] = dx.scatter_add_(1, t.clamp(min=0)[:, None], some_given).to(s["logits"].dtype)
    return out


# ---------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if not own:
        return {"lookup": _plain_lookup, "dropout": _plain_dropout, "gated": _plain_gated,
                "logprobs": _plain_logprobs}[case["op"]](s, case)
    import paper_2404_09679_amd as A

    if case["op"] == "lookup":
        drop = A.Dropout(case["p"], s["seed"], CALL) if case["p"] else None
        out = {"out": A.token_lookup(s["table"], s["tokens"], s["scale"], dropout=drop, out=s["out"])}
        if case["train"]:
            out["grad"] = A.token_gradient(s["dy"], s["tokens"], case["rows"], s["scale"], dropout=drop, out=s["grad"])
        return out
    if case["op"] == "dropout":
        return A.dropout(s["x"], A.Dropout(case["p"], s["seed"], CALL), residual=s["residual"], out=s["out"])
    if case["op"] == "gated":
        if not case["train"]:
            return {"h": A.gated_forward(s["x"], s["wg"], s["wu"], case["act"], out=s["h"])}
        saved = A.gated_saved(s["x"], s["wg"])
        h = A.gated_forward(s["x"], s["wg"], s["wu"], case["act"], out=s["h"], saved=saved)
        dx, dwg, dwu = A.gated_backward(s["dh"], s["x"], s["wg"], s["wu"], saved, dx=s["dx"], dwg=s["dwg"], dwu=s["dwu"])
        return {"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}
    r = A.token_logprobs(s["logits"], s["tokens"], top=case["top"])
    out = {"logp": r.logp, "entropy": r.entropy}
    if case["top"]:
        out |= {"top_logp": r.top_logp, "top_index": r.top_index}
    if case["train"]:
        out["d_logits"] = A.token_logprobs_gradient(s["logits"], s["tokens"], r.stats, s["d_logp"], s["d_entropy"],
                                                    out=s["d_logits"])
    return out


# ---------------------------------------------------------------------------- the definition in 64 bits
def _philox_lots(rows, cols, seed):
    """16-bit lots [rows, cols] on the host, in numpy's unsigned arithmetic."""
    mask = np.uint64(0xFFFFFFFF)
    group = np.arange((cols + 7) // 8, dtype=np.uint64)
    row = np.arange(rows, dtype=np.uint64)
    shape = (rows, group.size)
    ctr = [np.broadcast_to(group, shape), np.broadcast_to((row & mask)[:, None], shape),
           np.broadcast_to((row >> np.uint64(32))[:, None], shape), np.full(shape, CALL, np.uint64)]
    key = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for i in range(10):
        k = [np.uint64((key[0] + i * 0x9E3779B9) & 0xFFFFFFFF), np.uint64((key[1] + i * 0xBB67AE85) & 0xFFFFFFFF)]
        first, third = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ctr = [(third >> np.uint64(32)) ^ ctr[1] ^ k[0], third & mask, (first >> np.uint64(32)) ^ ctr[3] ^ k[1],
               first & mask]
    words = np.stack(ctr, axis=-1).astype("<u4")
    return np.ascontiguousarray(words).view("<u2").reshape(rows, -1)[:, :cols]


def _factors(rows, cols, p, seed):
    t = int(math.floor(p * 65536 + 0.5))
    if t == 0:
        return torch.ones(rows, cols, device=DEV, dtype=torch.float64)
    keep = torch.from_numpy(_philox_lots(rows, cols, seed) >= t).to(DEV)
    return keep.double() * (65536 / (65536 - t))


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "lookup":
        V, N, D = case["rows"], case["tokens"], case["dim"]
        tok = s["tokens"].cpu().numpy().astype(np.int64)
        at = torch.from_numpy(np.flatnonzero((tok >= 0) & (tok < V))).to(DEV)
        row = s["tokens"].to(torch.int64)[at]
        m = _factors(N, D, case["p"], seed)
        out = torch.zeros(N, D, device=DEV, dtype=f64)
        out[at] = s["table"].to(f64)[row] * m[at] * s["scale"]
        res = {"out": out}
        if case["train"]:
            grad = torch.zeros(V, D, device=DEV, dtype=f64)
            grad.index_put_((row,), s["dy"].to(f64)[at] * m[at] * s["scale"], accumulate=True)
            res["grad"] = grad
        return res
    if case["op"] == "dropout":
        y = s["x"].to(f64) * _factors(case["rows"], case["cols"], case["p"], seed)
        return y + s["residual"].to(f64) if case["residual"] else y
    if case["op"] == "gated":
        x, w = s["x"].to(f64), torch.cat([s["wg"], s["wu"]], 1).to(f64)
        z = torch.mm(x, w)
        g, u = z.chunk(2, dim=1)
        phi = {"silu": torch.sigmoid, "sigmoid": torch.sigmoid, "relu": lambda v: (v > 0).to(f64),
               "gelu": torch.special.ndtr}[case["act"]](g)
        gate = phi if case["act"] == "sigmoid" else g * phi
        res = {"h": gate * u}
        if case["train"]:
            slope = {"silu": lambda: phi + g * phi * torch.sigmoid(-g), "sigmoid": lambda: phi * torch.sigmoid(-g),
                     "relu": lambda: phi, "gelu": lambda: phi + g * torch.exp(-g.square() / 2) / math.sqrt(2 * math.pi)}[case["act"]]()
            dh = s["dh"].to(f64)
            dz = torch.cat([dh * u * slope, dh * gate], 1)
            dw = torch.mm(x.t().contiguous(), dz)
            res["dx"] = torch.mm(dz, w.t().contiguous())
            res["dwg"], res["dwu"] = dw.chunk(2, dim=1)
        return res
    N, V = case["tokens"], case["vocab"]
    x, tok = s["logits"].to(f64), s["tokens"].tolist()
    empty = torch.isneginf(x).all(1, keepdim=True)
    lse = torch.logsumexp(x, dim=1, keepdim=True)
    logp = torch.where(empty, -math.inf, x - lse)
    p = torch.where(empty, 0.0, torch.exp(logp))
    plogp = torch.where(p > 0, p * logp, 0.0)
    h = -plogp.sum(1, keepdim=True)
    at = [n for n in range(N) if 0 <= tok[n] < V]
    n, t = torch.tensor(at, device=DEV, dtype=torch.int64), torch.tensor([tok[i] for i in at], device=DEV, dtype=torch.int64)
    chosen = torch.zeros(N, device=DEV, dtype=f64)
    chosen[n] = logp[n, t]
    res = {"logp": chosen, "entropy": h[:, 0]}
    if case["top"]:
        res |= {"top_logp": torch.sort(logp, dim=1, descending=True).values[:, :case["top"]], "top_index": None}
    if case["train"]:
        a = torch.zeros(N, 1, device=DEV, dtype=f64)
        a[n, 0] = s["d_logp"].to(f64)[n]
        dx = -(a * p)
        dx[n, t] += torch.where(empty[n, 0], 0.0, a[n, 0])
        if case["entropy_grad"]:
            dx -= s["d_entropy"].to(f64)[:, None] * (plogp + p * h)
        res["d_logits"] = dx
    return res
