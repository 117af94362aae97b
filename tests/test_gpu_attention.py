"""Attention over a user's history against its definitions in 64 bits (attention_formulas.py), at the sizes, lengths, pages and layouts where
the kernels can go wrong."""
import numpy as np
import pytest
import torch

import attention_formulas as F
import paper_2404_09679_amd as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAN = float("nan")


def host(t):
    return t.double().cpu().numpy()


def ints(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def normal(rng, *shape, dtype="f32", std=1.0):
    return torch.as_tensor(rng.normal(size=shape) * std).to(DEV, DT[dtype])


def within(got, want, bound, what):
    got = host(got) if torch.is_tensor(got) else got
    bad = ~(np.abs(got - want) <= bound) & ~(got == want)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3],
                           np.broadcast_to(bound, want.shape)[bad][:3])


def laid(t, how):
    """t [.., rows, heads, D] in another layout: heads before rows, inside a wider row, or as it is."""
    if how == "heads":
        return t.transpose(-3, -2).contiguous().transpose(-3, -2)
    if how == "wide":
        wide = torch.full((*t.shape[:-2], 2 * t.shape[-2] + 1, t.shape[-1]), NAN, dtype=t.dtype, device=t.device)
        wide[..., 1:1 + t.shape[-2], :] = t
        return wide[..., 1:1 + t.shape[-2], :]
    if how == "odd":                # columns of padding: heads start anywhere
        wide = torch.full((*t.shape[:-1], t.shape[-1] + 3), NAN, dtype=t.dtype, device=t.device)
        wide[..., 1:1 + t.shape[-1]] = t
        return wide[..., 1:1 + t.shape[-1]]
    return t


# ------------------------------------------------------------------ rotary positions
ROTARY = [(1, 1, 2, 2), (1, 8, 64, 64), (5, 3, 128, 128), (33, 2, 100, 36), (7, 5, 33, 20), (64, 1, 16, 16), (300, 3, 72, 24), (9, 16, 256, 256), (3, 40, 128, 64),
          (1000, 2, 8, 6), (17, 1, 250, 250), (20000, 1, 32, 32)]


@pytest.mark.parametrize("N,H,D,R", ROTARY)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,how", [("f32", ""), ("bf16", ""), ("f32", "odd"), ("bf16", "wide"), ("bf16", "odd"), ("f32", "heads")])
def test_rotary(N, H, D, R, interleaved, dtype, how):
    rng = np.random.default_rng(N + H + D)
    x = laid(normal(rng, N, H, D, dtype=dtype), how)
    p = rng.integers(0, 5000, N)
    p[0], p[N // 2], p[N - 1] = 0, -3, 2 ** 31 - 1
    m = 1.25 if N % 2 else 1.0
    rot = A.Rotary(R, 10000.0, interleaved, magnitude=m, device=DEV)
    some = slice(None) if N <= 300 else [0, 1, 77, N // 2, N - 2, N - 1]
    turns = rot.turns.tolist()
    for inverse, call in ((False, A.rotary), (True, A.rotary_gradient)):
        want, e = F.rotate(host(x)[some], p[some], turns, interleaved, m, inverse)
        y = call(x, ints(p), rot)
        within(host(y)[some], want, e + F.HALF[dtype] * (np.abs(want) + e), inverse)
        into = laid(torch.zeros(N, H, D, dtype=DT[dtype], device=DEV), how)
        assert call(x, ints(p), rot, out=into) is into and torch.equal(into, y)
        same = x.clone()
        assert call(same, ints(p), rot, out=same) is same and torch.equal(same, y)
    assert torch.equal(y[..., R:], x[..., R:])


def test_rotary_back_and_forth():
    """The gradient of a sum of squares' half is what was put in: the rotation keeps lengths."""
    x, p = torch.randn(257, 4, 64, device=DEV), torch.arange(257, device=DEV, dtype=torch.int32) * 4001
    rot = A.Rotary(64, factor=8.0, original=4096, low=1.0, high=32.0, device=DEV)
    y = A.rotary(x, p, rot)
    # two passes, each off by 7 u (|u| + |v|) <= 7 sqrt(2) u of the pair's length, the second's operand by the first's
    pair = (x[..., :32] ** 2 + x[..., 32:] ** 2).sqrt().repeat(1, 1, 2)
    assert bool(((A.rotary_gradient(y, p, rot) - x).abs() <= 3 * 7 * 2 ** 0.5 * F.U * pair).all())


def test_rotary_without_rows():
    rot = A.Rotary(8, device=DEV)
    assert A.rotary(torch.empty(0, 3, 8, device=DEV), ints([]), rot).shape == (0, 3, 8)
    assert A.rotary(torch.empty(3, 0, 8, device=DEV), ints([1, 2, 3]), rot).shape == (3, 0, 8)


# ------------------------------------------------------------------ the paged cache
def cache_of(rng, lengths, page, H, D, dtype, spare=2, cols=0):
    """(k, v, table) with the users' pages scattered, the rest of the table -1; what is in no user's pages is NaN."""
    per = [-(-n // page) for n in lengths]
    place = rng.permutation(sum(per) + spare)
    table = np.full((len(per), max([cols, 1] + per)), -1)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = place[at:at + n]
        at += n
    k, v = (torch.full((sum(per) + spare, page, H, D), NAN, dtype=DT[dtype], device=DEV) for _ in range(2))
    return k, v, table


def append_formula(lengths, offsets, N):
    """(sequence, position) of every token, position -1: none."""
    seq, pos = np.zeros(N, int), np.full(N, -1)
    for b, n in enumerate(lengths):
        first, behind = (b, b + 1) if offsets is None else (offsets[b], offsets[b + 1])
        for i in range(max(first, 0), min(behind, N)):
            seq[i], pos[i] = b, max(-1, n - (behind - i))
    return seq, pos


APPEND = [  # lengths, new tokens (None: one each), page, q heads, heads, D, rotated, interleaved
    ([5], None, 16, 1, 1, 16, 16, False), ([1, 0, 17, 32, 33, 0, 500], None, 16, 8, 2, 64, 64, False), ([9, 0, 3], None, 1, 2, 1, 40, 0, False),
    ([30, 64, 7, 0, 1], [30, 10, 7, 0, 1], 24, 3, 3, 72, 24, True), ([100, 513], [40, 513], 64, 0, 4, 128, 128, False), ([12], [12], 5, 2, 2, 33, 20, False),
    ([300, 2, 2], [7, 1, 2], 100, 4, 1, 250, 250, True), (list(range(1, 130)), None, 7, 16, 8, 128, 64, True), ([40] * 3, [41, 40, 39], 16, 2, 2, 32, 32, False)]


@pytest.mark.parametrize("lengths,new,page,HQ,H,D,R,interleaved", APPEND)
@pytest.mark.parametrize("dtype,how", [("f32", ""), ("bf16", ""), ("bf16", "wide"), ("f32", "odd")])
def test_cache_append(lengths, new, page, HQ, H, D, R, interleaved, dtype, how):
    rng = np.random.default_rng(sum(lengths) + D)
    kc, vc, table = cache_of(rng, lengths, page, H, D, dtype)
    if len(lengths) > 2:
        table[2, -1] = len(kc)                              # a page that there is not
    offsets = None if new is None else np.cumsum([0] + new)
    N = len(lengths) if new is None else int(offsets[-1]) + 3   # three tokens in no sequence
    k, v = (laid(normal(rng, N, H, D, dtype=dtype), how) for _ in range(2))
    q = laid(normal(rng, N, HQ, D, dtype=dtype), how) if HQ else None
    rot = A.Rotary(R, 500.0, interleaved, device=DEV) if R else None
    turns = rot.turns.tolist() if R else []
    before = kc.clone(), vc.clone()
    kc, vc = laid(kc, how), laid(vc, how)
    got = A.cache_append(k, v, kc, vc, ints(table), ints(lengths), None if new is None else ints(offsets), rot, q)
    seq, pos = append_formula(lengths, offsets, N)
    want, e = F.rotate(host(k), np.maximum(pos, 0), turns, interleaved, 1.0)
    wk, wv = (host(t) for t in before)
    ek = np.zeros_like(wk)
    for n in range(N):
        at = pos[n] // page
        if pos[n] >= 0 and at < table.shape[1] and 0 <= table[seq[n], at] < len(kc):
            i = (table[seq[n], at], pos[n] % page)
            wk[i], ek[i], wv[i] = want[n], (e[n] + F.HALF[dtype] * (np.abs(want[n]) + e[n])) * bool(R), host(v)[n]
    gk, gv = host(kc), host(vc)
    assert np.array_equal(np.isnan(gk), np.isnan(wk)) and np.array_equal(np.isnan(gv), np.isnan(wv))
    within(np.nan_to_num(gk), np.nan_to_num(wk), ek, "keys")
    assert np.array_equal(np.nan_to_num(gv), np.nan_to_num(wv))
    if HQ == 0:
        assert got is None
        return
    want, e = F.rotate(host(q), np.maximum(pos, 0), turns, interleaved, 1.0)
    want[pos < 0] = e[pos < 0] = 0
    within(got, want, (e + F.HALF[dtype] * (np.abs(want) + e)) * bool(R), "queries")
    assert A.cache_append(k, v, kc, vc, ints(table), ints(lengths), None if new is None else ints(offsets), rot, q, q_out=q) is q
    assert torch.equal(q, got)


DECODE = [  # lengths, page, q heads, heads, D
    ([1], 16, 1, 1, 8), ([0], 16, 4, 2, 64), ([33], 7, 3, 3, 40), ([5, 0, 31, 32, 33, 64, 65, 1000, 1], 16, 8, 2, 128), ([700, 1, 333], 24, 6, 2, 72),
    ([2000], 64, 16, 2, 64), ([4000, 3], 1, 4, 1, 32), ([129, 515], 100, 40, 1, 128), ([257] * 40, 16, 2, 1, 16), ([9000], 33, 70, 2, 24),
    ([0, 0, 0], 16, 2, 2, 32), (list(range(300)), 5, 3, 1, 56)]


def decode_inputs(rng, lengths, page, HQ, H, D, dtype, std=1.0):
    kc, vc, table = cache_of(rng, lengths, page, H, D, dtype)
    dense = []
    for b, n in enumerate(lengths):
        k, v = normal(rng, n, H, D, dtype=dtype, std=std), normal(rng, n, H, D, dtype=dtype)
        dense.append((k, v))
        for c, x in ((kc, k), (vc, v)):
            t = np.arange(n)
            c[torch.as_tensor(table[b, t // page], device=DEV), torch.as_tensor(t % page, device=DEV)] = x
    return kc, vc, table, dense, normal(rng, len(lengths), HQ, D, dtype=dtype, std=std)


def check_decode(got, q, dense, dtype, scale, what):
    G = q.shape[1] // dense[0][0].shape[1]
    for b, (k, v) in enumerate(dense):
        for h in range(q.shape[1]):
            f = F.attend(host(q[b, h])[None], host(k[:, h // G]), host(v[:, h // G]), scale, F.HALF[dtype] * (dtype == "bf16"))
            within(host(got[b, h])[None], f["out"], f["e"] + F.HALF[dtype] * (np.abs(f["out"]) + f["e"]), (what, b, h))


@pytest.mark.parametrize("lengths,page,HQ,H,D", DECODE, ids=[f"{len(d[0])}x{max(d[0])}-{d[1]}-{d[2]}-{d[3]}-{d[4]}" for d in DECODE])
@pytest.mark.parametrize("dtype,how", [("f32", ""), ("bf16", ""), ("bf16", "wide"), ("bf16", "heads")])
def test_cache_attention(lengths, page, HQ, H, D, dtype, how):
    rng = np.random.default_rng(sum(lengths) + D)
    kc, vc, table, dense, q = decode_inputs(rng, lengths, page, HQ, H, D, dtype)
    kc, vc, q = laid(kc, how), laid(vc, how), laid(q, "wide" if how else "")
    got = A.cache_attention(q, kc, vc, ints(table), ints(lengths))
    check_decode(got, q, dense, dtype, D ** -0.5, "")
    into = laid(torch.full_like(got, 7.0), "wide" if how else "")
    assert A.cache_attention(q, kc, vc, ints(table), ints(lengths), out=into) is into and torch.equal(into, got)
    got = A.cache_attention(q, kc, vc, ints(table), ints(lengths), scale=1.5)
    check_decode(got, q, dense, dtype, 1.5, "scale")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cache_attention_leaves_out_pages_that_there_are_not(dtype):
    rng = np.random.default_rng(3)
    lengths, page, D = [200, 96, 40], 16, 64
    kc, vc, table, dense, q = decode_inputs(rng, lengths, page, 4, 2, D, dtype)
    gone = [(0, 0), (0, 3), (0, 12), (1, 5), (2, 0), (2, 1), (2, 2)]
    bad = [-1, len(kc), 2 ** 31 - 1, -2 ** 31, -1, len(kc) + 7, -5]
    for (b, i), page_of in zip(gone, bad):
        table[b, i] = page_of
    for b, n in enumerate(lengths):
        keep = torch.as_tensor([t for t in range(n) if (b, t // page) not in gone], dtype=torch.int64, device=DEV)
        dense[b] = tuple(x[keep] for x in dense[b])
    assert len(dense[2][0]) == 0
    got = A.cache_attention(q, kc, vc, ints(table), ints(lengths))
    check_decode(got, q, dense, dtype, D ** -0.5, "")
    # lengths beyond the table's pages, and below zero
    got2 = A.cache_attention(q, kc, vc, ints(table), ints([10 ** 6, -4, 40]))
    assert torch.equal(got2[0], A.cache_attention(q, kc, vc, ints(table), ints([table.shape[1] * page, 0, 40]))[0])
    assert not got2[1].any() and torch.equal(got2[2], got[2])


def test_cache_far_into_its_memory():
    """Pages behind 2^31 elements of a cache."""
    pages, page, D = 18_000, 1024, 128
    kc, vc = (torch.empty(pages, page, 1, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    assert kc.numel() > 2 ** 31
    rng = np.random.default_rng(5)
    table, lengths = ints([[17_999, 3, 16_500], [16_400, 1, 17_000]]), [2100, 1500]
    dense = [(normal(rng, n, 1, D, dtype="bf16"), normal(rng, n, 1, D, dtype="bf16")) for n in lengths]
    k, v = (torch.cat(x) for x in zip(*dense))
    A.cache_append(k, v, kc, vc, table, ints(lengths), ints([0, 2100, 3600]))
    q = normal(rng, 2, 2, D, dtype="bf16")
    check_decode(A.cache_attention(q, kc, vc, table, ints(lengths)), q, dense, "bf16", D ** -0.5, "")
    assert torch.equal(kc[16_500, :52], k[2048:2100]) and torch.equal(vc[17_000 - 600, 0], v[2100])


# ------------------------------------------------------------------ attention to a history of another length
CROSS = [  # B, S, T, q heads, heads, D, lengths: all, "ragged"
    (1, 1, 1, 1, 1, 8, ""), (2, 1, 5, 2, 2, 32, "ragged"), (3, 1, 700, 4, 2, 64, "ragged"), (2, 5, 33, 3, 1, 40, ""), (1, 33, 65, 2, 2, 16, "ragged"),
    (2, 127, 64, 2, 1, 128, ""), (3, 129, 200, 4, 2, 72, "ragged"), (2, 200, 31, 2, 2, 64, "ragged"), (1, 300, 333, 8, 2, 32, ""), (6, 40, 130, 6, 2, 56, "ragged"),
    (1, 16, 2000, 2, 1, 128, ""), (2, 260, 513, 2, 2, 104, "ragged"), (1, 50, 1, 1, 1, 24, ""), (4, 3, 4, 70, 10, 8, "ragged"),
    # few results with many terms each, and so many results that nothing is shared out
    (1, 40, 1100, 2, 1, 64, ""), (2, 70, 900, 1, 1, 88, "ragged"), (1, 33, 1500, 2, 2, 128, "ragged"), (1, 1000, 40, 4, 1, 64, ""), (2, 700, 20, 2, 1, 128, "ragged"),
    (3, 600, 33, 2, 1, 16, "ragged"), (9, 130, 140, 32, 32, 24, "ragged"), (9, 140, 130, 32, 32, 64, ""), (5, 131, 200, 64, 64, 88, "ragged"), (9, 129, 131, 32, 32, 128, "ragged")]


def cross_inputs(rng, B, S, T, HQ, H, D, kind, dtype, std=1.0):
    q, k, v, g = (normal(rng, B, n, h, D, dtype=dtype, std=s) for n, h, s in ((S, HQ, std), (T, H, std), (T, H, 1.0), (S, HQ, 1.0)))
    ql, kl = [S] * B, [T] * B
    if kind:
        ql, kl = rng.integers(1, S + 1, B).tolist(), rng.integers(1, T + 1, B).tolist()
        ql[0], kl[-1] = S, T
        if B > 1:
            kl[0] = max(1, T // 2)
        if B > 2:
            kl[1], ql[2] = 0, 0
        for b in range(B):                                   # what lies behind a length is not read into a result
            for x, n in ((q, ql), (k, kl), (v, kl), (g, ql)):
                x[b, n[b]:] = NAN
    return q, k, v, g, ql, kl


def check_cross(got, q, k, v, g, ql, kl, scale, dtype, what):
    """got: (out, dq, dk, dv), or (out,)."""
    B, S, HQ, D = q.shape
    T, H = k.shape[1:3]
    G, half = HQ // H, F.HALF[dtype] * (dtype == "bf16")
    names = ("out", "dq", "dk", "dv")[:len(got)]
    want, bound = ([np.zeros(tuple(x.shape)) for x in got] for _ in range(2))
    q, k, v, g = (host(x) for x in (q, k, v, g))
    for b in range(B):
        for h in range(HQ):
            x = q[b, :ql[b], h], k[b, :kl[b], h // G], v[b, :kl[b], h // G]
            f = F.attend(*x, scale, half)
            want[0][b, :ql[b], h], bound[0][b, :ql[b], h] = f["out"], f["e"]
            if len(got) > 1:
                r = F.attend_gradients(*x, g[b, :ql[b], h], scale, f, half, F.HALF[dtype])
                for i, at in ((1, (b, slice(ql[b]), h)), (2, (b, slice(kl[b]), h // G)), (3, (b, slice(kl[b]), h // G))):
                    want[i][at] += r[i - 1][0]
                    bound[i][at] += r[i - 1][1] * (1 + 4 * G * F.U) + 4 * G * F.U * np.abs(r[i - 1][0])     # (heads of a group add up too)
    for n, x, w, e in zip(names, got, want, bound):
        within(x, w, e + F.HALF[dtype] * (np.abs(w) + e), (what, n))


def cross(q, k, v, g, ql, kl, scale=None, **kw):
    stats = A.cross_attention_stats(q)
    out = A.cross_attention(q, k, v, ql, kl, scale, stats=stats)
    return (out, *A.cross_attention_backward(g, q, k, v, out, stats, ql, kl, scale))


@pytest.mark.parametrize("B,S,T,HQ,H,D,kind", CROSS)
@pytest.mark.parametrize("dtype,how", [("f32", ""), ("bf16", ""), ("bf16", "wide"), ("f32", "heads")])
def test_cross_attention(B, S, T, HQ, H, D, kind, dtype, how):
    rng = np.random.default_rng(S + T + D)
    q, k, v, g, ql, kl = cross_inputs(rng, B, S, T, HQ, H, D, kind, dtype)
    q, k, v, g = laid(q, how), laid(k, how), laid(v, "wide" if how else ""), laid(g, "heads" if how else "")
    dl = (ints(ql), ints(kl)) if kind else (None, None)
    got = cross(q, k, v, g, *dl)
    check_cross(got, q, k, v, g, ql, kl, D ** -0.5, dtype, "")
    assert all(torch.equal(a, b) for a, b in zip(cross(q, k, v, g, *dl), got))          # one order of addition
    assert torch.equal(A.cross_attention(q, k, v, *dl), got[0])
    stats, into = A.cross_attention_stats(q), [laid(torch.full_like(x, 7.0), how) for x in got]
    A.cross_attention(q, k, v, *dl, out=into[0], stats=stats)
    A.cross_attention_backward(g, q, k, v, into[0], stats, *dl, dq=into[1], dk=into[2], dv=into[3])
    assert all(torch.equal(a, b) for a, b in zip(into, got))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S", [3, 150])
def test_cross_attention_of_sharp_and_odd_scores(dtype, S):
    """Scores in the thousands, whose maximum moves from tile to tile; keys whose scores are -infinity, for some queries all."""
    rng = np.random.default_rng(S)
    T, D = 260, 64
    q, k, v, g, ql, kl = cross_inputs(rng, 1, S, T, 2, 1, D, "", dtype, std=8.0)
    q[0, :, 1] = q[0, :, 1].abs() + 1
    k = k * (torch.arange(1, T + 1, device=DEV) / 50).to(k.dtype)[None, :, None, None]
    check_cross((A.cross_attention(q, k, v),), q, k, v, g, ql, kl, D ** -0.5, dtype, "sharp")
    q = q.abs() + 0.5
    k[0, ::3] = -float("inf")
    check_cross((A.cross_attention(q, k, v),), q, k, v, g, ql, kl, D ** -0.5, dtype, "some")
    k[:] = -float("inf")
    out = cross(q, k, v, g, None, None)
    assert not out[0].any()


@pytest.mark.parametrize("S", [2, 140])
def test_cross_attention_keeps_what_is_not_a_number(S):
    q, k, v = (torch.randn(2, n, 2, 32, device=DEV) for n in (S, 70, 70))
    want = A.cross_attention(q, k, v)
    q2, v2 = q.clone(), v.clone()
    q2[0, 1, 1, 3] = NAN
    v2[1, 5, 0, 7] = NAN
    out = A.cross_attention(q2, k, v2)
    assert bool(out[0, 1, 1].isnan().all()) and bool(out[1, :, 0, 7].isnan().all())
    rest = torch.ones_like(out, dtype=torch.bool)
    rest[0, 1, 1] = rest[1, :, 0, 7] = False
    assert torch.equal(out[rest], want[rest])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S", [4, 130])
def test_cross_attention_of_a_repeated_history(dtype, S):
    """Every batch entry and every head reads the same keys: strides of 0."""
    rng = np.random.default_rng(S)
    B, T, H, D = 3, 90, 2, 64
    q, k, v, g, ql, kl = cross_inputs(rng, B, S, T, H, H, D, "", dtype)
    k, v = k[:1, :, :1].expand(B, T, H, D), v[:1].expand(B, T, H, D)
    check_cross(cross(q, k, v, g, None, None), q, k, v, g, ql, kl, D ** -0.5, dtype, "")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_of_a_single_key(dtype):
    """p = 1 and dP - d = 0, whatever out lost to its rounding: p is off by (4 |z| + 4) u and d = p dP by as much and 2 u more."""
    rng = np.random.default_rng(8)
    q, k, v, g, _, _ = cross_inputs(rng, 2, 150, 1, 2, 2, 64, "", dtype)
    out, dq, dk, dv = (host(x) for x in cross(q, k, v, g, None, None))
    # p is its own sum l; p v, 1 / l and their product round (in bf16 p rounds to 1, and v / l back to v)
    within(out, np.broadcast_to(host(v), out.shape), np.broadcast_to(3 * F.U * np.abs(host(v)) * (dtype == "f32"), out.shape), "out")
    dp = (np.abs(host(g)) * np.abs(host(v))).sum(-1, keepdims=True)
    z = (np.abs(host(q)) * np.abs(host(k))).sum(-1, keepdims=True) / 8
    dz = dp * (8 * z + 12) * F.U
    assert bool((np.abs(dq) <= dz * np.abs(host(k)) / 8 * 1.1).all())
    assert bool((np.abs(dk) <= (dz * np.abs(host(q))).sum(1, keepdims=True) / 8 * 1.1).all())


def test_cross_attention_of_nothing():
    e = torch.empty
    for B, S, T in ((0, 3, 4), (2, 0, 4), (2, 3, 0)):
        q, k = torch.randn(B, S, 4, 16, device=DEV), torch.randn(B, T, 2, 16, device=DEV)
        out = cross(q, k, k, q, None, None)
        assert [x.shape for x in out] == [q.shape, q.shape, k.shape, k.shape] and not any(x.any() for x in out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_against_differences(dtype):
    """The loss's change along a direction, from the definition in 64 bits, against the gradients' product with it."""
    rng = np.random.default_rng(11)
    q, k, v, g, ql, kl = cross_inputs(rng, 2, 20, 45, 4, 2, 32, "ragged", dtype)
    got = cross(q, k, v, g, ints(ql), ints(kl))

    def loss(x, y, z):
        total = 0.0
        for b in range(2):
            for h in range(4):
                f = F.attend(x[b, :ql[b], h], y[b, :kl[b], h // 2], z[b, :kl[b], h // 2], 32 ** -0.5, 0)
                total += (f["out"] * host(g)[b, :ql[b], h]).sum()
        return total

    args = [np.nan_to_num(host(x)) for x in (q, k, v)]
    for i, d in enumerate(got[1:]):
        # (an element of a gradient is off by a few roundings of its terms, at most 1 in magnitude here; their signs in the sum are even odds)
        way, eps = rng.normal(size=args[i].shape), 1e-5
        up, down = ([a + s * eps * way if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        want, size = (loss(*up) - loss(*down)) / (2 * eps), np.sqrt((way ** 2 * (host(d) ** 2 + 1)).sum())
        assert abs((host(d) * way).sum() - want) <= 8 * F.HALF[dtype] * size + 1e-4, i


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_history_trained_on_and_answered_from(dtype):
    """Positions, attention and its gradients over an encoded history as in training; the same history token by token through the cache gives the
    same keys bit for bit, and the same answers."""
    rng = np.random.default_rng(21)
    B, T, HQ, H, D, page = 3, 40, 4, 2, 64, 16
    rot = A.Rotary(D, device=DEV)
    q, k, v, g = (normal(rng, B, T, h, D, dtype=dtype) for h in (HQ, H, H, HQ))
    at = ints(np.tile(np.arange(T), B))
    rq, rk = (A.rotary(x.view(B * T, -1, D), at, rot).view(x.shape) for x in (q, k))
    kc, vc = (torch.full((10, page, H, D), NAN, dtype=DT[dtype], device=DEV) for _ in range(2))
    table, lengths = ints(rng.permutation(10)[:9].reshape(3, 3)), ints([0, 0, 0])
    first = [30, 0, 7]                                      # read in one go
    take = torch.cat([torch.arange(n, device=DEV) + b * T for b, n in enumerate(first)])
    lengths += ints(first)
    A.cache_append(k.view(B * T, H, D)[take], v.view(B * T, H, D)[take], kc, vc, table, lengths, ints([0, 30, 30, 37]), rot)
    for step in range(10):
        n = [f + step for f in first]
        now = torch.as_tensor([b * T + i for b, i in enumerate(n)], device=DEV)
        lengths += 1
        tq, tk, tv = (x.view(B * T, -1, D)[now] for x in (q, k, v))
        turned = A.cache_append(tk, tv, kc, vc, table, lengths, rotary=rot, q=tq)
        assert torch.equal(turned, rq.view(B * T, HQ, D)[now])
        got = A.cache_attention(turned, kc, vc, table, lengths)
        for b, i in enumerate(n):
            assert torch.equal(kc[table[b].long()].view(-1, H, D)[:i + 1], rk[b, :i + 1])
        stats = A.cross_attention_stats(turned[:, None])
        want = A.cross_attention(turned[:, None], rk, v, k_lengths=lengths, stats=stats)
        check_cross((want,), turned[:, None], rk, v, turned[:, None], [1] * B, [i + 1 for i in n], D ** -0.5, dtype, step)
        check_cross((got[:, None],), turned[:, None], rk, v, turned[:, None], [1] * B, [i + 1 for i in n], D ** -0.5, dtype, step)
    out = cross(rq, rk, v, g, None, None)
    check_cross(out, rq, rk, v, g, [T] * B, [T] * B, D ** -0.5, dtype, "trained")
    dk = A.rotary_gradient(out[2].view(B * T, H, D), at, rot)
    want, e = F.rotate(host(out[2]).reshape(B * T, H, D), np.tile(np.arange(T), B), rot.turns.tolist(), False, 1.0, True)
    within(dk, want, e + F.HALF[dtype] * (np.abs(want) + e), "dk")


def test_in_graphs_that_share_a_workspace():
    """A step of answering and a training step, captured; replayed in turn, with other inputs and eager calls between."""
    B, HQ, H, D, page = 5, 4, 2, 64, 16
    torch.manual_seed(0)
    rot = A.Rotary(D, device=DEV)
    kc, vc = (torch.zeros(40, page, H, D, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    table, lengths = torch.randperm(40, device=DEV)[:35].view(5, 7).int(), ints([40, 0, 17, 90, 1])
    tok = [torch.randn(B, h, D, device=DEV).bfloat16() for h in (HQ, H, H)]
    q, g = (torch.randn(2, 70, HQ, D, device=DEV).bfloat16() for _ in range(2))
    k, v = (torch.randn(2, 300, H, D, device=DEV).bfloat16() for _ in range(2))
    few = torch.randn(2, 1, HQ, D, device=DEV).bfloat16()
    workspace = torch.empty(16 << 20, dtype=torch.uint8, device=DEV)

    def answer(workspace=workspace):
        turned = A.cache_append(tok[1], tok[2], kc, vc, table, lengths, rotary=rot, q=tok[0])
        return turned, A.cache_attention(turned, kc, vc, table, lengths, workspace=workspace), A.cross_attention(few, k, v, workspace=workspace)

    def train(workspace=workspace):
        stats = A.cross_attention_stats(q)
        out = A.cross_attention(q, k, v, stats=stats, workspace=workspace)
        return (out, *A.cross_attention_backward(g, q, k, v, out, stats, workspace=workspace))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        answer(), train()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for f in (answer, train):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = f()
        graphs.append((f, graph, out))
    for i in range(4):
        for t in (*tok, q, k, v, g, few):
            t.copy_(torch.randn_like(t, dtype=torch.float32))
        lengths += 1
        for f, graph, out in graphs:
            graph.replay()
            got = [x.clone() for x in out]
            torch.cuda.synchronize()
            want = f(None)
            assert all(torch.equal(a, b) for a, b in zip(got, want)), (i, f.__name__)


def test_on_another_stream():
    q, k, v = (torch.randn(2, n, 4, 64, device=DEV) for n in (200, 300, 300))
    want = A.cross_attention(q, k, v)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = A.cross_attention(q, k, v)
    side.synchronize()
    assert torch.equal(got, want)
