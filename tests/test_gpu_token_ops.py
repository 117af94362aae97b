"""The operators on sequences of tokens against their definitions in 64 bits (token_formulas.py), at the sizes, masks
and layouts where the kernels can go wrong."""
import numpy as np
import pytest
import torch

import paper_2404_09679_amd as A
import token_formulas as F

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def strided(x, dtype, pad=0, offset=0, fill=float("nan")):
    """x on the device, `pad` columns (of NaN) behind every row, the first row `offset` elements into its buffer."""
    rows, cols = x.shape
    buf = torch.full((rows * (cols + pad) + offset + 16,), fill, dtype=DT[dtype], device=DEV)
    t = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.as_tensor(x))
    return t


def host(t):
    return t.double().cpu().numpy()


def ints(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def within(got, want, bound, what):
    got = host(got) if torch.is_tensor(got) else got
    bad = ~(np.abs(got - want) <= bound) & ~(got == want)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3],
                           np.broadcast_to(bound, want.shape)[bad][:3])


# ------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (3, 7, 0, 0), (5, 8, 0, 0), (4, 12, 0, 0), (4, 12, 4, 4), (7, 250, 1, 3),
                                                  (33, 1000, 8, 8), (3, 4099, 0, 1), (300, 64, 0, 0)])
def test_dropout(dtype, rows, cols, pad, offset):
    rng = np.random.default_rng(rows * 1000 + cols)
    x, r = rng.normal(size=(rows, cols)), rng.normal(size=(rows, cols))
    dx, dr = strided(x, dtype, pad, offset), strided(r, dtype, pad, offset)
    x, r = host(dx), host(dr)
    for p, seed, call in ((0.3, 12345678901234567890, 7), (0.0, 3, 0), (1.0, 5, 2)):
        m = F.keep(rows, cols, p, seed, call)
        drop = A.Dropout(p, seed, call)
        within(A.dropout(dx, drop), x * m, (2 * F.U32 + F.HALF[dtype]) * np.abs(x * m), ("plain", p))
        y = A.dropout(dx, drop, residual=dr)
        want = r + x * m
        within(y, want, 3 * F.U32 * (np.abs(r) + np.abs(x * m)) + F.HALF[dtype] * np.abs(want) * 1.01, ("residual", p))
    inplace = strided(x, dtype, pad, offset)
    assert A.dropout(inplace, drop, residual=dr, out=inplace) is inplace and torch.equal(inplace, y)
    into = strided(r, dtype, pad, offset)
    assert torch.equal(A.dropout(dx, drop, residual=into, out=into), y)


def test_dropout_drops_what_is_not_finite_and_keeps_the_mean():
    n = 1 << 20
    x = torch.full((n // 512, 512), float("inf"), device=DEV)
    y = A.dropout(x, A.Dropout(0.25, 99))
    assert not torch.isnan(y).any() and bool(((y == 0) | torch.isinf(y)).all())
    dropped = int((y == 0).sum())
    assert abs(dropped - 0.25 * n) < 6 * (0.25 * 0.75 * n) ** 0.5       # six standard deviations
    other = A.dropout(x, A.Dropout(0.25, 99, call=1))
    same = int(((y == 0) & (other == 0)).sum())
    assert abs(same - 0.0625 * n) < 6 * (0.0625 * 0.9375 * n) ** 0.5    # another call's mask is another one


def test_dropout_in_a_graph_draws_anew():
    x = torch.randn(64, 96, device=DEV)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    drop, out = A.Dropout(0.5, 41, 3, step), torch.empty_like(x)
    A.dropout(x, drop, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        A.dropout(x, drop, out=out)
    for i in range(4):
        step.fill_(i)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, A.dropout(x, A.Dropout(0.5, 41 + i, 3)))


# ------------------------------------------------------------------ lookup and its gradient
def tokens_of(rng, kind, N, V):
    if kind == "zipf":
        t = np.minimum(rng.zipf(1.3, N) - 1, V - 1)
    elif kind == "one":
        t = np.full(N, V // 2)
    elif kind == "two":
        t = np.where(rng.random(N) < 0.5, V - 1, 0)
    elif kind == "padding":
        t = np.full(N, -1)
    elif kind == "each":
        t = rng.permutation(np.arange(N) % V)
    else:
        t = rng.integers(0, V, N)
    if kind in ("zipf", "even") and N > 3:
        t[rng.random(N) < 0.1] = -1
        t[0], t[1], t[2] = V, 2 ** 31 - 1, -2 ** 31
    return t.astype(np.int64)


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("N,V,D,pad,offset", [(1, 1, 1, 0, 0), (5, 9, 8, 0, 0), (37, 100, 20, 0, 0), (64, 50, 12, 4, 4), (100, 333, 63, 1, 1),
                                              (1000, 77, 256, 0, 0), (9, 40, 2056, 8, 0)])
def test_lookup(dtype, out, N, V, D, pad, offset):
    rng = np.random.default_rng(N + D)
    table = strided(rng.normal(size=(V, D)), dtype, pad, offset)
    t = tokens_of(rng, "even", N, V)
    for p in (0.0, 0.4):
        m = F.keep(N, D, p, 7, 2)
        want = F.lookup(host(table), t, 1.7, m)
        got = A.token_lookup(table, ints(t), 1.7, dropout=A.Dropout(p, 7, 2), out_dtype=DT[out])
        assert got.dtype == DT[out]
        within(got, want, (4 * F.U32 + F.HALF[out]) * np.abs(want), p)
    into = strided(np.zeros((N, D)), out, pad, offset)
    A.token_lookup(table, ints(t), 1.7, dropout=A.Dropout(p, 7, 2), out=into)
    assert torch.equal(into, got)


SUMS = [("zipf", 1, 5, 8), ("zipf", 9, 3, 16), ("zipf", 1000, 200, 20), ("even", 3001, 5000, 100), ("one", 5000, 9, 32), ("two", 3000, 70, 8),
        ("padding", 300, 20, 16), ("each", 2048, 2048, 4), ("each", 640, 64, 63), ("zipf", 20000, 3000, 64), ("one", 40000, 4, 40),
        ("zipf", 300, 50, 1100), ("even", 17000, 1 << 21, 8)]


@pytest.mark.parametrize("kind,N,V,D", SUMS, ids=["-".join(map(str, s)) for s in SUMS])
@pytest.mark.parametrize("dtype,pad,offset", [("f32", 0, 0), ("bf16", 0, 0), ("bf16", 3, 1), ("f32", 4, 0)])
def test_token_gradient(kind, N, V, D, dtype, pad, offset):
    rng = np.random.default_rng(N + D)
    t = tokens_of(rng, kind, N, V)
    dy = strided(rng.normal(size=(N, D)), dtype, pad, offset)
    for p in (0.0, 0.3):
        m = F.keep(N, D, p, 21, 4)
        want, mag, n = F.table_gradient(host(dy), t, V, 0.5, m)
        bound = (n[:, None] + 4) * F.U32 * mag
        drop = A.Dropout(p, 21, 4)
        got = A.token_gradient(dy, ints(t), V, 0.5, dropout=drop)
        within(got, want, bound, p)
        assert torch.equal(A.token_gradient(dy, ints(t), V, 0.5, dropout=drop), got)      # one order of addition
    old = rng.normal(size=(V, D))
    grad = strided(old, "f32", pad, offset)
    old = host(grad)
    A.token_gradient(dy, ints(t), V, 0.5, dropout=drop, out=grad, accumulate=True)
    within(grad, old + want, bound + 2 * F.U32 * (np.abs(old) + np.abs(want)), "accumulated")
    assert np.array_equal(host(grad)[n == 0], old[n == 0])
    over = strided(np.full((V, D), 3.0), "f32", pad, offset)
    A.token_gradient(dy, ints(t), V, 0.5, dropout=drop, out=over)
    assert torch.equal(over, got)


def test_token_gradient_without_tokens():
    dy, none = torch.empty(0, 12, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    assert not A.token_gradient(dy, none, 7).any()
    grad = torch.ones(7, 12, device=DEV)
    A.token_gradient(dy, none, 7, out=grad, accumulate=True)
    assert bool((grad == 1).all())
    assert A.token_lookup(grad, none).shape == (0, 12)


def test_lookup_far_into_a_table():
    V, D = 9_000_000, 256                                     # 2.3e9 elements
    table = torch.empty(V, D, dtype=torch.bfloat16, device=DEV)
    rows = [0, 4_194_303, 8_388_608, V - 1]
    for i, r in enumerate(rows):
        table[r] = i + 1
    got = A.token_lookup(table, ints(rows), 2.0)
    assert torch.equal(got.float(), torch.tensor([2.0, 4.0, 6.0, 8.0], device=DEV)[:, None].expand(4, D))
    del table
    grad = torch.full((V, D), 5.0, device=DEV)
    A.token_gradient(got, ints(rows), V, out=grad)
    assert all(bool((grad[r] == 2.0 * (i + 1)).all()) for i, r in enumerate(rows))
    assert int(torch.count_nonzero(grad[:, 0])) == 4 and int(torch.count_nonzero(grad[:, D - 1])) == 4


# ------------------------------------------------------------------ gated block
def gated_inputs(rng, N, K, H, dtype, pad, offset):
    x, wg, wu = rng.normal(size=(N, K)), rng.normal(size=(K, H)) / K ** 0.5, rng.normal(size=(K, H)) / K ** 0.5
    return [strided(v, dtype, pad, offset) for v in (x, wg, wu, rng.normal(size=(N, H)))]


# tokens, widths: one row, one element, a tile and one more or less, several tiles of every size, odd ones of fp32
GATED = [(1, 8, 8, 0, 0), (3, 64, 72, 8, 8), (16, 136, 264, 0, 0), (31, 72, 40, 0, 0), (65, 128, 128, 8, 0), (129, 520, 328, 0, 0), (300, 64, 1400, 0, 0),
         (513, 200, 136, 8, 8), (1, 2048, 1032, 0, 0), (7, 1000, 520, 0, 0)]
GATED_LARGE = [(2500, 1288, 2056), (8200, 264, 520), (300, 2056, 7000)]
GATED_ODD = [(1, 1, 1, 0, 0), (5, 7, 3, 1, 1), (67, 33, 130, 0, 0), (130, 201, 65, 3, 2), (64, 68, 36, 0, 1), (2, 333, 1001, 0, 0)]


@pytest.mark.parametrize("act", ["silu", "gelu", "relu", "sigmoid"])
@pytest.mark.parametrize("dtype,N,K,H,pad,offset", [("bf16", *s) for s in GATED] + [("f32", *s) for s in GATED + GATED_ODD])
def test_gated(dtype, N, K, H, pad, offset, act):
    rng = np.random.default_rng(N + K + H)
    x, wg, wu, dh = gated_inputs(rng, N, K, H, dtype, pad, offset)
    f = F.gated(host(x), host(wg), host(wu), act, F.HALF[dtype])
    h = A.gated_forward(x, wg, wu, act)
    within(h, f["h"], f["eh"], "h")
    saved = A.gated_saved(x, wg)
    into = strided(np.zeros((N, H)), dtype, pad, offset)
    within(A.gated_forward(x, wg, wu, act, out=into, saved=saved), f["h"], f["eh"], "h, saving")
    want = F.gated_gradients(host(x), host(wg), host(wu), host(dh), f, F.HALF[dtype])
    outs = [strided(np.zeros(s), dtype, pad, offset) for s in ((N, K), (K, H), (K, H))]
    got = A.gated_backward(dh, x, wg, wu, saved, *outs)
    # a rounding of dz and one of the result; the sums' own errors as of random signs
    norm = 2 * F.HALF[dtype] if dtype == "bf16" else (8 + (N + K + H) ** 0.5) * F.U32
    for name, g, (w, e) in zip(("dx", "dwg", "dwu"), got, want):
        within(g, w, e, name)
        if act != "relu" and min(N, K, H) > 4:
            assert np.linalg.norm(host(g) - w) <= norm * np.linalg.norm(w), name
    for a, b in zip(A.gated_backward(dh, x, wg, wu, saved), got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,K,H", GATED_LARGE)
def test_gated_large(dtype, N, K, H):
    """Sizes of the larger tiles, against products in 64 bits on the device."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(N)
    x, wg, wu, dh = (torch.randn(*s, device=DEV, generator=gen).mul_(v).to(DT[dtype])
                     for s, v in (((N, K), 1), ((K, H), K ** -0.5), ((K, H), K ** -0.5), ((N, H), 1)))
    saved = A.gated_saved(x, wg)
    h = A.gated_forward(x, wg, wu, "silu", saved=saved)
    assert torch.equal(A.gated_forward(x, wg, wu, "silu"), h)
    got = (h,) + A.gated_backward(dh, x, wg, wu, saved)
    X, G, U, D = x.double(), wg.double(), wu.double(), dh.double()
    g, u = X @ G, X @ U
    s = torch.sigmoid(g)
    dg, du = D * u * s * (1 + g * (1 - s)), D * g * s
    want = (g * s * u, dg @ G.t().contiguous() + du @ U.t().contiguous(), X.t().contiguous() @ dg, X.t().contiguous() @ du)
    norm = 2 * F.HALF[dtype] if dtype == "bf16" else (8 + (N + K + H) ** 0.5) * F.U32
    for name, a, b in zip(("h", "dx", "dwg", "dwu"), got, want):
        off = a.double() - b
        assert float(off.norm() / b.norm()) <= norm, name
        # tile by tile too: a corner that was missed would hide in the whole
        for r in range(0, b.shape[0], 512):
            for c in range(0, b.shape[1], 512):
                assert float(off[r:r + 512, c:c + 512].norm()) <= 2 * norm * float(b[r:r + 512, c:c + 512].norm()), (name, r, c)


def test_gated_gradient_against_differences():
    """<gradient, v> against differences of the fp32 forward pass's definition in 64 bits."""
    rng = np.random.default_rng(8)
    x, wg, wu, dh = gated_inputs(rng, 19, 24, 40, "f32", 0, 0)
    for act in ("silu", "gelu", "sigmoid"):
        saved = A.gated_saved(x, wg)
        A.gated_forward(x, wg, wu, act, saved=saved)
        args = [host(x), host(wg), host(wu)]
        for k, g in enumerate(A.gated_backward(dh, x, wg, wu, saved)):
            v = rng.normal(size=tuple(g.shape))
            up, down = ([a + s * 1e-5 * v if i == k else a for i, a in enumerate(args)] for s in (1, -1))
            diff = sum(s * (F.gated(*a, act, 0)["h"] * host(dh)).sum() for s, a in ((1, up), (-1, down))) / 2e-5
            assert abs(diff - (host(g) * v).sum()) <= 1e-5 * np.abs(host(g) * v).sum(), (act, k)


def test_gated_wide_rows():
    """Rows so far apart that their offsets pass 2^32 bytes."""
    N, K, H, ld = 2000, 64, 72, (1 << 21) - 8
    buf = torch.empty(N * ld, dtype=torch.bfloat16, device=DEV)
    x = buf.view(N, ld)[:, :K]
    x.normal_()
    wg, wu = torch.randn(K, H, device=DEV).bfloat16(), torch.randn(K, H, device=DEV).bfloat16()
    assert torch.equal(A.gated_forward(x, wg, wu), A.gated_forward(x.contiguous(), wg, wu))
    saved, dh = A.gated_saved(x, wg), torch.randn(N, H, device=DEV).bfloat16()
    A.gated_forward(x, wg, wu, saved=saved)
    for a, b in zip(A.gated_backward(dh, x, wg, wu, saved), A.gated_backward(dh, x.contiguous(), wg, wu, saved)):
        assert torch.equal(a, b)


def test_gated_without_tokens_and_what_is_not_finite():
    w = torch.randn(16, 24, device=DEV)
    none = torch.empty(0, 16, device=DEV)
    assert A.gated_forward(none, w, w).shape == (0, 24)
    dx, dwg, dwu = A.gated_backward(torch.empty(0, 24, device=DEV), none, w, w, A.gated_saved(none, w))
    assert dx.shape == (0, 16) and not dwg.any() and not dwu.any()
    x = torch.randn(70, 16, device=DEV)
    x[3, 5], x[69, 0] = float("nan"), float("nan")
    for act in ("silu", "gelu", "relu", "sigmoid"):
        h = A.gated_forward(x, w, w, act)
        assert bool(torch.isnan(h[[3, 69]]).all()) and not bool(torch.isnan(h[[0, 2, 4, 68]]).any())
    big = torch.full((4, 16), 1e4, device=DEV) * torch.tensor([1.0, -1.0, 1.0, -1.0], device=DEV)[:, None]
    one = torch.ones(16, 24, device=DEV)
    saved = A.gated_saved(big, one)
    h = A.gated_forward(big, one, one, "silu", saved=saved)
    assert bool((h[0] == 1.6e5 ** 2).all()) and bool((h[1] == 0).all())
    assert bool(torch.isfinite(A.gated_backward(torch.ones(4, 24, device=DEV), big, one, one, saved)[0]).all())


# ------------------------------------------------------------------ log probabilities
LOGPROBS = [(1, 1, 1), (3, 5, 3), (2, 8, 8), (5, 63, 7), (4, 600, 64), (7, 4099, 10), (600, 130, 4), (3, 20011, 64), (1, 300000, 33), (2, 65536, 1), (520, 9000, 5)]


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype,pad,offset", [("f32", 0, 0), ("bf16", 0, 0), ("bf16", 5, 3), ("f32", 1, 1), ("bf16", 8, 0)])
@pytest.mark.parametrize("N,V,top", LOGPROBS)
def test_logprobs(N, V, top, dtype, pad, offset, masked):
    rng = np.random.default_rng(N + V)
    x = rng.normal(size=(N, V)) * 3
    if masked:
        x[rng.random((N, V)) < 0.4] = -np.inf
        x[N // 2] = -np.inf
        lowest = torch.finfo(DT[dtype]).min
        x[0, rng.random(V) < 0.5] = lowest                    # the other way to mask
    t = rng.integers(0, V, N)
    if N > 2:
        t[1], t[2] = -1, V
    dx = strided(x, dtype, pad, offset)
    f = F.logprobs(host(dx), t, top)
    r = A.token_logprobs(dx, ints(t), top)

    def near(got, want, x):
        fin = np.isfinite(want)
        got = host(got)
        assert np.array_equal(got[~fin], want[~fin])
        within(got[fin], want[fin], F.U32 * (f["depth"] + 4 * x)[fin], "value")

    spread = np.abs(np.where(np.isfinite(f["logp"]), f["logp"], 0)) + np.abs(f["log_s"])
    near(r.logp, f["logp"], spread)
    near(r.entropy, f["entropy"], 4 + f["entropy"] * f["depth"])
    assert np.array_equal(host(r.top_index).astype(np.int64), f["top_index"])
    near(r.top_logp, f["top_logp"], np.abs(np.where(np.isfinite(f["top_logp"]), f["top_logp"], 0)) + np.abs(f["log_s"])[:, None])
    again = A.token_logprobs(dx, None, 0)
    assert again.logp is None and again.top_index is None
    within(again.entropy, host(r.entropy), 0, "without the top")

    a, b = rng.normal(size=N), rng.normal(size=N)
    da, db = (torch.as_tensor(v, dtype=torch.float32, device=DEV) for v in (a, b))
    for ga, gb in ((da, db), (da, None), (None, db)):
        want, e = F.logprobs_gradient(f, t, host(da) if ga is not None else np.zeros(N), host(db) if gb is not None else np.zeros(N))
        got = A.token_logprobs_gradient(dx, ints(t) if ga is not None else None, r.stats, ga, gb)
        within(got, want, e + F.HALF[dtype] * (np.abs(want) + e) + 1e-38, "gradient")
    into = strided(np.zeros((N, V)), dtype, 2, 1)
    A.token_logprobs_gradient(dx, None, r.stats, None, db, out=into)
    assert torch.equal(into, got)
    A.token_logprobs_gradient(dx, None, r.stats, None, db, out=dx)
    assert torch.equal(dx, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [500, 5000, 70000])
def test_top_of_equal_and_of_unevenly_spread_logits(dtype, V):
    few = np.random.default_rng(V).integers(0, 3, size=(2, V)).astype(float)      # many equal logits
    flat = np.zeros((1, V))
    signs = np.where(np.arange(V) % 2, 0.0, -0.0)[None]                            # 0 and -0 are equal
    # all of the largest in the columns that a few threads read: every 512th group of 16 bytes
    per = 16 // (4 if dtype == "f32" else 2)
    lumps = np.where((np.arange(V) // per) % 512 < 4, np.arange(V) / 64.0, -5.0)[None]
    down = -np.arange(V, dtype=float)[None]
    x = strided(np.concatenate([few, flat, signs, lumps, down, -down]), dtype)
    top = 40
    f = F.logprobs(host(x), np.zeros(len(x), np.int64), top)
    r = A.token_logprobs(x, None, top)
    assert np.array_equal(host(r.top_index).astype(np.int64), f["top_index"])


@pytest.mark.parametrize("top", [1, 6, 7, 16, 17, 32, 64])
@pytest.mark.parametrize("N,V", [(2, 64), (3, 3001), (1, 40000), (513, 70)])
def test_how_many_of_the_top(N, V, top):
    """Every way to find the threshold, over one block and over pieces, with logits that differ and with many that do not."""
    rng = np.random.default_rng(V + top)
    x = np.concatenate([rng.normal(size=(N, V)), np.round(rng.normal(size=(N, V)))])
    x[-1, : V // 2] = -np.inf
    dx = strided(x, "f32", 1, 0)
    r = A.token_logprobs(dx, None, top)
    f = F.logprobs(host(dx), np.zeros(2 * N, np.int64), top)
    assert np.array_equal(host(r.top_index).astype(np.int64), f["top_index"])


@pytest.mark.parametrize("V", [300, 40000])
def test_logprobs_of_rows_with_what_is_not_finite(V):
    x = torch.randn(4, V, device=DEV)
    x[0, 17], x[1, V - 1], x[2, :] = float("nan"), float("inf"), float("nan")
    r = A.token_logprobs(x, ints([3, 4, 5, 6]), 3)
    assert bool(torch.isnan(r.logp[:3]).all()) and bool(torch.isnan(r.entropy[:3]).all())
    assert torch.isfinite(r.logp[3]) and torch.isfinite(r.entropy[3])
    assert r.top_index[0, 0] == 17 and r.top_index[1, 0] == V - 1 and r.top_index[2].tolist() == [0, 1, 2]
    rest = x[0].clone()
    rest[17] = -float("inf")
    assert r.top_index[0, 1:].tolist() == rest.topk(2).indices.tolist()
    assert torch.equal(r.top_index[3].long(), x[3].topk(3).indices)


def test_logprobs_far_into_the_logits():
    N, V = 48000, 50000                                       # 2.4e9 elements
    x = torch.zeros(N, V, dtype=torch.bfloat16, device=DEV)
    x[N - 1, V - 3] = 4
    t = torch.full((N,), V - 3, dtype=torch.int32, device=DEV)
    r = A.token_logprobs(x, t, 1)
    assert r.top_index[N - 1, 0] == V - 3 and r.top_index[N - 2, 0] == 0
    s = V - 1 + np.exp(4)
    assert abs(float(r.logp[N - 1]) - (4 - np.log(s))) < 1e-4 and abs(float(r.logp[N - 2]) + np.log(V)) < 1e-4
    d = A.token_logprobs_gradient(x, t, r.stats, torch.ones(N, device=DEV), out=x)
    assert abs(float(d[N - 1, V - 3]) - (1 - np.exp(4) / s)) < 0.01 and abs(float(d[N - 1, 0]) * s + 1) < 0.01


# ------------------------------------------------------------------ together
def test_operators_on_another_stream_and_in_a_graph():
    """The path tokens -> lookup -> gated -> logits -> log probabilities and back on a stream of its own, and replayed
    from a graph with other tokens in the same buffers."""
    V, D, H, N = 700, 64, 128, 96
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    table = torch.randn(V, D, device=DEV, generator=gen).bfloat16()
    wg, wu = (torch.randn(D, H, device=DEV, generator=gen).mul_(D ** -0.5).bfloat16() for _ in range(2))
    wd = torch.randn(H, V, device=DEV, generator=gen).mul_(H ** -0.5).bfloat16()
    wdt = wd.t().contiguous()
    batch = [[torch.randint(0, V, (N,), device=DEV, generator=gen).int() for _ in range(2)] for _ in range(4)]
    tokens, target = (b.clone() for b in batch[0])
    ones = torch.full((N,), -1.0 / N, device=DEV)
    drop = A.Dropout(0.1, 17)

    def step():
        x = A.token_lookup(table, tokens, 8.0, dropout=drop)
        saved = A.gated_saved(x, wg)
        h = A.gated_forward(x, wg, wu, saved=saved)
        logits = h @ wd
        r = A.token_logprobs(logits, target, 4)
        dl = A.token_logprobs_gradient(logits, target, r.stats, ones)
        dx, dwg, dwu = A.gated_backward(dl @ wdt, x, wg, wu, saved)
        return r.logp, r.top_index, dwg, dwu, A.token_gradient(dx, tokens, V, 8.0, dropout=drop)

    want = []
    for b in batch:
        tokens.copy_(b[0])
        target.copy_(b[1])
        want.append([t.clone() for t in step()])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for b, w in zip(batch, want):
            tokens.copy_(b[0])
            target.copy_(b[1])
            got = step()
            side.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, w))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs = step()
    torch.cuda.synchronize()
    for b, w in list(zip(batch, want)) * 2:
        tokens.copy_(b[0])
        target.copy_(b[1])
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, w))
        assert torch.equal(step()[0], w[0])                    # eager work between the replays
        torch.cuda.synchronize()


def test_next_item_example_learns():
    """examples/next_item.py: the operators in one training step, and the answer to a single user."""
    import importlib.util
    import os
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "next_item.py")
    spec = importlib.util.spec_from_file_location("next_item", at)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    model, loss = m.train(steps=60, items=200, width=64, hidden=256, n=2048)
    assert loss[0] > 4 and loss[-1] < 0.5 * loss[0], (loss[0], loss[-1])
    again = m.train(steps=3, items=200, width=64, hidden=256, n=2048)[1]
    assert again[0] == loss[0]
    items, p = model.answer(5, top=3)
    assert len(items) == 3 and p[0] >= p[1] >= p[2] > 0 and sum(p) <= 1 + 1e-4


def test_refusals_of_tensors():
    x, t = torch.zeros(4, 8, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    for call in (lambda: A.token_lookup(x, t.long()), lambda: A.token_lookup(x.t()[:, ::2], t), lambda: A.token_lookup(x.half(), t),
                 lambda: A.token_lookup(x.cpu(), t), lambda: A.token_gradient(x, t[:3], 5), lambda: A.token_gradient(x, t, 5, accumulate=True),
                 lambda: A.gated_forward(x, x, x), lambda: A.gated_forward(x, x.t(), x.t()), lambda: A.token_logprobs(x, t[:2]),
                 lambda: A.gated_forward(x, torch.zeros(8, 8, device=DEV), torch.zeros(8, 8, device=DEV), "tanh"),
                 lambda: A.dropout(x, A.Dropout(0.1, 1), residual=x.bfloat16()),
                 lambda: A.token_logprobs_gradient(x, t, x, torch.zeros(4, device=DEV))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: A.dropout(x, A.Dropout(2.0, 1)), lambda: A.token_logprobs(x, t, 9),
                 lambda: A.gated_forward(torch.zeros(4, 12, device=DEV).bfloat16(), torch.zeros(12, 8, device=DEV).bfloat16(),
                                         torch.zeros(12, 8, device=DEV).bfloat16())):
        with pytest.raises(A.AntdtError):
            call()


@pytest.mark.parametrize("N,K,H", [(8192, 8, 2048), (8200, 32, 2056), (8192, 40, 2048), (8192, 72, 4096), (8192, 104, 2048), (8192, 136, 2048), (8, 8192, 4096),
                                   (40, 4096, 8192)])
def test_gated_with_few_contraction_slots(N, K, H):
    """Large tiles whose products end before, at and behind the stages their pipeline is filled with."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(K)
    x, wg, wu, dh = (torch.randn(*s, device=DEV, generator=gen).mul_(v).bfloat16()
                     for s, v in (((N, K), 1), ((K, H), K ** -0.5), ((K, H), K ** -0.5), ((N, H), 1)))
    saved = A.gated_saved(x, wg)
    h = A.gated_forward(x, wg, wu, "sigmoid", saved=saved)
    got = (h,) + A.gated_backward(dh, x, wg, wu, saved)
    X, G, U, D = x.double(), wg.double(), wu.double(), dh.double()
    s, u = torch.sigmoid(X @ G), X @ U
    dg, du = D * u * s * (1 - s), D * s
    want = (s * u, dg @ G.t().contiguous() + du @ U.t().contiguous(), X.t().contiguous() @ dg, X.t().contiguous() @ du)
    for name, a, b in zip(("h", "dx", "dwg", "dwu"), got, want):
        off = a.double() - b
        for r in range(0, b.shape[0], 256):      # (a rounding of dz and one of the result)
            for c in range(0, b.shape[1], 256):
                assert float(off[r:r + 256, c:c + 256].norm()) <= 4 * F.HALF["bf16"] * float(b[r:r + 256, c:c + 256].norm()), (name, r, c)


def test_logprobs_without_rows_and_with_a_workspace():
    none = A.token_logprobs(torch.empty(0, 40, device=DEV), ints([]), 3)
    assert none.logp.shape == (0,) and none.entropy.shape == (0,) and none.stats.shape == (0, 4)
    assert none.top_logp.shape == (0, 3) and none.top_index.shape == (0, 3) and none.top_index.dtype == torch.int32
    x = torch.randn(2, 100003, device=DEV)
    want = A.token_logprobs(x, ints([5, -1]), 9)
    given = A.token_logprobs(x, ints([5, -1]), 9, workspace=torch.full((1 << 20,), 255, dtype=torch.uint8, device=DEV))
    for a, b in zip(want, given):
        assert torch.equal(a, b) and a.is_contiguous()
    with pytest.raises(A.AntdtError):
        A.token_logprobs(x, None, 9, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    with pytest.raises(A.AntdtError):
        A.token_logprobs(x, None, -1)


@pytest.mark.parametrize("top", [3, 6, 9, 40])
@pytest.mark.parametrize("V", [2000, 30000, 100000])
def test_top_of_logits_far_apart_and_alike(top, V):
    """Where the distance from the largest logit decides least: all of a row equal (and not allowed), one far above the rest, logits over the
    type's whole range, negative ones, and values next to each other."""
    rng = np.random.default_rng(V + top)
    x = rng.normal(size=(8, V))
    x[0] = -np.inf
    x[1] = 7.25
    x[2, V // 3] = 1e30
    x[3] = np.sign(x[3]) * 10.0 ** rng.uniform(-37, 38, V)
    x[4] = -np.abs(x[4]) * 1e-30
    x[5] = 1 + rng.integers(0, 50, V) * 2.0 ** -23
    x[6, rng.random(V) < 0.999] = -np.inf
    x[7] = np.where(rng.random(V) < 0.5, torch.finfo(torch.float32).min, 0.0)
    dx = strided(x, "f32", 1, 1)
    f = F.logprobs(host(dx), np.zeros(8, np.int64), top)
    r = A.token_logprobs(dx, None, top)
    assert np.array_equal(host(r.top_index).astype(np.int64), f["top_index"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 8, 9])
@pytest.mark.parametrize("K,H", [(48, 9736), (1104, 2408)])
def test_gated_of_a_few_tokens_and_wide_blocks(N, K, H, dtype):
    """The ways to share out a few tokens' columns, with columns behind the last whole share."""
    rng = np.random.default_rng(N + H)
    x, wg, wu, _ = gated_inputs(rng, N, K, H, dtype, 8, 8)
    f = F.gated(host(x), host(wg), host(wu), "silu", F.HALF[dtype])
    saved = A.gated_saved(x, wg)
    h = A.gated_forward(x, wg, wu, "silu", saved=saved)
    within(h, f["h"], f["eh"], "h")
    p, r = saved.view(torch.float32).view(2, N, H)
    within(p, f["p"], f["ep"], "act(g)")
    within(r, f["u"] * f["r"], f["er"] * (np.abs(f["u"]) + f["eu"]) + np.abs(f["r"]) * f["eu"] + F.U32 * np.abs(f["u"] * f["r"]), "u act'(g)")


@pytest.mark.parametrize("N,K,H", [(8292, 512, 1160), (8192, 1024, 1408), (6500, 520, 1704), (2048, 2048, 4224)])
def test_gated_with_a_partly_filled_last_round_of_tiles(N, K, H):
    """More tiles than compute units: what is left over, by halves or in parts, row by row and column by column."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(N)
    x, wg, wu = (torch.randn(*s, device=DEV, generator=gen).mul_(v).bfloat16() for s, v in (((N, K), 1), ((K, H), K ** -0.5), ((K, H), K ** -0.5)))
    saved = A.gated_saved(x, wg)
    saved.view(torch.float32).fill_(float("nan"))
    out = torch.full((N, H), float("nan"), device=DEV).bfloat16()
    h = A.gated_forward(x, wg, wu, "silu", out=out, saved=saved)
    g, u = x.double() @ wg.double(), x.double() @ wu.double()
    s = torch.sigmoid(g)
    p, r = saved.view(torch.float32).view(2, N, H)
    # sums of K products of random signs in fp32 are off by about sqrt(K) roundings; an element's by 16 times that at most, relative to the row's and column's norms
    off = 16 * (K + 16) ** 0.5 * F.U32 * 1.2
    for name, got, want in (("P", p, g * s), ("R", r, u * s * (1 + g * (1 - s)))):
        assert bool(((got.double() - want).abs() <= off * (1 + want.abs()) * 8).all()), name
    want = g * s * u
    assert bool(((h.double() - want).abs() <= F.HALF["bf16"] * want.abs() + off * (1 + want.abs()) * 64).all())
    assert torch.equal(A.gated_forward(x, wg, wu, "silu"), h)
