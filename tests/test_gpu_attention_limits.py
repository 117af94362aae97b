"""Attention over a user's history at the largest sizes that it takes and over many users, against its definitions in 64 bits
(attention_formulas.py)."""
import ctypes as C

import numpy as np
import pytest
import torch

import attention_formulas as F
import paper_2404_09679_amd as A
from test_gpu_attention import (DEV, DT, NAN, check_cross, check_decode, cross, cross_inputs, decode_inputs, host, ints, normal,
                                within)

pytestmark = pytest.mark.gpu
INF = float("inf")


def check_entries(got, operands, ql, kl, entries, what):
    """check_cross of some entries of a batch; got: (out,) or with the gradients, operands: q, k, v, g."""
    at = torch.as_tensor(entries, device=DEV)
    check_cross([x[at] for x in got], *(x[at] for x in operands), [ql[b] for b in entries], [kl[b] for b in entries], operands[0].shape[3] ** -0.5, "bf16", what)


def test_more_queries_than_a_launch_has_threads_for():
    """2^25 queries of heads, joined by a block of 128 threads each: 2^32 threads."""
    B, S, T, HQ, H, D = 65536, 16, 100, 32, 4, 8
    n = C.c_size_t()
    assert A.lib.antdt_cross_attention_bytes(B, S, T, HQ, H, D, 1, C.byref(n)) == 0 and n.value > 0      # (equal shares and a join)
    assert B * S * HQ * 128 == 2 ** 32
    torch.manual_seed(1)
    q, k, v = (torch.randn(B, r, h, D, device=DEV, dtype=torch.bfloat16) for r, h in ((S, HQ), (T, H), (T, H)))
    kl = torch.randint(1, T + 1, (B,), device=DEV, dtype=torch.int32)
    kl[3] = kl[-2] = 0
    out = A.cross_attention(q, k, v, k_lengths=kl, out=torch.full_like(q, 7.0))
    lengths = kl.tolist()
    border = 2 ** 22 // (S * HQ)                                  # (the entry that a second launch starts with)
    check_entries([out], (q, k, v, q), [S] * B, lengths, [0, 1, 3, border - 1, border, border + 1, B // 2, B - 3, B - 2, B - 1], "entries")
    # every entry, from calls of a part of the batch: both are within two roundings of the largest value from the definition, and (scores of at most 70, from
    # operands below 5) 4096 u
    most = v.abs().amax(1).repeat_interleave(HQ // H, 1)[:, None].float()
    for b in range(0, B, 4096):
        part = slice(b, b + 4096)
        x = A.cross_attention(q[part], k[part], v[part], k_lengths=kl[part])
        assert bool(((x.float() - out[part].float()).abs() <= 2 * (2 * F.HALF["bf16"] + 4096 * F.U) * most[part]).all()), b


@pytest.mark.parametrize("B,S,T,HQ,H", [(2 ** 19, 1, 2, 16, 16), (2 ** 20, 1, 10, 8, 8), (2 ** 20 - 1, 2, 3, 15, 3)])
def test_gradients_of_more_blocks_than_a_launch_has_threads_for(B, S, T, HQ, H):
    """Blocks of keys and blocks of queries are 2^24 together, and more."""
    D = 8
    assert B * HQ < 2 ** 24 <= B * (HQ + H)
    torch.manual_seed(2)
    q, k, v, g = (torch.randn(B, r, h, D, device=DEV, dtype=torch.bfloat16) for r, h in ((S, HQ), (T, H), (T, H), (S, HQ)))
    kl = torch.randint(0, T + 1, (B,), device=DEV, dtype=torch.int32)
    ql = torch.randint(0, S + 1, (B,), device=DEV, dtype=torch.int32)
    kl[-1], ql[-1] = T, S
    got = cross(q, k, v, g, ql, kl)
    entries = [0, 1, 2, 3, B // 2 - 1, B // 2, B - 9, B - 3, B - 2, B - 1]
    check_entries(got, (q, k, v, g), ql.tolist(), kl.tolist(), entries, (B, T))
    # every entry, from calls of a part of the batch
    for b in range(0, B, 2 ** 17):
        part = slice(b, b + 2 ** 17)
        for x, y in zip(cross(q[part], k[part], v[part], g[part], ql[part], kl[part]), got):
            assert torch.equal(x, y[part]), b


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("S,T", [(1, 40), (200, 40), (1, 6000), (5, 9000)])
def test_scores_below_the_range(S, T, dtype):
    """Products of finite operands below fp32's range are -infinity: their keys have no weight, and a query that has no others has zeros and passes no
    gradient.  Where the scale takes the largest score there, NaN."""
    D, n = 8, C.c_size_t()
    assert A.lib.antdt_cross_attention_bytes(1, S, T, 2, 2, D, int(dtype is torch.bfloat16), C.byref(n)) == 0 and (n.value > 0) == (T > 40)
    torch.manual_seed(S)
    q, k = torch.zeros(1, S, 2, D, device=DEV, dtype=dtype), torch.zeros(1, T, 2, D, device=DEV, dtype=dtype)
    v, g = (torch.randn(1, r, 2, D, device=DEV).to(dtype) for r in (T, S))
    q[..., 0], k[..., 0] = -2e19, 2e19
    stats = A.cross_attention_stats(q)
    out = A.cross_attention(q, k, v, stats=stats, out=torch.full_like(q, 7.0))
    assert not out.any() and bool((stats == float("inf")).all())
    assert not any(x.any() for x in A.cross_attention_backward(g, q, k, v, out, stats))
    some = torch.rand(T, device=DEV) < 0.3                        # (scores of 0)
    k[0, some] = 0
    got = cross(q, k, v, g, None, None)
    x = host(v)[0, some.cpu().numpy()]
    e = (len(x) + 8) * F.U * np.abs(x).mean(0)
    half = F.HALF["bf16"] if dtype is torch.bfloat16 else F.HALF["f32"]
    want = np.broadcast_to(x.mean(0), got[0][0].shape)
    within(got[0][0], want, e + half * (np.abs(want) + e), "the others' mean")
    assert all(bool(x.isfinite().all()) for x in got) and not got[3][0, ~some].any()
    k[..., 0] = 1e19                                              # (products of -2e38)
    assert bool(A.cross_attention(q, k, v, scale=4.0).isnan().all())


TWO_PARTS = 2.0 ** -15                                            # a bf16 number cut off takes 2^-7 away, of which rounding loses 2^-8


def check_two_parts(got, q, k, v, scale, what):
    """Rows q [S, D], got [S, D] of a head over k, v [T, D], all of bf16: only the result is rounded to bf16."""
    f = F.attend(host(q), host(k), host(v), scale, TWO_PARTS)
    within(host(got), f["out"], f["e"] + F.HALF["bf16"] * (np.abs(f["out"]) + f["e"]), what)


@pytest.mark.parametrize("lengths,page,HQ,H,D", [([100, 33, 64, 7], 16, 4, 2, 64), ([500, 90], 7, 40, 2, 128), ([300, 0, 70], 64, 8, 8, 96), ([150, 0, 31], 16, 4, 1, 40),
                                                 ([130] * 40, 16, 3, 1, 32)])
@pytest.mark.parametrize("room", [0, 2050])
def test_probabilities_over_a_cache_are_not_rounded_to_bf16(lengths, page, HQ, H, D, room):
    rng = np.random.default_rng(D)
    kc, vc, table, dense, q = decode_inputs(rng, lengths, page, HQ, H, D, "bf16")
    table = np.pad(table, ((0, 0), (0, max(0, room - table.shape[1]))), constant_values=-1)
    got = A.cache_attention(q, kc, vc, ints(table), ints(lengths))
    for b, (k, v) in enumerate(dense):
        for h in range(H):
            of = slice(h * HQ // H, (h + 1) * HQ // H)
            check_two_parts(got[b, of], q[b, of], k[:, h], v[:, h], D ** -0.5, (b, h))


@pytest.mark.parametrize("S,T,HQ,H,D", [(1, 6000, 4, 4, 64), (3, 9000, 8, 2, 128), (17, 9000, 4, 2, 96)])
def test_probabilities_of_few_queries_are_not_rounded_to_bf16(S, T, HQ, H, D):
    n = C.c_size_t()
    assert A.lib.antdt_cross_attention_bytes(2, S, T, HQ, H, D, 1, C.byref(n)) == 0 and n.value > 0      # (equal shares)
    rng = np.random.default_rng(T)
    q, k, v, _, _, _ = cross_inputs(rng, 2, S, T, HQ, H, D, "", "bf16")
    kl = [200, 63]                                                # (of few terms: the bound on sums' rounding stays below that on the probabilities')
    got = A.cross_attention(q, k, v, k_lengths=ints(kl))
    for b in range(2):
        for h in range(HQ):
            check_two_parts(got[b, :, h], q[b, :, h], k[b, :kl[b], h * H // HQ], v[b, :kl[b], h * H // HQ], D ** -0.5, (b, h))


@pytest.mark.parametrize("S,T", [(1, 40), (1, 6000), (20, 9000), (0, 60), (0, 5000)])
def test_infinite_values(S, T):
    """A value's infinity is the result's, of one sign; S = 0: over a cache.  Probabilities that bf16 holds and such that it does not."""
    rng = np.random.default_rng(T)
    H, D = 2, 64
    q, k, v, _, _, _ = cross_inputs(rng, 1, max(S, 1), T, H, H, D, "", "bf16")
    k[0, ::2] = 0
    v[0, 7, 0, 3], v[0, 8, 0, 5], v[0, 8, 1, 9], v[0, 30, 1, 9] = INF, -INF, INF, -INF
    if S:
        out = A.cross_attention(q, k, v)[0]
    else:
        out = A.cache_attention(q[0], k, v, ints([[0]]), ints([T]))
    inf = torch.zeros(H, D, device=DEV)
    inf[0, 3], inf[0, 5], inf[1, 9] = INF, -INF, float("nan")
    for row in out.float():
        assert torch.equal(torch.where(row.isfinite(), 0, row).nan_to_num(9, INF, -INF), inf.nan_to_num(9, INF, -INF))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,page,cols,HQ,H,D", [(1, 32, 1, 8, 8, 64), (7, 16, 2, 6, 2, 128), (70, 5, 6, 40, 1, 24), (200, 1, 3, 8, 2, 64), (16, 7, 1, 4, 4, 96),
                                                (3, 33, 1, 4, 2, 40)])
def test_caches_of_one_tile(B, page, cols, HQ, H, D, dtype):
    """Room for at most 32 tokens, and one more; pages that there are not, lengths of 0 and beyond the room."""
    rng = np.random.default_rng(B + page)
    room = page * cols
    lengths = rng.integers(0, room + 1, B).tolist()
    lengths[-1] = room
    kc, vc, table, dense, q = decode_inputs(rng, lengths, page, HQ, H, D, dtype)
    table = np.pad(table, ((0, 0), (0, cols - table.shape[1])), constant_values=-1)
    gone = rng.integers(0, B)
    if B > 1 and lengths[gone] > page:
        table[gone, 0] = len(kc)
        dense[gone] = tuple(x[page:] for x in dense[gone])
    given = [n + 1000 if n == room else n - 5 if n == 0 else n for n in lengths]
    got = A.cache_attention(q, kc, vc, ints(table), ints(given), out=torch.full_like(q, 7.0))
    check_decode(got, q, dense, dtype, D ** -0.5, "")
    wide = np.pad(table, ((0, 0), (0, 2050)), constant_values=-1)
    check_decode(A.cache_attention(q, kc, vc, ints(wide), ints(lengths)), q, dense, dtype, D ** -0.5, "in a large table")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,longest,page,HQ,H,D", [(1000, 90, 16, 4, 2, 32), (4097, 40, 5, 2, 1, 16), (20000, 9, 4, 3, 1, 8)])
def test_caches_of_many_users(B, longest, page, HQ, H, D, dtype):
    """Several sequences to a lane of the wavefronts that look for theirs; many without tokens, alone and side by side."""
    rng = np.random.default_rng(B)
    lengths = rng.integers(0, longest + 1, B)
    lengths[rng.random(B) < 0.3] = 0
    lengths[100:400] = lengths[-50:] = 0
    pages = -(-lengths // page)
    order, start = rng.permutation(int(pages.sum())), np.cumsum(pages) - pages
    table = np.full((B, -(-longest // page)), -1)
    for b in range(B):
        table[b, :pages[b]] = order[start[b]:start[b] + pages[b]]
    kc, vc = (torch.full((len(order), page, H, D), NAN, device=DEV, dtype=DT[dtype]) for _ in range(2))
    seq = np.repeat(np.arange(B), lengths)
    t = np.arange(len(seq)) - np.repeat(np.cumsum(lengths) - lengths, lengths)
    slot = torch.as_tensor(table[seq, t // page], device=DEV), torch.as_tensor(t % page, device=DEV)
    dense = torch.zeros(2, B, longest, H, D, device=DEV, dtype=torch.float64)
    for c, x in zip((kc, vc), dense):
        c[slot] = normal(rng, len(seq), H, D, dtype=dtype)
        x[torch.as_tensor(seq, device=DEV), torch.as_tensor(t, device=DEV)] = c[slot].double()
    q = normal(rng, B, HQ, D, dtype=dtype)
    got = A.cache_attention(q, kc, vc, ints(table), ints(lengths), out=torch.full_like(q, 7.0))
    some = np.flatnonzero(lengths)[[0, 1, 2, 30, 300, -3, -2, -1]]
    check_decode(got[torch.as_tensor(some, device=DEV)], q[torch.as_tensor(some, device=DEV)], [tuple(x[b, :lengths[b]] for x in dense) for b in some], dtype,
                 D ** -0.5, "some")
    # all of them in 64 bits, and the bound with the largest values in the place of their mean: scores of at most 70, as in attention_formulas.attend
    k, v = (x.repeat_interleave(HQ // H, 2) for x in dense)
    z = torch.where(torch.arange(longest, device=DEV)[None, None] < ints(lengths)[:, None, None], (q.double()[:, None] * k).sum(3).transpose(1, 2) * D ** -0.5, -INF)
    want = (torch.softmax(z, 2).nan_to_num(0)[..., None] * v.transpose(1, 2)).sum(2)
    e = ((2 * (D + 14) * 70 + longest + 16) * F.U + (TWO_PARTS if dtype == "bf16" else 0)) * v.abs().amax(1) + F.HALF[dtype] * (want.abs() * 1.01)
    assert float(z[z > -INF].abs().max()) < 70
    assert bool(((got.double() - want).abs() <= e).all())
    assert torch.equal(A.cache_attention(q, kc, vc, ints(table), ints(lengths)), got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,S,T,HQ,H,D", [(3000, 2, 40, 4, 1, 16), (1100, 1, 300, 2, 2, 32), (700, 40, 33, 2, 1, 8)])
def test_many_histories(B, S, T, HQ, H, D, dtype):
    rng = np.random.default_rng(B)
    q, k, v, g = (normal(rng, B, n, h, D, dtype=dtype) for n, h in ((S, HQ), (T, H), (T, H), (S, HQ)))
    ql, kl = rng.integers(0, S + 1, B), rng.integers(0, T + 1, B)
    kl[rng.random(B) < 0.3] = 0
    ql[-1], kl[-1], kl[60:200] = S, T, 0
    for x, n in ((q, ql), (g, ql), (k, kl), (v, kl)):
        x[torch.arange(x.shape[1], device=DEV)[None] >= ints(n)[:, None]] = NAN
    got = cross(q, k, v, g, ints(ql), ints(kl))
    at = np.concatenate([np.arange(64), np.arange(B // 2, B // 2 + 32), np.arange(B - 64, B), rng.choice(B, 100, False)])
    on = torch.as_tensor(at, device=DEV)
    check_cross([x[on] for x in got], q[on], k[on], v[on], g[on], ql[at].tolist(), kl[at].tolist(), D ** -0.5, dtype, "")
    assert not any(bool(x.isnan().any()) for x in got)
    for x, n in zip(got, (ql, ql, kl, kl)):
        assert not x[torch.arange(x.shape[1], device=DEV)[None] >= ints(n)[:, None]].any()
    assert all(torch.equal(x, y) for x, y in zip(cross(q, k, v, g, ints(ql), ints(kl)), got))
