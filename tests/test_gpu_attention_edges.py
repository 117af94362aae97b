"""Attention over a user's history at the borders of what it takes, against its definitions in 64 bits (attention_formulas.py)."""
import ctypes as C

import numpy as np
import pytest
import torch

import attention_formulas as F
import paper_2404_09679_amd as A
from test_gpu_attention import (DEV, DT, NAN, append_formula, cache_of, check_cross, check_decode, cross, cross_inputs, decode_inputs, host, ints,
                                normal, within)

pytestmark = pytest.mark.gpu


def pointers(*tensors):
    """(address, strides but the columns') of each, as the C boundary takes them."""
    return [x for t in tensors for x in (t.data_ptr(), *t.stride()[:-1])]


@pytest.mark.parametrize("B,S,T,HQ,H,D", [(2, 150, 210, 4, 2, 64), (1, 40, 1100, 2, 1, 96), (1, 1000, 40, 4, 1, 128), (9, 130, 140, 32, 32, 32)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_side_of_the_backward_pass_in_a_workspace_of_the_size_reported(B, S, T, HQ, H, D, dtype):
    rng = np.random.default_rng(S)
    q, k, v, g, ql, kl = cross_inputs(rng, B, S, T, HQ, H, D, "", dtype)
    want = cross(q, k, v, g, None, None)
    code, n, m = {"f32": 0, "bf16": 1}[dtype], C.c_size_t(), C.c_size_t()
    assert A.lib.antdt_cross_attention_bytes(B, S, T, HQ, H, D, code, C.byref(n)) == 0
    assert A.lib.antdt_cross_attention_backward_bytes(B, S, T, HQ, H, D, code, C.byref(m)) == 0
    ws = torch.empty(max(n.value, m.value) + 512, dtype=torch.uint8, device=DEV).fill_(255)       # (NaN wherever it is read unwritten)
    stats, out = torch.full((B, HQ, S), NAN, device=DEV), torch.full_like(q, 7.0)
    stream = torch.cuda.current_stream().cuda_stream
    sizes = (B, S, T, HQ, H, D, code, None, None, D ** -0.5)
    assert A.lib.antdt_cross_attention(*pointers(q, k, v), *sizes, *pointers(out), stats.data_ptr(), ws.data_ptr(), n.value, stream) == 0
    assert torch.equal(out, want[0]) and bool((ws[n.value:] == 255).all())
    for sides in ((True, False), (False, True), (True, True)):
        ws.fill_(255)
        d = [torch.full_like(x, 7.0) for x in (q, k, v)]
        p = [x if w else None for x, w in zip(d, (sides[0], sides[1], sides[1]))]
        at = [y for x, t in zip(p, d) for y in ((None, 0, 0, 0) if x is None else pointers(t))]
        assert A.lib.antdt_cross_attention_backward(*pointers(g, q, k, v, out), stats.data_ptr(), *sizes, *at, ws.data_ptr(), m.value, stream) == 0
        for x, w, t in zip(p, want[1:], d):
            assert torch.equal(t, w) if x is not None else bool((t == 7).all())
        assert bool((ws[m.value:] == 255).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", [[1], [4500], [3, 0, 900]])
def test_cache_attention_in_a_workspace_of_the_size_reported(lengths, dtype):
    rng = np.random.default_rng(len(lengths))
    B, HQ, H, D, page = len(lengths), 6, 2, 64, 16
    kc, vc, table = cache_of(rng, lengths, page, H, D, dtype)
    kc.copy_(normal(rng, *kc.shape, dtype=dtype)), vc.copy_(normal(rng, *vc.shape, dtype=dtype))
    q, code, n = normal(rng, B, HQ, D, dtype=dtype), {"f32": 0, "bf16": 1}[dtype], C.c_size_t()
    assert A.lib.antdt_cache_attention_bytes(B, HQ, H, D, code, C.byref(n)) == 0
    ws = torch.empty(n.value + 512, dtype=torch.uint8, device=DEV).fill_(255)
    want = A.cache_attention(q, kc, vc, ints(table), ints(lengths))
    assert torch.equal(A.cache_attention(q, kc, vc, ints(table), ints(lengths), workspace=ws[:n.value]), want)
    assert bool((ws[n.value:] == 255).all())


@pytest.mark.parametrize("S", [3, 70, 700])
def test_lengths_outside_the_sizes(S):
    rng = np.random.default_rng(S)
    q, k, v, g, _, _ = cross_inputs(rng, 4, S, 90, 2, 2, 32, "", "f32")
    ql, kl = [S, S + 5, -3, 2 ** 31 - 1], [2 ** 31 - 1, -2 ** 31, 90, 91]
    a = cross(q, k, v, g, ints(ql), ints(kl))
    b = cross(q, k, v, g, ints([S, S, 0, S]), ints([90, 0, 90, 90]))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert not a[0][1].any() and not a[0][2].any() and not a[2][1:3].any()


@pytest.mark.parametrize("S", [1, 200])
def test_scores_beyond_the_range(S):
    """Finite products of queries and keys whose scores are not: NaN, never a number."""
    q, k, v = torch.zeros(1, S, 2, 8, device=DEV), torch.zeros(1, 40, 2, 8, device=DEV), torch.randn(1, 40, 2, 8, device=DEV)
    q[..., 0], k[..., 0] = 2e19, 1e19
    assert bool(A.cross_attention(q, k, v, scale=4.0).isnan().all())
    q[0, 0, 0] = 0                                                # (that row's are)
    out = A.cross_attention(q, k, v, scale=4.0)
    within(out[0, 0, 0], host(v)[0, :, 0].mean(0), 48 * F.U * np.abs(host(v)[0, :, 0]).mean(0), "zeros")
    assert bool(out[0, :, 1].isnan().all())


@pytest.mark.parametrize("B,most", [(63, 5), (64, 5), (65, 4), (700, 3), (5000, 2)])
def test_cache_append_of_many_sequences(B, most):
    """Tokens that find their sequence among few and many offsets, sequences without new tokens among them."""
    rng = np.random.default_rng(B)
    new = rng.integers(0, most + 1, B)
    new[-1], new[0] = 0, 0
    lengths = new + rng.integers(0, 20, B) * (rng.random(B) < 0.8)
    page, H, D = 7, 1, 16
    kc, vc, table = cache_of(rng, lengths.tolist(), page, H, D, "f32")
    offsets = np.cumsum(np.concatenate([[0], new]))
    N = int(offsets[-1]) + 2
    k, v = (normal(rng, N, H, D) for _ in range(2))
    rot = A.Rotary(D, 100.0, device=DEV)
    want_k, want_v = kc.clone(), vc.clone()
    q = A.cache_append(k, v, kc, vc, ints(table), ints(lengths), ints(offsets), rot, k.clone())
    seq, pos = append_formula(lengths.tolist(), offsets, N)
    at = np.flatnonzero(pos >= 0)
    turned = A.rotary(k, ints(np.maximum(pos, 0)), rot)
    slot = [torch.as_tensor(x, device=DEV) for x in (table[seq[at], pos[at] // page], pos[at] % page)]
    want_k[slot[0], slot[1]], want_v[slot[0], slot[1]] = turned[at], v[at]
    assert torch.equal(kc.nan_to_num(9), want_k.nan_to_num(9)) and torch.equal(vc.nan_to_num(9), want_v.nan_to_num(9))
    assert torch.equal(q, torch.where(torch.as_tensor(pos >= 0, device=DEV)[:, None, None], turned, 0.0))


def test_positions_beyond_the_table():
    """Not appended, the query turned all the same; offsets that are none harm nobody."""
    rng = np.random.default_rng(2)
    kc, vc = (torch.full((4, 16, 1, 32), 5.0, device=DEV) for _ in range(2))
    table, k, q = ints([[0, 1], [2, 3], [1, 2]]), normal(rng, 3, 1, 32), normal(rng, 3, 2, 32)
    rot = A.Rotary(32, device=DEV)
    got = A.cache_append(k, k, kc, vc, table, ints([33, 2 ** 31 - 1, 0]), rotary=rot, q=q)
    assert bool((kc == 5).all()) and bool((vc == 5).all()) and not got[2].any()
    assert torch.equal(got[:2], A.rotary(q, ints([32, 2 ** 31 - 2, 0]), rot)[:2])
    for offsets in ([3, 2, 1, 0], [-5, 100, -7, 2 ** 31 - 1], [0, 0, 0, 0], [2 ** 31 - 1] * 4, [-2 ** 31] * 4):
        A.cache_append(k, k, kc, vc, table, ints([33, 40, 0]), ints(offsets), rot, q)
        torch.cuda.synchronize()


def test_keys_that_no_cache_holds():
    """More than 256 MB of keys and values, read past the caches."""
    rng = np.random.default_rng(4)
    T, H, D, page = 70_000, 8, 128, 64
    pages = -(-T // page)
    kc, vc = (torch.randn(pages, page, H, D, device=DEV).bfloat16() for _ in range(2))
    assert 2 * kc.numel() * 2 > 256 << 20
    table, q = torch.randperm(pages, device=DEV).int()[None], normal(rng, 1, 16, D, dtype="bf16", std=2.0)
    k, v = (x[table[0].long()].view(-1, H, D)[:T] for x in (kc, vc))
    check_decode(A.cache_attention(q, kc, vc, table, ints([T])), q, [(k, v)], "bf16", D ** -0.5, "")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_head_for_many(dtype):
    """64 heads of the queries on one of the keys, a query each and several."""
    rng = np.random.default_rng(6)
    for S in (1, 3):
        q, k, v, g, ql, kl = cross_inputs(rng, 2, S, 150, 64, 1, 40, "ragged", dtype)
        check_cross(cross(q, k, v, g, ints(ql), ints(kl)), q, k, v, g, ql, kl, 40 ** -0.5, dtype, S)


def test_two_calls_at_once():
    """Two streams at a time, each with tensors and workspaces of its own."""
    torch.manual_seed(3)
    jobs = [[torch.randn(2, n, 4, 64, device=DEV).bfloat16() for n in (260, 500, 500, 260)] for _ in range(2)]
    want = [cross(*j, None, None) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[] for _ in jobs]
    for _ in range(3):
        for i, (s, j) in enumerate(zip(streams, jobs)):
            with torch.cuda.stream(s):
                got[i] = cross(*j, None, None)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_of_no_sequence_at_all(dtype):
    rng = np.random.default_rng(5)
    kc, vc = (torch.full((2, 4, 1, 32), 5.0, device=DEV, dtype=DT[dtype]) for _ in range(2))
    k, q = normal(rng, 3, 1, 32, dtype=dtype), normal(rng, 3, 2, 32, dtype=dtype)
    for rot in (None, A.Rotary(32, device=DEV)):
        q_out = torch.full_like(q, 7.0)
        A.cache_append(k, k, kc, vc, torch.zeros(0, 2, dtype=torch.int32, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV), ints([0]), rot, q, q_out)
        assert not q_out.any() and bool((kc == 5).all()) and bool((vc == 5).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,S,T,HQ,H,D", [(37, 400, 512, 4, 2, 32), (16, 500, 700, 12, 6, 64), (50, 640, 384, 4, 1, 8)])
def test_entries_in_another_order(B, S, T, HQ, H, D, dtype):
    """More blocks than run at once, long and short entries: each has its results wherever in the batch it stands."""
    rng = np.random.default_rng(B)
    q, k, v, g, ql, kl = cross_inputs(rng, B, S, T, HQ, H, D, "ragged", dtype)
    kl[5] = kl[6] = kl[7]
    ql[9] = ql[8]
    for b in (5, 6, 8, 9):
        k[b].nan_to_num_(1.0), v[b].nan_to_num_(1.0), q[b].nan_to_num_(1.0), g[b].nan_to_num_(1.0)
    got = cross(q, k, v, g, ints(ql), ints(kl))
    check_cross([x[:12] for x in got], q[:12], k[:12], v[:12], g[:12], ql[:12], kl[:12], D ** -0.5, dtype, "")
    order = rng.permutation(B)
    other = cross(*(x[torch.as_tensor(order, device=DEV)] for x in (q, k, v, g)), ints(np.array(ql)[order]), ints(np.array(kl)[order]))
    assert all(torch.equal(x[torch.as_tensor(order, device=DEV)], y) for x, y in zip(got, other))
    full = [normal(rng, *x.shape, dtype=dtype) for x in (q, k, v, g)]
    assert all(torch.equal(x, y) for x, y in zip(cross(*full, None, ints([T] * B)), cross(*full, ints([S] * B), None)))


@pytest.mark.parametrize("S,far", [(3, 2 ** 22 - 16), (70, 2 ** 22), (70, 2 ** 22 - 16)])
def test_rows_far_apart(S, far):
    """Rows of 2^24 bytes and a little less from one to the next: offsets within a tile in 32 bits and in 64."""
    rng = np.random.default_rng(S)
    q, k, v, g, ql, kl = cross_inputs(rng, 1, S, 69, 2, 1, 32, "", "f32")
    want = cross(q, k, v, g, None, None)
    room = torch.empty(71, far, device=DEV)
    assert room.stride(0) == far
    q2, k2, v2, g2 = (room[:x.shape[1], i * 256:i * 256 + x[0, 0].numel()].view(1, x.shape[1], *x.shape[2:]).copy_(x) for i, x in enumerate((q, k, v, g)))
    assert all(torch.equal(x, y) for x, y in zip(cross(q2, k2, v2, g2, None, None), want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths,page,HQ,H,D", [([1, 64, 0, 33, 31], 16, 4, 4, 64), ([130, 7, 100], 5, 12, 2, 128), ([300, 299, 0, 1], 1, 66, 2, 32),
                                                 ([65] * 30, 32, 8, 1, 96), ([450, 12], 100, 3, 1, 8), ([40], 16, 40, 1, 40)])
def test_small_and_large_caches(lengths, page, HQ, H, D, dtype):
    """The same tokens in a cache with room for hardly more, and in tables of thousands of pages; some of the pages are none."""
    rng = np.random.default_rng(D)
    kc, vc, table, dense, q = decode_inputs(rng, lengths, page, HQ, H, D, dtype, std=2.0)
    gone = [(b, i) for b in range(len(lengths)) for i in range(-(-lengths[b] // page)) if lengths[b] > 64 and rng.random() < 0.2]
    for n, (b, i) in enumerate(gone):
        table[b, i] = (-1, len(kc), -2 ** 31, 2 ** 31 - 1)[n % 4]
    for b, n in enumerate(lengths):
        keep = torch.as_tensor([t for t in range(n) if (b, t // page) not in gone], dtype=torch.int64, device=DEV)
        dense[b] = tuple(x[keep] for x in dense[b])
    for cols in (0, 2050):
        wide = np.pad(table, ((0, 0), (0, max(0, cols - table.shape[1]))), constant_values=-1)
        got = A.cache_attention(q, kc, vc, ints(wide), ints(lengths))
        check_decode(got, q, dense, dtype, D ** -0.5, cols)
        assert torch.equal(A.cache_attention(q, kc, vc, ints(wide), ints(lengths), out=torch.full_like(q, 7.0)), got)
    k, v = (torch.randn(3, 16, H, D, device=DEV).to(kc.dtype) for _ in range(2))      # scores of -infinity and NaN
    k[0], k[2, 3] = -float("inf"), NAN
    q = q[:1].abs() + 0.5
    for cols in (3, 2050):
        t = np.full((1, cols), -1)
        t[0, :3] = [0, 1, 2]
        out = [A.cache_attention(q, k, v, ints(t), ints([n])) for n in (16, 32, 48)]
        assert not out[0].any() and bool(out[2].isnan().all())
        check_decode(out[1], q, [(k[1], v[1])], dtype, D ** -0.5, "infinity")
