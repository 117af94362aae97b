"""Attention over a user's history at the largest sizes that it takes and over many users, against its definitions in 64 bits
(attention_formulas.py)."""
import ctypes as C

import numpy as np
import pytest
import torch

import attention_formulas as F
import paper_2404_09679_amd as A
from test_gpu_attention import DEV, check_cross, cross, host, within

pytestmark = pytest.mark.gpu


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
    border = 2 ** 22 // (S * HQ)                                  # (the entry that starts the launch's second row)
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
