"""The operators on sequences of tokens at the borders of what they take, against their definitions in 64 bits (token_formulas.py)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2404_09679_amd as A
import token_formulas as F

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def host(t):
    return t.double().cpu().numpy()


def within(got, want, bound, what):
    got = host(got) if torch.is_tensor(got) else got
    bad = ~(np.abs(got - want) <= bound) & ~(got == want)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3])


@pytest.mark.parametrize("N,K,H", [(1, 8, 16), (67, 200, 136), (777, 520, 328), (300, 1032, 2056)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_backward_of_one_side(dtype, N, K, H):
    """The gradient of x alone and those of the weights alone, which have plans of their own, in a workspace of the size reported."""
    rng = np.random.default_rng(N + H)
    x, wg, wu, dh = (torch.as_tensor(v).to(DEV, DT[dtype]) for v in (rng.normal(size=(N, K)), rng.normal(size=(K, H)) / K ** 0.5,
                                                                     rng.normal(size=(K, H)) / K ** 0.5, rng.normal(size=(N, H))))
    saved = A.gated_saved(x, wg)
    A.gated_forward(x, wg, wu, "silu", saved=saved)
    f = F.gated(host(x), host(wg), host(wu), "silu", F.HALF[dtype])
    want = F.gated_gradients(host(x), host(wg), host(wu), host(dh), f, F.HALF[dtype])
    code, n = {"f32": 0, "bf16": 1}[dtype], C.c_size_t()
    assert A.lib.antdt_gated_backward_bytes(N, K, H, code, C.byref(n)) == 0
    ws = torch.empty(n.value + 256, dtype=torch.uint8, device=DEV).fill_(255)
    for dx, dw in ((True, False), (False, True)):
        outs = [torch.full(s, 7.0, dtype=DT[dtype], device=DEV) for s in ((N, K), (K, H), (K, H))]
        p = [t.data_ptr() if w else None for t, w in zip(outs, (dx, dw, dw))]
        rc = A.lib.antdt_gated_backward(dh.data_ptr(), H, x.data_ptr(), K, wg.data_ptr(), wu.data_ptr(), H, N, K, H, code, saved.data_ptr(),
                                        p[0], K, p[1], p[2], H, ws.data_ptr(), n.value, torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        for name, t, w, (v, e) in zip(("dx", "dwg", "dwu"), outs, (dx, dw, dw), want):
            if w:
                within(t, v, e, (name, dx, dw))
            else:
                assert bool((t == 7).all())
        assert bool((ws[n.value:] == 255).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [8, 600, 20011])
@pytest.mark.parametrize("top", [0, 3])
def test_entropy_of_finite_logits_whose_differences_are_not(V, top, dtype):
    """The lowest value of the type as a mask beside a large logit: their difference overflows, and the term is 0."""
    rng = np.random.default_rng(V)
    x = rng.normal(size=(6, V))
    x[0], x[0, V // 2] = torch.finfo(DT[dtype]).min, 1e38
    x[1, 0], x[1, 1] = torch.finfo(DT[dtype]).min, 1e38
    x[2] = np.where(np.arange(V) % 2, -3e38, 3e38)
    x[3] = np.sign(x[3]) * 10.0 ** rng.uniform(30, 38.4, V)
    x[4] = torch.finfo(DT[dtype]).min
    x[5, V - 1] = torch.finfo(DT[dtype]).max
    dx = torch.as_tensor(x).to(DEV, DT[dtype])
    f = F.logprobs(host(dx), np.zeros(6, np.int64), top)
    r = A.token_logprobs(dx, None, top)
    bound = F.U32 * (f["depth"] + 4 * (4 + f["entropy"] * f["depth"]))
    within(r.entropy, f["entropy"], bound, "entropy")
    within(r.stats[:, 2], f["entropy"], bound, "stats")
    if top:
        assert np.array_equal(host(r.top_index).astype(np.int64), f["top_index"])
    b = rng.normal(size=6)
    db = torch.as_tensor(b, dtype=torch.float32, device=DEV)
    want, e = F.logprobs_gradient(f, np.full(6, -1), np.zeros(6), host(db))
    within(A.token_logprobs_gradient(dx, None, r.stats, None, db), want, e + F.HALF[dtype] * (np.abs(want) + e) + 1e-38, "gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 2, 9])
def test_slope_of_the_logistic_function_far_out(N, dtype):
    """s (1 - s) where s is 1 in fp32, relative to its own size.  With u = 2^-24: the exponential of an argument of |g| is off by (2 |g| + 2) u, the
    reciprocal of its sum with 1 by (|g| + 4) u, once in s and twice in the slope, and three products round."""
    g = np.array([-30, 17.5, 24, 60, -17, 8.25, 0, 40, -1.5])[:N]
    x = np.zeros((N, 8))
    x[:, 0], x[:, 1] = g, 1
    wg, wu = np.zeros((8, 16)), np.zeros((8, 16))
    wg[0], wu[1] = np.where(np.arange(16) % 2, -1, 1), 1          # g or -g, and u = 1
    x, wg, wu = (torch.as_tensor(v).to(DEV, DT[dtype]) for v in (x, wg, wu))
    saved = A.gated_saved(x, wg)
    A.gated_forward(x, wg, wu, "sigmoid", saved=saved)
    p, r = saved.view(torch.float32).view(2, N, 16)
    g = g[:, None] * np.where(np.arange(16) % 2, -1, 1)[None]
    s, rest = 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))
    within(p, s, (3 * np.abs(g) + 8) * F.U32 * s, "s")
    within(r, s * rest, (4 * np.abs(g) + 13) * F.U32 * s * rest, "slope")


def test_one_token_of_a_long_sequence():
    """x [1, K] out of [1, T, K] with T K beyond the leading dimensions that are taken, for one row has none."""
    T, K, H = 2100, 1024, 264
    x = torch.randn(1, T, K, device=DEV).bfloat16()[:, -1]
    wg, wu = (torch.randn(K, H, device=DEV).mul_(K ** -0.5).bfloat16() for _ in range(2))
    saved, dh = A.gated_saved(x, wg), torch.randn(1, H, device=DEV).bfloat16()
    h = A.gated_forward(x, wg, wu, saved=saved)
    assert torch.equal(h, A.gated_forward(x.contiguous(), wg, wu))
    for a, b in zip(A.gated_backward(dh, x, wg, wu, saved), A.gated_backward(dh, x.contiguous(), wg, wu, saved)):
        assert torch.equal(a, b)
