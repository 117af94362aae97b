"""Attention over a user's history without a GPU: what the calls refuse, sizes they report, the frequencies, what the binding does around the
calls, and the formulas of the GPU tests against differences."""
import ctypes as C
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

import attention_formulas as F
from test_token_binding_host import Boundary

A = pytest.importorskip("paper_2404_09679_amd", reason="build the library first (python paper_2404_09679_amd/build.py)")
lib, T = A.lib, A.attention
OK, INVALID, SMALL, UNSUPPORTED = 0, -1, -3, -5
PTR = 1 << 20            # an address that the checks accept and nothing reads
ROT = A.Rotary(8, device="cpu")


def message():
    return lib.antdt_last_error(None).decode()


def turns(dim, base=10000.0, factor=1.0, original=0.0, low=0.0, high=0.0):
    out = (C.c_uint64 * max(dim // 2, 1))()
    rc = lib.antdt_rotary_turns(dim, base, factor, original, low, high, out)
    return rc or list(out)


@pytest.mark.parametrize("dim,base,factor,original,low,high", [(64, 10000.0, 1.0, 0, 0, 0), (128, 500000.0, 8.0, 8192, 1.0, 4.0), (36, 10000.0, 16.0, 4096, 1, 32),
                                                               (256, 1e6, 2.5, 0, 0, 0), (2, 1.0, 1.0, 0, 0, 0)])
def test_frequencies(dim, base, factor, original, low, high):
    """To what a double's power, quotient and products lose: eight halves of its last place."""
    getcontext().prec = 50
    two_pi = 2 * Decimal("3.14159265358979323846264338327950288419716939937510")
    for i, t in enumerate(turns(dim, base, factor, original, low, high)):
        f = (Decimal(base).ln() * Decimal(-2 * i) / dim).exp() / two_pi
        keep = min(Decimal(1), max(Decimal(0), (f * Decimal(original) - Decimal(low)) / (Decimal(high) - Decimal(low)))) if high else Decimal(0)
        want = f * (keep + (1 - keep) / Decimal(factor)) * 2 ** 64
        # (the mixture's slope: an error of f counts up to original / (high - low) times, relative to the whole)
        assert abs(Decimal(t) - want) <= want * Decimal(2.0 ** -53) * 8 * (1 + (int(factor) if high else 0)) + 1


def test_frequency_refusals():
    assert turns(64, high=4.0, low=1.0, original=4096.0, factor=8.0) != INVALID
    for kw in (dict(dim=0), dict(dim=7), dict(dim=258), dict(dim=8, base=0.5), dict(dim=8, base=float("inf")), dict(dim=8, base=float("nan")),
               dict(dim=8, factor=0.5), dict(dim=8, factor=float("nan")), dict(dim=8, factor=2.0, low=4.0, high=1.0, original=10.0),
               dict(dim=8, factor=2.0, low=-1.0, high=1.0, original=10.0), dict(dim=8, low=1.0, high=2.0, original=0.0), dict(dim=8, high=float("nan"))):
        assert turns(**kw) == INVALID, kw
    assert lib.antdt_rotary_turns(8, 2.0, 1.0, 0.0, 0.0, 0.0, None) == INVALID
    for kw in (dict(dim=7), dict(dim=8, factor=0.0), dict(dim=-2)):
        with pytest.raises(A.AntdtError, match="antdt_rotary_turns"):
            A.Rotary(device="cpu", **kw)


def spec(dim=8, interleaved=0, magnitude=1.0, where=PTR):
    return C.byref(A.binding.RotarySpec(dim, interleaved, magnitude, where))


def test_rotary_refusals():
    def call(x=PTR, ldx=32, ldh=8, N=3, H=4, D=8, dtype=0, p=PTR, rot=None, y=2 * PTR, ldy=32, ldyh=8):
        return lib.antdt_rotary(x, ldx, ldh, N, H, D, dtype, p, rot or spec(), 0, y, ldy, ldyh, None)

    assert call(dtype=2) == INVALID and call(x=None) == INVALID and call(y=None) == INVALID and call(p=None) == INVALID
    assert call(x=PTR + 2) == INVALID and call(p=PTR + 2) == INVALID
    for rot in (spec(dim=10), spec(dim=0), spec(dim=3), spec(interleaved=2), spec(magnitude=float("inf")), spec(where=None), spec(where=PTR + 4)):
        assert call(rot=rot) == INVALID and "rotary" in message()
    assert lib.antdt_rotary(PTR, 32, 8, 3, 4, 8, 0, PTR, None, 0, PTR, 32, 8, None) == INVALID
    assert call(N=-1) == INVALID and call(N=2 ** 31) == INVALID and call(H=65537) == INVALID and call(D=257) == INVALID
    # results that would share memory, operands of negative stride
    assert call(ldy=31) == INVALID and call(ldyh=7) == INVALID and call(ldy=0) == INVALID and call(ldx=-1) == INVALID
    assert call(N=0, x=None, y=None) == OK and call(H=0, x=None, y=None) == OK and call(D=0, x=None) == OK


def test_cache_append_refusals():
    def call(q=PTR, qo=2 * PTR, k=PTR, v=PTR, N=3, HQ=4, H=2, D=8, dtype=0, rot=None, kc=3 * PTR, vc=4 * PTR, lp=256, lr=16, lh=8, pages=5, page=16, table=PTR,
             ldt=7, B=3, W=7, lengths=PTR, offsets=None, ldqo=32):
        return lib.antdt_cache_append(q, 32, 8, qo, ldqo, 8, k, 16, 8, v, 16, 8, N, HQ, H, D, dtype, rot, kc, vc, lp, lr, lh, pages, page, table, ldt, B, W, lengths,
                                      offsets, None)

    assert call(dtype=5) == INVALID
    for name in ("q", "qo", "k", "v", "kc", "vc", "table", "lengths"):
        assert call(**{name: None}) == INVALID, name
    assert call(N=4) == INVALID and "a token for each" in message()
    assert call(offsets=PTR + 2) == INVALID and call(page=0) == INVALID and call(page=2 ** 31) == INVALID and call(pages=-1) == INVALID and call(W=-1) == INVALID
    assert call(ldt=6) == INVALID and call(lp=255) == INVALID and call(lr=15) == INVALID and call(lh=7) == INVALID and call(ldqo=8) == INVALID
    assert call(D=300) == INVALID and call(rot=spec(dim=10)) == INVALID and call(lengths=PTR + 1) == INVALID
    assert call(N=0, B=0, k=None, table=None) == OK and call(HQ=0, H=0) == OK


def test_cache_attention_refusals():
    n = C.c_size_t()
    assert lib.antdt_cache_attention_bytes(3, 4, 2, 64, 1, C.byref(n)) == OK and n.value > 0
    need = n.value
    assert lib.antdt_cache_attention_bytes(0, 4, 2, 64, 1, C.byref(n)) == OK and n.value == 0
    assert lib.antdt_cache_attention_bytes(3, 4, 2, 64, 1, None) == INVALID and lib.antdt_cache_attention_bytes(-1, 4, 2, 64, 1, C.byref(n)) == UNSUPPORTED
    assert lib.antdt_cache_attention_bytes(1 << 22, 4, 2, 64, 1, C.byref(n)) == UNSUPPORTED

    def call(q=PTR, ldq=256, ldqh=64, kc=PTR, vc=PTR, lp=2048, lr=128, lh=64, pages=5, page=16, table=PTR, ldt=7, B=3, W=7, lengths=PTR, HQ=4, H=2, D=64, dtype=1,
             scale=0.125, out=2 * PTR, ldo=256, ldoh=64, ws=PTR, size=1 << 30):
        return lib.antdt_cache_attention(q, ldq, ldqh, kc, vc, lp, lr, lh, pages, page, table, ldt, B, W, lengths, HQ, H, D, dtype, scale, out, ldo, ldoh, ws, size, None)

    for name in ("q", "kc", "vc", "table", "lengths", "out", "ws"):
        assert call(**{name: None}) == INVALID, name
    assert call(dtype=3) == INVALID and call(H=3) == INVALID and "heads" in message() and call(H=0) == INVALID and call(HQ=0) == INVALID
    assert call(D=12) == UNSUPPORTED and call(D=136) == UNSUPPORTED and call(D=0) == UNSUPPORTED
    assert call(q=PTR + 8) == UNSUPPORTED and call(ldq=260) == UNSUPPORTED and call(lr=132, lp=132 * 16) == UNSUPPORTED and "16 bytes" in message()
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(scale=scale) == INVALID and "scale" in message()
    assert call(page=0) == INVALID and call(pages=-1) == INVALID and call(ldo=255) == INVALID and call(ldoh=32) == INVALID and call(ldt=6) == INVALID
    assert call(size=need - 1) == SMALL and call(ws=PTR + 128) == INVALID
    assert call(B=0, q=None, out=None, table=None, lengths=None, ws=None, size=0) == OK


@pytest.mark.parametrize("dtype", [0, 1])
def test_cross_attention_refusals(dtype):
    n = C.c_size_t()
    for f in (lib.antdt_cross_attention_bytes, lib.antdt_cross_attention_backward_bytes):
        assert f(2, 300, 500, 4, 2, 64, dtype, C.byref(n)) == OK and f(2, 300, 500, 4, 2, 64, dtype, None) == INVALID
        assert f(2, 300, 500, 4, 3, 64, dtype, C.byref(n)) == INVALID and f(2, 300, 500, 4, 2, 60, dtype, C.byref(n)) == UNSUPPORTED
        assert f(2, -1, 500, 4, 2, 64, dtype, C.byref(n)) == INVALID and f(2, 5, 2 ** 31, 4, 2, 64, dtype, C.byref(n)) == INVALID
        assert f(1 << 22, 5, 5, 4, 2, 64, dtype, C.byref(n)) == UNSUPPORTED and f(2, 300, 500, 4, 2, 64, 2, C.byref(n)) == INVALID
    q_ld, k_ld = [64 * 4 * 300, 64 * 4, 64], [64 * 2 * 500, 64 * 2, 64]
    tail = dict(ql=PTR, kl=PTR, scale=0.125, ws=PTR, size=1 << 34, S=300, D=64, dt=dtype)

    def fwd(q=PTR, k=PTR, v=PTR, out=2 * PTR, stats=PTR, q_ld=q_ld, k_ld=k_ld, o_ld=q_ld, **kw):
        a = dict(tail, **kw)
        return lib.antdt_cross_attention(q, *q_ld, k, *k_ld, v, *k_ld, 2, a["S"], 500, 4, 2, a["D"], a["dt"], a["ql"], a["kl"], a["scale"], out, *o_ld, stats,
                                         a["ws"], a["size"], None)

    def bwd(g=PTR, q=PTR, k=PTR, v=PTR, out=PTR, stats=PTR, dq=2 * PTR, dk=3 * PTR, dv=4 * PTR, d_ld=q_ld, dk_ld=k_ld, **kw):
        a = dict(tail, **kw)
        return lib.antdt_cross_attention_backward(g, *q_ld, q, *q_ld, k, *k_ld, v, *k_ld, out, *q_ld, stats, 2, a["S"], 500, 4, 2, a["D"], a["dt"], a["ql"], a["kl"],
                                                  a["scale"], dq, *d_ld, dk, *dk_ld, dv, *dk_ld, a["ws"], a["size"], None)

    for name in ("q", "k", "v", "out"):
        assert fwd(**{name: None}) == INVALID, name
    for name in ("g", "q", "k", "v", "out", "stats", "dk", "dv", "ws"):
        assert bwd(**{name: None}) == INVALID, name
    for f in (fwd, bwd):
        assert f(ql=PTR + 2) == INVALID and f(kl=PTR + 1) == INVALID and f(scale=-1.0) == INVALID and f(scale=0.0) == INVALID and f(dt=4) == INVALID
        assert f(D=20) == UNSUPPORTED and f(S=-1) == INVALID
    assert fwd(q_ld=[64 * 4 * 300, 64 * 4 + 2, 64]) == UNSUPPORTED and fwd(k=PTR + 4) == UNSUPPORTED and fwd(o_ld=[0, 256, 64]) == INVALID
    assert fwd(o_ld=[64 * 4 * 300 - 64, 256, 64]) == INVALID and fwd(stats=PTR + 2) == INVALID and fwd(q_ld=[-16, 256, 64]) == INVALID
    assert bwd(d_ld=[0, 0, 64]) == INVALID and bwd(dk_ld=[64 * 2 * 500, 64, 64]) == INVALID and bwd(size=64) == SMALL
    assert fwd(S=0, q=None, out=None) == OK and bwd(dq=None, dk=None, dv=None) == OK


def test_sizes_of_workspaces():
    """Whatever the sizes, also none at all."""
    rng, n = np.random.default_rng(1), C.c_size_t()
    for _ in range(4000):
        B, S, T_ = (int(10 ** rng.uniform(0, 4)) * int(rng.random() > 0.1) for _ in range(3))
        H, D, dtype = int(rng.integers(1, 9)), 8 * int(rng.integers(1, 17)), int(rng.integers(0, 2))
        HQ = H * int(rng.integers(1, 9))
        for f in (lib.antdt_cross_attention_bytes, lib.antdt_cross_attention_backward_bytes):
            rc = f(B, S, T_, HQ, H, D, dtype, C.byref(n))
            assert rc == OK or (rc == UNSUPPORTED and B * HQ * (max(S, T_) / 128 + 1) >= 1 << 24), (B, S, T_, HQ, H, D, message())
            # d of the rows, or two parts of 32 rows of 128 columns, a maximum and a sum for each of 2048 wavefronts, and a word for each sequence
            assert rc or n.value <= 4 * B * S * HQ + 2048 * 2 * 32 * (128 * 4 + 8) + 4 * B + 512
    assert lib.antdt_cross_attention_bytes(0, 0, 0, 1, 1, 8, 0, C.byref(n)) == OK and n.value == 0


def test_formulas_against_differences():
    rng = np.random.default_rng(3)
    q, k, v, g = rng.normal(size=(4, 6)), rng.normal(size=(9, 6)), rng.normal(size=(9, 6)), rng.normal(size=(4, 6))
    f = F.attend(q, k, v, 0.7, 0)
    assert np.allclose(f["p"].sum(1), 1) and np.allclose(2.0 ** -f["L"][:, 0] * np.exp(0.7 * (q @ k.T)).sum(1), 1)
    for i, (d, _) in enumerate(F.attend_gradients(q, k, v, g, 0.7, f, 0, 0)):
        way, eps = rng.normal(size=d.shape), 1e-6
        up, down = ((F.attend(*[a + s * eps * way if j == i else a for j, a in enumerate((q, k, v))], 0.7, 0)["out"] * g).sum() for s in (1, -1))
        assert abs((up - down) / (2 * eps) - (d * way).sum()) < 1e-7, i
    x, t = rng.normal(size=(3, 2, 8)), [2 ** 61, 2 ** 40 + 12345, 7]
    y, _ = F.rotate(x, [1, -5, 2 ** 31 - 1], t, False, 1.5)
    assert np.allclose(y[0, :, 0], -1.5 * (x[0, :, 3] - x[0, :, 0]) / 2 ** 0.5) and np.array_equal(y[..., 6:], x[..., 6:])
    back, _ = F.rotate(y, [1, -5, 2 ** 31 - 1], t, False, 1 / 1.5, True)
    assert np.allclose(back, x)


# ------------------------------------------------------------------ around the calls
@pytest.fixture
def boundary(monkeypatch):
    b = Boundary()
    monkeypatch.setattr(T, "lib", b)
    monkeypatch.setattr(T, "_bytes", lambda call, *sizes: 4096)
    monkeypatch.setattr(T, "_stream", lambda device: 0)
    monkeypatch.setattr(T, "_current_device", lambda: b.device)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: b.on)

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, b.device = b.device, self.index

        def __exit__(self, *_):
            b.device = self.before

    monkeypatch.setattr(torch.cuda, "device", Device)
    return b


def operators():
    """Every operator once, by name: a function that calls it."""
    x, kv = torch.zeros(4, 3, 8), torch.zeros(2, 5, 3, 8)
    cache, table, i4 = torch.zeros(6, 16, 3, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    rot, stats, q = ROT, torch.zeros(2, 3, 4), torch.zeros(2, 4, 3, 8)
    return {"antdt_rotary": lambda: A.rotary(x, i4, rot),
            "antdt_cache_append": lambda: A.cache_append(x, x, cache, cache, table, i4, rotary=rot, q=x),
            "antdt_cache_attention": lambda: A.cache_attention(x, cache, cache, table, i4),
            "antdt_cross_attention": lambda: A.cross_attention(q, kv, kv, stats=stats),
            "antdt_cross_attention_backward": lambda: A.cross_attention_backward(q, q, kv, kv, q, stats)}


@pytest.mark.parametrize("name", list(operators()))
def test_kernels_go_to_the_operands_device(boundary, name):
    call, seen = operators()[name], []
    boundary.during = lambda: seen.append(boundary.device)
    for current, on in ((0, 0), (0, 1), (2, 0)):
        boundary.device, boundary.on = current, on
        call()
        assert [n for n, _ in boundary.calls] == [name] and seen.pop() == on and boundary.device == current
        boundary.calls.clear()


@pytest.mark.parametrize("name", [n for n in operators() if "attention" in n])
def test_buffers_live_until_the_call_returns(boundary, monkeypatch, name):
    import weakref

    made, seen = [], []
    for module, which in ((T, "_new"), (A.tokens, "_new")):
        def noted(*args, new=getattr(module, which)):
            out = new(*args)
            made.append(weakref.ref(out))
            return out
        monkeypatch.setattr(module, which, noted)
    call = operators()[name]
    boundary.during = lambda: seen.append([r() is not None for r in made])
    call()
    assert len(made) >= 2 and seen == [[True] * len(made)]


def test_refusals_of_tensors(boundary, monkeypatch):
    x, i4, rot = torch.zeros(4, 3, 8), torch.zeros(4, dtype=torch.int32), ROT
    cache, table = torch.zeros(6, 16, 3, 8), torch.zeros(4, 2, dtype=torch.int32)
    q, kv, stats = torch.zeros(2, 4, 3, 8), torch.zeros(2, 5, 3, 8), torch.zeros(2, 3, 4)
    t = torch
    for call in (
            lambda: A.rotary(x[0], i4, rot), lambda: A.rotary(x.half(), i4, rot), lambda: A.rotary(x, i4[:3], rot), lambda: A.rotary(x, i4.long(), rot),
            lambda: A.rotary(x.transpose(1, 2), i4, rot), lambda: A.rotary(x, i4, rot, out=x.bfloat16()), lambda: A.rotary(x, i4, rot, out=x[:3]),
            lambda: A.cache_append(x, x[:, :2], cache, cache, table, i4), lambda: A.cache_append(x, x, cache[0], cache[0], table, i4),
            lambda: A.cache_append(x, x, cache.bfloat16(), cache, table, i4), lambda: A.cache_append(x, x, cache, cache[:, :15], table, i4),
            lambda: A.cache_append(x, x, cache, cache.transpose(1, 2).contiguous().transpose(1, 2), table, i4),
            lambda: A.cache_append(x, x, cache[..., :2, :], cache[..., :2, :], table, i4), lambda: A.cache_append(x, x, cache, cache, table.long(), i4),
            lambda: A.cache_append(x, x, cache, cache, table[0], i4), lambda: A.cache_append(x, x, cache, cache, table, i4[:2]),
            lambda: A.cache_append(x, x, cache, cache, table, i4, offsets=i4), lambda: A.cache_append(x, x, cache, cache, table, i4, q_out=x),
            lambda: A.cache_append(x, x, cache, cache, table, i4, q=x[:3]), lambda: A.cache_append(x, x, cache, cache, table, i4, q=x[0]),
            lambda: A.cache_attention(x[:3], cache, cache, table, i4), lambda: A.cache_attention(x[..., :4], cache, cache, table, i4),
            lambda: A.cache_attention(x, cache, cache, table, i4, out=x[:2]), lambda: A.cache_attention(x, cache, cache, table.t(), i4),
            lambda: A.cross_attention(q[0], kv, kv), lambda: A.cross_attention(q, kv[:1], kv), lambda: A.cross_attention(q, kv, kv[:, :4]),
            lambda: A.cross_attention(q, kv, kv, stats=stats[:1]), lambda: A.cross_attention(q, kv, kv, stats=stats.transpose(1, 2)),
            lambda: A.cross_attention(q, kv, kv, k_lengths=i4), lambda: A.cross_attention(q, kv.bfloat16(), kv),
            lambda: A.cross_attention_backward(q[:1], q, kv, kv, q, stats), lambda: A.cross_attention_backward(q, q, kv, kv, q, t.zeros(2, 4, 3)),
            lambda: A.cross_attention_backward(q, q, kv, kv, q, stats, dk=q), lambda: A.cross_attention_stats(q[0])):
        with pytest.raises(ValueError):
            call()
    assert not boundary.calls
    monkeypatch.setattr(torch.Tensor, "get_device", lambda s: 1 if s.dtype == torch.int64 else 0)
    with pytest.raises(ValueError, match="Rotary"):
        A.rotary(x, i4, rot)


def test_the_largest_scale():
    def call(scale):
        return lib.antdt_cross_attention(PTR, 0, 64, 64, PTR, 0, 64, 64, PTR, 0, 64, 64, 1, 0, 4, 1, 1, 64, 0, None, None, scale, PTR, 0, 64, 64, None, None, 0, None)

    assert call(2.3e38) == OK and call(2.4e38) == INVALID and "scale" in message()      # (times log2(e): 3.32e38 and 3.46e38, of 3.40e38)


def test_sizes_whose_product_passes_64_bits():
    n = C.c_size_t()
    for B in (1 << 50, 1 << 60, (1 << 63) - 1):
        assert lib.antdt_cache_attention_bytes(B, 1 << 14, 1, 64, 1, C.byref(n)) == UNSUPPORTED
        assert lib.antdt_cross_attention_bytes(B, 1, 1, 1 << 14, 1, 64, 1, C.byref(n)) == INVALID


def test_tokens_of_no_sequence_have_their_operands_checked():
    """Offsets of no sequences: every token is in none, and its query's place is written all the same."""
    def call(q, qo):
        return lib.antdt_cache_append(q, 32, 8, qo, 32, 8, PTR, 16, 8, PTR, 16, 8, 3, 4, 2, 8, 0, None, 3 * PTR, 4 * PTR, 256, 16, 8, 5, 16, None, 7, 0, 7, None,
                                      PTR, None)

    assert call(None, 2 * PTR) == INVALID and call(PTR, None) == INVALID and "q_out" in message()


def test_heads_without_columns():
    """Refused by the call, not by the default scale."""
    for name in ("antdt_cache_attention_bytes", "antdt_cross_attention_bytes"):
        assert getattr(lib, name)(1, *((1, 1) if "cross" in name else ()), 1, 1, 0, 0, C.byref(C.c_size_t())) == UNSUPPORTED
    assert T._scale(None, 0) == 1.0 and T._scale(None, 64) == 0.125 and T._scale(0.5, 64) == 0.5


def test_caches_of_too_much_room():
    """Few large pages or many: one limit."""
    for page, cols in ((1 << 30, 2), (16, 1 << 27)):
        rc = lib.antdt_cache_attention(PTR, 512, 64, PTR, PTR, page * 512, 512, 64, 5, page, PTR, cols, 8, cols, PTR, 8, 8, 64, 1, 0.125, 2 * PTR, 512, 64, PTR, 1 << 30,
                                       None)
        assert rc == UNSUPPORTED and "2^31" in message()


def test_the_most_blocks():
    """2^24 blocks of rows of one kind are refused, one fewer are not."""
    n = C.c_size_t()
    for f in (lib.antdt_cross_attention_bytes, lib.antdt_cross_attention_backward_bytes):
        for S, T_ in ((1, 1), (1, 128), (128, 1)):
            assert f((1 << 24) - 1, S, T_, 1, 1, 8, 1, C.byref(n)) == OK and f(1 << 24, S, T_, 1, 1, 8, 1, C.byref(n)) == UNSUPPORTED
            assert "2^24" in message()
        assert f(1 << 23, 1, 129, 1, 1, 8, 1, C.byref(n)) == UNSUPPORTED and f((1 << 23) - 1, 129, 1, 1, 1, 8, 1, C.byref(n)) == OK


def test_blocks_in_two_rounds():
    """fp32 heads above 32 columns, a block of which fills a compute unit: more of them than compute units take twice as long, and equal shares of the keys
    less (they need a workspace); many rows of few keys stay with the blocks."""
    def shares(heads, S, keys, D, dtype=0):
        n = C.c_size_t()
        assert lib.antdt_cross_attention_bytes(1, S, keys, heads, heads, D, dtype, C.byref(n)) == OK
        return n.value > 0

    assert shares(260, 2, 300, 64) and shares(400, 9, 300, 128) and shares(16, 1024, 1000, 128)
    assert not shares(250, 2, 300, 64) and not shares(260, 2, 300, 32) and not shares(16, 1024, 100, 128) and not shares(260, 2, 300, 64, 1)
