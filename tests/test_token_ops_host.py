"""The operators on sequences of tokens without a GPU: what they refuse, sizes they report, the generator's known
answers, and the formulas of the GPU tests against differences."""
import ctypes as C

import numpy as np
import pytest

import token_formulas as F

A = pytest.importorskip("paper_2404_09679_amd", reason="build the library first (python paper_2404_09679_amd/build.py)")
lib = A.lib
OK, INVALID, SMALL, UNSUPPORTED = 0, -1, -3, -5
PTR = 1 << 20            # an address that the checks accept and nothing reads


def spec(p=0.1, step=None):
    return C.byref(A.binding.DropoutSpec(p, 0, 1, step))


def message():
    return lib.antdt_last_error(None).decode()


def test_philox_known_answers():
    # the generator's published test vectors (Random123, philox4x32 with 10 rounds)
    assert F.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert F.philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    w = F.philox([2, 5, 0, 9], [0x11112222, 0x3333])
    assert F.lots(6, 24, 0x333311112222, 9)[5, 16:24].tolist() == [v for x in w for v in (x & 0xFFFF, x >> 16)]


def test_dropout_refusals():
    def call(x=PTR, ldx=16, r=None, ldr=0, rows=4, cols=16, dtype=0, drop=None, y=2 * PTR, ldy=16):
        return lib.antdt_dropout(x, ldx, r, ldr, rows, cols, dtype, spec() if drop is None else drop, y, ldy, None)

    assert call(dtype=2) == INVALID and call(dtype=-1) == INVALID
    assert call(x=None) == INVALID and "x is null" in message()
    assert call(y=None) == INVALID
    assert call(x=PTR + 2) == INVALID and "misaligned" in message()
    assert call(ldx=15) == INVALID and call(ldy=8) == INVALID and call(r=PTR, ldr=15) == INVALID
    assert call(rows=-1) == INVALID and call(cols=-1) == INVALID
    for p in (-0.1, 1.5, float("nan")):
        assert call(drop=spec(p)) == INVALID and "probability" in message()
    assert call(drop=spec(0.5, PTR + 4)) == INVALID
    assert lib.antdt_dropout(PTR, 16, None, 0, 4, 16, 0, None, PTR, 16, None) == INVALID
    assert call(x=None, y=None, rows=0) == OK and call(x=None, y=None, cols=0) == OK


def test_lookup_refusals():
    def call(table=PTR, ldt=16, V=10, D=16, dtype=0, tokens=PTR, N=3, drop=None, out=2 * PTR, ldo=16, out_dtype=0):
        return lib.antdt_token_lookup(table, ldt, V, D, dtype, tokens, N, 1.0, drop, out, ldo, out_dtype, None)

    assert call(dtype=7) == INVALID and call(out_dtype=7) == INVALID
    assert call(table=None) == INVALID and call(tokens=None) == INVALID and call(out=None) == INVALID
    assert call(tokens=PTR + 2) == INVALID
    assert call(V=2 ** 31) == INVALID and call(N=-1) == INVALID and call(D=1 << 24) == INVALID
    assert call(ldt=15) == INVALID and call(ldo=15) == INVALID
    assert call(drop=spec(2.0)) == INVALID
    assert call(N=0, tokens=None, out=None) == OK and call(D=0, table=None, out=None) == OK


def test_token_gradient_refusals():
    n = C.c_size_t()
    assert lib.antdt_token_gradient_bytes(1000, 50, 16, C.byref(n)) == OK and n.value > 16000
    assert lib.antdt_token_gradient_bytes(0, 50, 16, C.byref(n)) == OK and n.value == 0
    assert lib.antdt_token_gradient_bytes(-1, 50, 16, C.byref(n)) == INVALID
    assert lib.antdt_token_gradient_bytes(1, 50, 16, None) == INVALID

    def call(dy=PTR, lddy=16, dtype=0, tokens=PTR, N=3, drop=None, grad=2 * PTR, ldg=16, V=10, D=16, acc=0, ws=PTR, size=1 << 30):
        return lib.antdt_token_gradient(dy, lddy, dtype, tokens, N, 1.0, drop, grad, ldg, V, D, acc, ws, size, None)

    assert call(dtype=3) == INVALID and call(dy=None) == INVALID and call(tokens=None) == INVALID and call(grad=None) == INVALID
    assert call(ws=None) == INVALID and call(ws=PTR + 128) == INVALID
    assert call(size=16) == SMALL and "needed" in message()
    assert call(lddy=3) == INVALID and call(ldg=15) == INVALID and call(N=2 ** 31) == INVALID
    assert call(N=0, acc=1, ws=None, size=0) == OK and call(V=0, grad=None) == OK


@pytest.mark.parametrize("dtype", [0, 1])
def test_gated_refusals(dtype):
    n = C.c_size_t()
    assert lib.antdt_gated_saved_bytes(3, 16, dtype, C.byref(n)) == OK and n.value > 0
    assert lib.antdt_gated_backward_bytes(3, 8, 16, dtype, C.byref(n)) == OK and n.value >= 3 * 32 * (2 if dtype else 4)
    assert lib.antdt_gated_forward_bytes(3, 0, 16, dtype, C.byref(n)) == INVALID
    for call in (lib.antdt_gated_forward_bytes, lib.antdt_gated_backward_bytes):
        assert call(3, 8, 16, dtype, None) == INVALID and call(3, 1 << 20, 16, dtype, C.byref(n)) == INVALID
        assert call(1 << 30, 8, 1 << 10, dtype, C.byref(n)) == INVALID

    def fwd(x=PTR, ldx=8, wg=PTR, wu=PTR, ldw=16, N=3, K=8, H=16, dt=dtype, act=0, h=PTR, ldh=16, saved=None, ws=PTR, size=1 << 30):
        return lib.antdt_gated_forward(x, ldx, wg, wu, ldw, N, K, H, dt, act, h, ldh, saved, ws, size, None)

    assert fwd(dt=2) == INVALID and fwd(act=4) == INVALID and fwd(act=-1) == INVALID
    for name in ("x", "wg", "wu", "h"):
        assert fwd(**{name: None}) == INVALID, name
    assert fwd(ldx=7) == INVALID and fwd(ldw=8) == INVALID and fwd(ldh=15) == INVALID and fwd(saved=PTR + 16) == INVALID
    assert fwd(ldw=1 << 21) == UNSUPPORTED
    assert fwd(N=0, x=None, h=None) == OK
    if dtype:
        assert fwd(K=12, ldx=16) == UNSUPPORTED and fwd(H=12) == UNSUPPORTED and fwd(x=PTR + 8) == UNSUPPORTED
        assert fwd(ldx=12) == UNSUPPORTED and "x:" in message()

    def bwd(dh=PTR, lddh=16, x=PTR, ldx=8, wg=PTR, wu=PTR, ldw=16, N=3, K=8, H=16, dt=dtype, saved=PTR, dx=PTR, lddx=8, dwg=PTR,
            dwu=PTR, lddw=16, ws=PTR, size=1 << 30):
        return lib.antdt_gated_backward(dh, lddh, x, ldx, wg, wu, ldw, N, K, H, dt, saved, dx, lddx, dwg, dwu, lddw, ws, size, None)

    for name in ("dh", "x", "wg", "wu", "saved", "dwg", "dwu", "ws"):
        assert bwd(**{name: None}) == INVALID, name
    assert bwd(size=8) == SMALL and bwd(lddx=7) == INVALID and bwd(lddw=15) == INVALID and bwd(lddh=1) == INVALID
    assert bwd(dx=None, dwg=None, dwu=None) == OK


def test_logprobs_refusals():
    n = C.c_size_t()
    assert lib.antdt_token_logprobs_bytes(4096, 1000, 5, C.byref(n)) == OK and n.value == 0
    assert lib.antdt_token_logprobs_bytes(1, 1000000, 5, C.byref(n)) == OK and n.value > 0
    assert lib.antdt_token_logprobs_bytes(1, 0, 0, C.byref(n)) == INVALID
    assert lib.antdt_token_logprobs_bytes(1, 100, 65, C.byref(n)) == INVALID

    def call(x=PTR, ld=100, N=3, V=100, dtype=0, tokens=PTR, logp=PTR, entropy=PTR, stats=PTR, top=0, tl=PTR, ti=PTR, ws=PTR, size=1 << 30):
        return lib.antdt_token_logprobs(x, ld, N, V, dtype, tokens, logp, entropy, stats, top, tl, ti, ws, size, None)

    assert call(dtype=9) == INVALID and call(x=None) == INVALID and call(tokens=None) == INVALID
    assert call(ld=99) == INVALID and call(V=0) == INVALID and call(top=-1) == INVALID and call(top=65) == INVALID
    assert call(V=4, ld=4, top=5) == INVALID and call(top=3, tl=None) == INVALID and call(top=3, ti=None) == INVALID
    assert call(stats=PTR + 4) == INVALID and call(N=1, V=1000000, ld=1000000, size=4) == SMALL
    assert call(N=0, x=None) == OK

    def grad(x=PTR, ld=100, N=3, V=100, dtype=0, tokens=PTR, stats=PTR, a=PTR, b=PTR, d=PTR, ldd=100):
        return lib.antdt_token_logprobs_gradient(x, ld, N, V, dtype, tokens, stats, a, b, d, ldd, None)

    assert grad(stats=None) == INVALID and grad(tokens=None) == INVALID and grad(d=None) == INVALID and grad(ldd=5) == INVALID
    assert grad(dtype=2) == INVALID and grad(N=0, x=None, d=None, stats=None) == OK


def test_formulas_against_differences():
    rng = np.random.default_rng(3)
    x, wg, wu, dh = rng.normal(size=(4, 6)), rng.normal(size=(6, 5)), rng.normal(size=(6, 5)), rng.normal(size=(4, 5))
    for act in ("silu", "gelu", "relu", "sigmoid"):
        f = F.gated(x, wg, wu, act, 0)
        got = [v for v, _ in F.gated_gradients(x, wg, wu, dh, f, 0)]
        for k, g in enumerate(got):
            v, eps = rng.normal(size=g.shape), 1e-6
            args = [[x, wg, wu], [x, wg, wu]]
            args[0][k], args[1][k] = args[0][k] + eps * v, args[1][k] - eps * v
            up, down = ((F.gated(*a, act, 0)["h"] * dh).sum() for a in args)
            assert abs((up - down) / (2 * eps) - (g * v).sum()) < 1e-6 * (1 + np.abs(g * v).sum()), (act, k)
    x, t = rng.normal(size=(5, 9)) * 2, np.array([0, 8, -1, 3, 4])
    x[3, :4] = -np.inf
    a, b = rng.normal(size=5), rng.normal(size=5)
    a[3] = 0          # its token is not allowed: log 0
    d, _ = F.logprobs_gradient(F.logprobs(x, t, 0), t, a, b)

    def value(y):
        f = F.logprobs(y, t, 0)
        return (np.where(a != 0, a * np.where(f["there"], f["logp"], 0), 0) + b * f["entropy"]).sum()

    v, eps = rng.normal(size=x.shape), 1e-6
    assert abs((value(x + eps * v) - value(x - eps * v)) / (2 * eps) - (d * v).sum()) < 1e-6
