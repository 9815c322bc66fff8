"""The entry points of the RMS norm, of 8-bit tensors and of the log probabilities of tokens refuse invalid
arguments before any HIP call, the binding refuses wrong tensors, and the plain reference forms agree with
their definitions."""
import ctypes

import numpy as np
import pytest

import lm_reference as ref

OK, E_NULL, E_NC, E_SHAPE, E_DTYPE, E_ALIAS, E_ARG = 0, -1, -2, -3, -4, -5, -7
F16, F32, F64, F16S, BF16 = 0, 1, 2, 3, 4
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def L():
    import paper_2207_08867_amd as m

    return m.lib()


def pointers(n):
    return [P(i << 28) for i in range(1, n + 1)]


def test_norm(L):
    h, x, w, ho, y, c, s = pointers(7)

    def both(status, dtype=F32, nc=1, rows=4, n=40, h=h, x=x, w=w, eps=1e-5, ho=ho, y=y, c=c, s=s):
        assert L.mc_rmsnorm_fwd(dtype, nc, rows, n, h, x, w, eps, ho, y, None) == status
        assert L.mc_rmsnorm_int8(dtype, nc, rows, n, h, x, w, eps, ho, c, s, None) == status

    for f in (F64, F16S, 5, -1):
        both(E_DTYPE, dtype=f)
    both(E_NC, nc=0)
    both(E_NC, nc=5)
    for rows, n in ((-1, 40), (4, -1), (4, 0), (4, (1 << 30) + 1), (1 << 41, 1), (1 << 40, 1 << 12)):
        both(E_SHAPE, rows=rows, n=n)
    for eps in (-1e-6, float("nan"), float("inf")):
        both(E_ARG, eps=eps)
    both(OK, rows=0, h=None, x=None, w=None, ho=None, y=None, c=None, s=None)
    both(E_NULL, h=None)
    both(E_NULL, ho=None)
    both(E_NULL, y=None, c=None)
    both(E_ARG, x=None)
    both(E_ALIAS, ho=x)
    both(E_ALIAS, ho=w)
    both(E_ALIAS, ho=P(h.value + 16))
    both(E_ALIAS, y=h, c=h)
    both(E_ALIAS, y=h, c=h, ho=h)
    both(E_ALIAS, y=ho, c=ho)
    both(E_ALIAS, nc=2, ho=P(h.value + 4 * 160))
    assert L.mc_rmsnorm_int8(F32, 1, 4, 40, h, x, w, 1e-5, ho, P(c.value + 8), s, None) == E_ARG
    assert L.mc_rmsnorm_int8(F32, 1, 4, 40, h, x, w, 1e-5, ho, c, P(s.value + 2), None) == E_ARG
    assert L.mc_rmsnorm_int8(F32, 1, 4, 40, h, x, w, 1e-5, ho, c, P(c.value + 4 * 127), None) == E_ALIAS


def test_norm_bwd(L):
    h, w, dy, g, dh, dw, ws = pointers(7)
    f, need = L.mc_rmsnorm_bwd, L.mc_rmsnorm_bwd_workspace(F32, 4, 40)
    assert need > 0
    assert f(F64, 1, 4, 40, h, w, dy, g, 1e-5, dh, dw, ws, need, None) == E_DTYPE
    assert f(F32, 5, 4, 40, h, w, dy, g, 1e-5, dh, dw, ws, need, None) == E_NC
    assert f(F32, 1, 4, 0, h, w, dy, g, 1e-5, dh, dw, ws, need, None) == E_SHAPE
    assert f(F32, 1, 4, 40, h, w, dy, g, -1.0, dh, dw, ws, need, None) == E_ARG
    assert f(F32, 1, 4, 40, h, w, dy, g, 1e-5, None, None, None, 0, None) == OK
    assert f(F32, 1, 0, 40, None, None, None, None, 1e-5, dh, None, None, 0, None) == OK
    assert f(F32, 1, 4, 40, None, w, dy, g, 1e-5, dh, dw, ws, need, None) == E_NULL
    assert f(F32, 1, 4, 40, h, w, None, g, 1e-5, dh, dw, ws, need, None) == E_NULL
    assert f(F32, 1, 4, 40, h, w, dy, g, 1e-5, dh, dw, None, 0, None) == E_NULL
    assert f(F32, 1, 4, 40, h, w, dy, g, 1e-5, dh, dw, ws, need - 1, None) == E_ARG
    assert f(F32, 1, 4, 40, h, w, dy, g, 1e-5, dh, dw, P(ws.value + 4), need, None) == E_ARG
    for a, b in ((h, dw), (dy, dw), (g, dw), (dh, w), (dh, dh), (ws, dw), (dh, ws)):
        assert f(F32, 1, 4, 40, h, w, dy, g, 1e-5, a, b, ws, need, None) == E_ALIAS
    assert L.mc_rmsnorm_bwd_workspace(F32, -1, 40) == E_SHAPE
    assert L.mc_rmsnorm_bwd_workspace(F64, 4, 40) == E_DTYPE
    for rows in (0, 1, 1000, 1 << 20):
        for n in (1, 512, 16384, 16385, 1 << 20):
            assert L.mc_rmsnorm_bwd_workspace(BF16, rows, n) >= 0


def test_int8(L):
    x, c, s, o = pointers(4)
    q, d = L.mc_int8_quantize, L.mc_int8_dequantize
    for f in (F64, F16S, 5, -1):
        assert q(f, 1, 4, 40, x, c, s, None) == E_DTYPE and d(f, 4, 40, c, s, o, None) == E_DTYPE
    assert q(F16, 0, 4, 40, x, c, s, None) == E_NC and q(F16, 5, 4, 40, x, c, s, None) == E_NC
    for rows, n in ((-1, 4), (4, -1), (1, (1 << 30) + 1), (1 << 41, 1), (1 << 40, 1 << 11)):
        assert q(F16, 1, rows, n, x, c, s, None) == E_SHAPE and d(F16, rows, n, c, s, o, None) == E_SHAPE
    assert q(F16, 1, 0, 40, None, None, None, None) == OK and d(F16, 0, 40, None, None, None, None) == OK
    assert d(F16, 4, 0, None, None, None, None) == OK
    assert q(F16, 1, 4, 0, None, None, None, None) == E_NULL  # the scales are written
    for a in ((None, c, s), (x, None, s), (x, c, None)):
        assert q(F16, 1, 4, 40, *a, None) == E_NULL
    assert d(F16, 4, 40, None, s, o, None) == E_NULL and d(F16, 4, 40, c, s, None, None) == E_NULL
    assert q(F16, 1, 4, 40, x, P(c.value + 8), s, None) == E_ARG and q(F16, 1, 4, 40, x, c, P(s.value + 1), None) == E_ARG
    assert q(F16, 1, 4, 40, x, x, s, None) == E_ALIAS and q(F16, 1, 4, 40, x, c, P(c.value + 508), None) == E_ALIAS
    assert d(F16, 4, 40, c, s, P(c.value + 500), None) == E_ALIAS


def test_products(L):
    a, sa, b, sb, bias, w, y = pointers(7)
    f, lin = L.mc_int8_matmul, L.mc_int8_linear_fwd

    def both(status, dtype=F16, M=40, N=50, K=300, a=a, sa=sa, b=b, sb=sb, bias=bias, w=w, size=1 << 24, y=y):
        assert f(dtype, M, N, K, a, sa, b, sb, bias, w, size, y, None) == status
        assert lin(dtype, M, K, N, a, b, sb, bias, w, size, y, None) == status

    both(E_DTYPE, dtype=F64)
    for M, N, K in ((-1, 4, 4), (4, -1, 4), (4, 4, -1), ((1 << 20) + 1, 4, 4), (4, (1 << 24) + 1, 4), (4, 4, 131073)):
        both(E_SHAPE, M=M, N=N, K=K)
        assert L.mc_int8_matmul_workspace(F16, M, N, K) == E_SHAPE
        assert L.mc_int8_linear_fwd_workspace(F16, M, K, N) == E_SHAPE
    both(OK, M=0, a=None, sa=None, b=None, sb=None, y=None, w=None, size=0)
    both(OK, N=0, a=None, sa=None, b=None, sb=None, y=None, w=None, size=0)
    both(E_NULL, a=None)
    both(E_NULL, b=None)
    both(E_NULL, sb=None)
    both(E_NULL, y=None)
    assert f(F16, 4, 4, 40, a, None, b, sb, None, w, 1 << 20, y, None) == E_NULL
    both(E_ARG, b=P(b.value + 8))
    both(E_ARG, sb=P(sb.value + 2))
    both(E_ALIAS, y=b)
    both(E_ALIAS, y=sb)
    both(E_ALIAS, y=bias)
    both(E_ALIAS, y=P(a.value + 64))
    need = L.mc_int8_linear_fwd_workspace(F16, 40, 300, 50)
    assert need > 0
    assert lin(F16, 40, 300, 50, a, b, sb, bias, w, need - 1, y, None) == E_ARG
    assert lin(F16, 40, 300, 50, a, b, sb, bias, None, 0, y, None) == E_NULL
    assert lin(F16, 40, 300, 50, a, b, sb, bias, b, need, y, None) == E_ALIAS
    big = L.mc_int8_matmul_workspace(F16, 200, 64, 8192)
    assert big > 0 and f(F16, 200, 64, 8192, a, sa, b, sb, None, None, 0, y, None) == E_NULL
    for M in (0, 1, 16, 17, 32, 33, 1000, 1 << 20):
        for N in (0, 1, 300, 1 << 24):
            for K in (0, 1, 1000, 131072):
                assert L.mc_int8_matmul_workspace(F32, M, N, K) >= 0
                assert L.mc_int8_linear_fwd_workspace(F32, M, K, N) >= 0


def test_logprobs(L):
    z, ids, w, logp, ent, ti, tl, st, g, gh, dz = pointers(11)
    fwd, bwd = L.mc_logprobs_fwd, L.mc_logprobs_bwd

    def both(status, dtype=F32, nc=1, rows=3, vocab=50, given=2, T=1.0):
        assert fwd(dtype, nc, rows, vocab, given, 5, z, ids, T, w, 1 << 20, logp, ent, ti, tl, st, None) == status
        assert bwd(dtype, nc, rows, vocab, given, z, ids, T, st, g, gh, dz, None) == status

    both(E_DTYPE, dtype=F64)
    both(E_NC, nc=0)
    both(E_NC, nc=5)
    for a in (dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(given=-1), dict(given=1025),
              dict(rows=(1 << 31) - 1, vocab=1 << 30)):
        both(E_SHAPE, **a)
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-60, 1e60):
        both(E_ARG, T=T)
    both(OK, rows=0)
    for top in (-1, 129):
        assert fwd(F32, 1, 3, 50, 2, top, z, ids, 1.0, w, 1 << 20, logp, ent, ti, tl, st, None) == E_SHAPE
        assert L.mc_logprobs_workspace(3, 50, top) == E_SHAPE
    for a in ((None, ids, logp, ti, tl), (z, None, logp, ti, tl), (z, ids, None, ti, tl), (z, ids, logp, None, tl),
              (z, ids, logp, ti, None)):
        assert fwd(F32, 1, 3, 50, 2, 5, a[0], a[1], 1.0, w, 1 << 20, a[2], ent, a[3], a[4], st, None) == E_NULL
    assert fwd(F32, 1, 3, 50, 2, 5, z, P(ids.value + 2), 1.0, w, 1 << 20, logp, ent, ti, tl, st, None) == E_ARG
    assert fwd(F32, 1, 3, 50, 2, 5, z, ids, 1.0, w, 1 << 20, logp, P(logp.value + 20), ti, tl, st, None) == E_ALIAS
    assert fwd(F32, 1, 3, 50, 2, 5, z, ids, 1.0, w, 1 << 20, z, ent, ti, tl, st, None) == E_ALIAS
    assert fwd(F32, 1, 3, 50, 2, 5, z, ids, 1.0, w, 1 << 20, logp, ent, ti, ti, st, None) == E_ALIAS
    assert bwd(F32, 1, 3, 50, 2, z, ids, 1.0, None, g, gh, dz, None) == E_NULL
    assert bwd(F32, 1, 3, 50, 2, z, ids, 1.0, st, g, gh, None, None) == E_NULL
    for o in (z, ids, st, g, gh):
        assert bwd(F32, 1, 3, 50, 2, z, ids, 1.0, st, g, gh, o, None) == E_ALIAS
    need = L.mc_logprobs_workspace(2, 100000, 5)
    assert need > 0
    assert fwd(F32, 1, 2, 100000, 2, 5, z, ids, 1.0, None, 0, logp, ent, ti, tl, st, None) == E_NULL
    assert fwd(F32, 1, 2, 100000, 2, 5, z, ids, 1.0, w, need - 1, logp, ent, ti, tl, st, None) == E_ARG
    assert fwd(F32, 1, 2, 100000, 2, 5, z, ids, 1.0, z, need, logp, ent, ti, tl, st, None) == E_ALIAS


def test_binding_refuses():
    """Wrong kinds of tensors: refused by the binding's own checks, on the CPU already."""
    import torch

    import paper_2207_08867_amd as m

    h, w = torch.zeros(3, 40), torch.zeros(40)
    with pytest.raises(TypeError):
        m.mc_rmsnorm_fwd(h.double(), None)
    with pytest.raises(ValueError):
        m.mc_rmsnorm_fwd(h, w[:39])
    with pytest.raises(ValueError):
        m.mc_rmsnorm_fwd(h, w.half())
    with pytest.raises(ValueError):
        m.mc_rmsnorm_fwd(h, w, x=h[:2])
    with pytest.raises(ValueError):
        m.mc_rmsnorm_int8(h, w, h_out=h)
    with pytest.raises(ValueError):
        m.mc_rmsnorm_int8(w, None, h_mc=True)
    with pytest.raises(ValueError):
        m.mc_rmsnorm_bwd(h, w, h.half())
    with pytest.raises(ValueError):
        m.mc_rmsnorm_fwd(h, w)  # not on a GPU
    c, s = torch.zeros(3, 128, dtype=torch.int8), torch.zeros(3)
    with pytest.raises(TypeError):
        m.mc_int8_dequantize(c.to(torch.uint8), s, 40, dtype=torch.float32)
    with pytest.raises(ValueError):
        m.mc_int8_dequantize(c, s, 129, dtype=torch.float32)
    with pytest.raises(ValueError):
        m.mc_int8_dequantize(c, s[:2], 40, dtype=torch.float32)
    with pytest.raises(ValueError):
        m.mc_int8_linear_fwd(h[0], (c, s))
    with pytest.raises(TypeError):
        m.mc_logprobs_fwd(h, torch.zeros(3, 1, dtype=torch.int64))
    with pytest.raises(ValueError):
        m.mc_logprobs_fwd(h, torch.zeros(2, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        m.mc_logprobs_bwd(h, torch.zeros(3, 1, dtype=torch.int32), torch.zeros(3, 2))
    with pytest.raises(ValueError):
        m.mc_logprobs_fwd(h, torch.zeros(3, 1, dtype=torch.int32), top=129)


def test_reference_codes():
    """The reference's integers against exact rational arithmetic."""
    from fractions import Fraction

    g = np.random.default_rng(0)
    p = np.concatenate([g.normal(size=(3, 60)), np.rint(g.normal(size=(4, 60)) * 8)], 0)
    p[4, 0] = 2 * np.abs(p[4]).max()  # many ties
    codes, scales = ref.quantize(p)
    for row, c, s in zip(p, codes, scales):
        m = Fraction(float(np.abs(row).max()))
        for v, k in zip(row, c):
            q = 127 * Fraction(float(v)) / m
            d = abs(q - int(k))
            assert d < Fraction(1, 2) or (d == Fraction(1, 2) and k % 2 == 0)
        assert abs(s - float(m) / 127) <= 2e-16 * s


def test_reference_gradients_by_differences():
    g = np.random.default_rng(1)
    h = 1e-6
    v, w, dy, later = g.normal(size=(3, 9)), g.normal(size=9), g.normal(size=(3, 9)), g.normal(size=(3, 9))
    dh, dw = ref.norm_bwd(v, w, dy, later, 1e-3)

    def loss(v, w):
        return (dy * v * w * ref.inverse_rms(v, 1e-3)).sum() + (later * v).sum()

    for i in np.ndindex(3, 9):
        e = np.zeros_like(v)
        e[i] = h
        assert abs((loss(v + e, w) - loss(v - e, w)) / (2 * h) - dh[i]) < 1e-7
    for i in range(9):
        e = np.zeros_like(w)
        e[i] = h
        assert abs((loss(v, w + e) - loss(v, w - e)) / (2 * h) - dw[i]) < 1e-7
    z, ids = 2 * g.normal(size=(4, 12)), np.array([[1, 1, 5], [-1, 12, 3], [0, -1, -1], [-1, -1, -1]])
    z[0, 7:] = -np.inf
    gi, gh = g.normal(size=(4, 3)), g.normal(size=4)
    for T in (0.7, 2.0):
        _, _, _, dz = ref.logprobs(z, ids, T, gi, gh)
        for r in range(4):
            for j in range(12):
                if not np.isfinite(z[r, j]):
                    continue
                e = np.zeros_like(z)
                e[r, j] = h

                def total(z):
                    logp, ent, _, _ = ref.logprobs(z, ids, T)
                    return (gi[r] * logp[r]).sum() + gh[r] * ent[r]

                assert abs((total(z + e) - total(z - e)) / (2 * h) - dz[r, j]) < 1e-7
