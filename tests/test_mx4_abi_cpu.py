"""The entry points on MXFP4 tensors and of the distillation loss refuse invalid arguments before
any HIP call, and their plain reference forms agree with their definitions."""
import ctypes

import numpy as np
import pytest

import mx4_reference as ref

OK, E_NULL, E_NC, E_SHAPE, E_DTYPE, E_ALIAS, E_ARG = 0, -1, -2, -3, -4, -5, -7
F16, F32, F64, F16S, BF16 = 0, 1, 2, 3, 4
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def L():
    import paper_2207_08867_amd as m

    return m.lib()


def test_quantize(L):
    x, c, s = P(0x100000), P(0x200000), P(0x300000)
    for f in (F64, F16S, 5, -1):
        assert L.mc_mx4_quantize(f, 1, 1, 4, 40, x, c, s, None) == E_DTYPE
    for nc_in, nc in ((0, 1), (5, 1), (1, 0), (1, 5)):
        assert L.mc_mx4_quantize(BF16, nc_in, nc, 4, 40, x, c, s, None) == E_NC
    for rows, n in ((-1, 40), (4, -1), (1 << 41, 1), (1 << 34, 300), (1, 1 << 39), (1 << 36, 1)):
        assert L.mc_mx4_quantize(F16, 1, 1, rows, n, x, c, s, None) == E_SHAPE
    assert L.mc_mx4_quantize(F16, 1, 1, 0, 40, None, None, None, None) == OK
    assert L.mc_mx4_quantize(F16, 1, 1, 4, 0, None, None, None, None) == OK
    for args in ((None, c, s), (x, None, s), (x, c, None)):
        assert L.mc_mx4_quantize(F16, 1, 1, 4, 40, *args, None) == E_NULL
    assert L.mc_mx4_quantize(F16, 1, 1, 4, 40, x, P(0x200008), s, None) == E_ARG
    assert L.mc_mx4_quantize(F16, 1, 1, 4, 40, x, c, P(0x300002), None) == E_ARG
    assert L.mc_mx4_quantize(F16, 1, 1, 4, 40, x, P(0x100000), s, None) == E_ALIAS
    assert L.mc_mx4_quantize(F16, 1, 1, 4, 40, x, c, P(0x200000 + 192), None) == E_ALIAS
    assert L.mc_mx4_dequantize(F64, 1, 4, 40, c, s, x, None) == E_DTYPE
    assert L.mc_mx4_dequantize(F16, 0, 4, 40, c, s, x, None) == E_NC
    assert L.mc_mx4_dequantize(F16, 1, 4, 40, c, s, None, None) == E_NULL
    assert L.mc_mx4_dequantize(F16, 1, 4, 40, c, s, P(0x200000 + 64), None) == E_ALIAS
    assert L.mc_mx4_dequantize(F16, 1, 0, 40, None, None, None, None) == OK


def test_matmul(L):
    a, sa, b, sb, c, w = (P(i << 24) for i in range(1, 7))
    f = L.mc_mx4_matmul
    assert f(F64, 4, 4, 40, a, sa, 1, b, sb, 1, w, 1 << 20, c, None) == E_DTYPE
    assert f(F16, 4, 4, 40, a, sa, 0, b, sb, 1, w, 1 << 20, c, None) == E_NC
    assert f(F16, 4, 4, 40, a, sa, 1, b, sb, 5, w, 1 << 20, c, None) == E_NC
    for M, N, K in ((-1, 4, 4), (4, -1, 4), (4, 4, -1), ((1 << 20) + 1, 4, 4), (4, (1 << 24) + 1, 4), (4, 4, (1 << 22) + 1)):
        assert f(F16, M, N, K, a, sa, 1, b, sb, 1, w, 1 << 20, c, None) == E_SHAPE
        assert L.mc_mx4_matmul_workspace(F16, M, N, K, 1, 1) == E_SHAPE
    assert f(F16, 0, 4, 40, None, None, 1, None, None, 1, None, 0, None, None) == OK
    assert f(F16, 4, 4, 40, a, None, 1, b, sb, 1, w, 1 << 20, c, None) == E_NULL
    assert f(F16, 4, 4, 40, a, sa, 1, b, sb, 1, w, 1 << 20, None, None) == E_NULL
    assert f(F16, 4, 4, 40, P(0x1000004), sa, 1, b, sb, 1, w, 1 << 20, c, None) == E_ARG
    assert f(F16, 4, 4, 40, a, sa, 1, b, sb, 1, w, 1 << 20, P(0x1000010), None) == E_ALIAS
    assert f(F16, 4, 4, 40, a, sa, 1, b, sb, 1, w, 1 << 20, sb, None) == E_ALIAS


def test_linear(L):
    x, c, s, b, y, w = (P(i << 24) for i in range(1, 7))
    f = L.mc_mx4_linear_fwd
    assert f(F16S, 1, 4, 40, 8, x, c, s, b, w, 1 << 20, y, None) == E_DTYPE
    assert f(F16, 5, 4, 40, 8, x, c, s, b, w, 1 << 20, y, None) == E_NC
    assert f(F16, 1, -4, 40, 8, x, c, s, b, w, 1 << 20, y, None) == E_SHAPE
    assert f(F16, 1, 0, 40, 8, None, None, None, None, None, 0, None, None) == OK
    assert f(F16, 1, 4, 40, 8, x, None, s, b, w, 1 << 20, y, None) == E_NULL
    assert f(F16, 1, 4, 40, 8, x, c, P(s.value + 1), b, w, 1 << 20, y, None) == E_ARG
    assert f(F16, 1, 4, 40, 8, x, c, s, b, w, 1 << 20, b, None) == E_ALIAS
    assert f(F16, 1, 4, 40, 8, x, c, s, b, w, 1 << 20, P(x.value + 16), None) == E_ALIAS


def test_linear_bwd(L):
    x, c, s, dy, dx, dw, db, w = (P(i << 26) for i in range(1, 9))
    f = L.mc_mx4_linear_bwd
    need = L.mc_mx4_linear_bwd_workspace(F32, 2, 100, 784, 99)
    assert need > 0
    assert f(F64, 1, 4, 40, 8, x, c, s, dy, dx, dw, db, w, 1 << 24, None) == E_DTYPE
    assert f(F32, 0, 4, 40, 8, x, c, s, dy, dx, dw, db, w, 1 << 24, None) == E_NC
    assert f(F32, 1, 4, 40, (1 << 20) + 1, x, c, s, dy, dx, dw, db, w, 1 << 24, None) == E_SHAPE
    assert f(F32, 1, 4, 40, 8, x, c, s, dy, None, None, None, None, 0, None) == OK
    assert f(F32, 1, 4, 40, 8, x, c, s, None, dx, None, None, w, 1 << 24, None) == E_NULL
    assert f(F32, 1, 4, 40, 8, None, None, None, dy, dx, None, None, w, 1 << 24, None) == E_NULL
    assert f(F32, 1, 4, 40, 8, None, None, None, dy, None, dw, None, w, 1 << 24, None) == E_NULL
    assert f(F32, 2, 100, 784, 99, x, c, s, dy, dx, dw, db, w, need - 1, None) == E_ARG
    assert f(F32, 2, 100, 784, 99, x, c, s, dy, dx, dw, db, None, 0, None) == E_NULL
    assert f(F32, 2, 100, 784, 99, x, c, s, dy, dx, dw, db, P(w.value + 4), need, None) == E_ARG
    assert f(F32, 2, 100, 784, 99, x, c, s, dy, dx, dx, db, w, need, None) == E_ALIAS
    assert f(F32, 2, 100, 784, 99, x, c, s, dy, x, dw, db, w, need, None) == E_ALIAS
    assert f(F32, 2, 100, 784, 99, x, c, s, dy, dx, dw, db, dy, need, None) == E_ALIAS


def test_workspace_sizes(L):
    """Every size gives a size, empty ones included; results of nothing need none."""
    for dtype in (F16, BF16, F32):
        for T in (0, 1, 17, 65, 1000, 1 << 20):
            for I in (0, 1, 128, 1000):
                for O in (0, 1, 300, 5000):
                    assert L.mc_mx4_matmul_workspace(dtype, T, O, I, 1, 2) >= 0
                    assert L.mc_mx4_linear_fwd_workspace(dtype, 3, T, I, O) >= 0
                    assert L.mc_mx4_linear_bwd_workspace(dtype, 4, T, I, O) >= 0
    assert L.mc_mx4_linear_bwd_workspace(F32, 1, 0, 0, 0) == 0
    assert L.mc_mx4_linear_fwd_workspace(F32, 5, 1, 1, 1) == E_NC
    assert L.mc_mx4_linear_bwd_workspace(F32, 1, 1, 1, (1 << 20) + 1) == E_SHAPE
    assert L.mc_distill_workspace(-1, 5) == E_SHAPE and L.mc_distill_workspace(0, 5) == 0


def test_distill(L):
    z, ids, t, g, w, loss, stats, dz = (P(i << 26) for i in range(1, 9))
    fwd, bwd, both = L.mc_distill_fwd, L.mc_distill_bwd, L.mc_distill_fwd_bwd

    def all_give(status, dtype=F32, nc=1, rows=3, vocab=50, k=2, T=1.0):
        a = (dtype, nc, rows, vocab, k, z, ids, t, T)
        assert fwd(*a, w, 1 << 20, loss, stats, None) == status
        assert bwd(*a, stats, g, dz, None) == status
        assert both(*a, g, w, 1 << 20, loss, dz, None) == status

    all_give(E_DTYPE, dtype=F64)
    all_give(E_NC, nc=5)
    all_give(E_SHAPE, rows=-1)
    all_give(E_SHAPE, vocab=0)
    all_give(E_SHAPE, vocab=(1 << 30) + 1)
    all_give(E_SHAPE, k=1025)
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-60, 1e60):
        all_give(E_ARG, T=T)
    all_give(OK, rows=0)
    a = (F32, 1, 3, 50, 2)
    assert fwd(*a, z, None, t, 1.0, w, 1 << 20, loss, stats, None) == E_NULL
    assert fwd(*a, z, ids, t, 1.0, w, 1 << 20, None, stats, None) == E_NULL
    assert both(*a, z, ids, t, 1.0, g, w, 1 << 20, loss, None, None) == E_NULL
    assert bwd(*a, z, ids, t, 1.0, None, g, dz, None) == E_NULL
    assert both(*a, z, ids, t, 1.0, g, w, 1 << 20, loss, z, None) == E_ALIAS
    assert bwd(*a, z, ids, t, 1.0, stats, g, P(stats.value + 8), None) == E_ALIAS
    assert fwd(*a, z, P(ids.value + 2), t, 1.0, w, 1 << 20, loss, stats, None) == E_ARG
    need = L.mc_distill_workspace(2, 100000)
    assert need > 0
    assert fwd(F32, 1, 2, 100000, 2, z, ids, t, 1.0, None, 0, loss, stats, None) == E_NULL
    assert fwd(F32, 1, 2, 100000, 2, z, ids, t, 1.0, w, need - 1, loss, stats, None) == E_ARG


def test_reference_rounding():
    """The reference's E2M1 rounding against a search over all magnitudes, ties to even."""
    y = np.concatenate([np.linspace(-9, 9, 7201), [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]])
    got = ref.round_e2m1(y)
    for v, i in zip(y, got):
        d = np.abs(min(abs(v), 6.0) - ref.MAGNITUDES)
        best = [j for j in range(8) if d[j] == d.min()]
        assert i == (best[0] if len(best) == 1 else next(j for j in best if j % 2 == 0))


def test_reference_gradient_by_differences():
    g = np.random.default_rng(0)
    z, ids, t, w = g.normal(size=(4, 30)), np.array([[1, 5, -1], [0, 0, 29], [-1, 40, -2], [3, 4, 5]]), g.normal(size=(4, 3)), g.uniform(size=4)
    loss, dz = ref.distill(z, ids, t, w, 2.0)
    assert loss[2] == 0 and not dz[2].any() and (loss >= -1e-15).all()
    h = 1e-5
    for r in range(4):
        for j in range(30):
            e = np.zeros_like(z)
            e[r, j] = h
            d = (ref.distill(z + e, ids, t, w, 2.0)[0][r] - ref.distill(z - e, ids, t, w, 2.0)[0][r]) / (2 * h)
            assert abs(w[r] * d - dz[r, j]) < 1e-8
