"""Products of 8-bit tensors on the GPU.  The integers' sums are exact and the outputs three (with a bias
four) binary32 operations and a rounding in a stated order, so every result must come out exactly."""
import numpy as np
import pytest

from lm_reference import DTYPES, dev, host, rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mcf():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2207_08867_amd as m

    m.lib()
    return m


def pack(c, s):
    pitch = (c.shape[1] + 127) // 128 * 128
    full = np.zeros((c.shape[0], pitch), np.int8)
    full[:, :c.shape[1]] = c
    return dev(full), dev(s)


def operand(g, rows, K):
    c = g.integers(-127, 128, size=(rows, K)).astype(np.int8)
    return c, (0.01 * np.exp2(g.uniform(-3, 3, rows))).astype(np.float32)


def product(a, sa, b, sb, bias, dtype):
    """The stated binary32 operations on the exact sums (binary64 products of 8-bit integers are exact)."""
    s = (a.astype(np.float64) @ b.astype(np.float64).T).astype(np.float32)
    y = (s * sa[:, None]) * sb
    return rounded(y if bias is None else y + bias.astype(np.float32), dtype)


SIZES = [(1, 1, 1), (1, 4096, 4096), (2, 17, 100), (8, 1000, 1024), (16, 16, 64), (17, 33, 129), (32, 50, 500), (33, 1, 40),
         (33, 70, 127), (64, 64, 128), (65, 130, 31), (100, 99, 784), (128, 128, 4096), (129, 257, 513), (300, 8, 2050),
         (200, 64, 8192), (777, 1023, 1025), (1031, 1029, 260), (40, 20, 131072), (3, 20, 131072)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M, N, K", SIZES)
def test_matmul(mcf, dtype, M, N, K):
    import torch

    g = np.random.default_rng(M + N + K)
    (a, sa), (b, sb) = operand(g, M, K), operand(g, N, K)
    a[0], b[0] = 127, -127  # the largest sum
    bias = rounded(g.normal(size=N), dtype)
    ta, tb = pack(a, sa), pack(b, sb)
    for bi in (None, bias):
        got = mcf.mc_int8_matmul(ta, tb, K, None if bi is None else dev(bi, dtype), dtype=getattr(torch, dtype))
        want = product(a, sa, b, sb, bi, dtype)
        assert np.array_equal(host(got), want), np.argwhere(host(got) != want)[:4]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, I, O", [(1, 1, 1), (1, 4096, 4096), (1, 4100, 77), (2, 1000, 300), (4, 784, 99), (5, 100, 20),
                                     (16, 129, 50), (17, 300, 40), (40, 513, 65), (100, 784, 99), (300, 1024, 700)])
def test_linear(mcf, dtype, T, I, O):
    """The layer is the quantisation and the product, from the same rows whatever their number."""
    import torch

    g = np.random.default_rng(T + I + O)
    w, sw = operand(g, O, I)
    W = pack(w, sw)
    x = dev(rounded(g.normal(size=(T, I)), dtype), dtype)
    b = dev(rounded(g.normal(size=O), dtype), dtype)
    for bias in (None, b):
        y = mcf.mc_int8_linear_fwd(x, W, bias)
        assert torch.equal(y, mcf.mc_int8_matmul(mcf.mc_int8_quantize(x), W, I, bias, dtype=x.dtype))
        assert torch.equal(y[-1:], mcf.mc_int8_linear_fwd(x[-1:].contiguous(), W, bias))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1, 3, 40])
def test_special_rows(mcf, dtype, T):
    """Rows of zeros, with an infinity, with NaN; a weight row whose scale is NaN."""
    import torch

    g = np.random.default_rng(T)
    w, sw = operand(g, 50, 200)
    sw[7] = np.nan
    W = pack(w, sw)
    x = rounded(g.normal(size=(T, 200)), dtype)
    for kind in (0.0, np.inf, -np.inf, np.nan):
        x[0, 3:] = x[0, 3:] if kind else 0.0
        x[0, 0:3] = kind
        y = host(mcf.mc_int8_linear_fwd(dev(x, dtype), W))
        assert np.isnan(y[:, 7]).all()
        rest = np.delete(y, 7, 1)
        assert (not rest[0].any()) if kind == 0.0 else np.isnan(rest[0]).all()
        assert np.isfinite(rest[1:]).all()
        x[0] = rounded(g.normal(size=200), dtype)


def test_empty(mcf):
    import torch

    g = np.random.default_rng(0)
    for M, N, K in ((0, 5, 40), (5, 0, 40), (0, 0, 0)):
        y = mcf.mc_int8_matmul(pack(*operand(g, M, K)), pack(*operand(g, N, K)), K, dtype=torch.float32)
        assert y.shape == (M, N)
    for M in (1, 5, 70):
        bias = torch.arange(6.0, device="cuda")
        a, b = pack(*operand(g, M, 0)), pack(*operand(g, 6, 0))
        assert not mcf.mc_int8_matmul(a, b, 0, dtype=torch.float32).any()
        assert torch.equal(mcf.mc_int8_matmul(a, b, 0, bias, dtype=torch.float32), bias.expand(M, 6))
        assert torch.equal(mcf.mc_int8_linear_fwd(torch.empty(M, 0, device="cuda"), b, bias), bias.expand(M, 6))


@pytest.mark.parametrize("M, N, K", [(4096, 4096, 512), (2048, 8192, 1024)])
def test_large_tiles(mcf, M, N, K):
    """The largest tiles: sampled rows."""
    import torch

    g = np.random.default_rng(1)
    (a, sa), (b, sb) = operand(g, M, K), operand(g, N, K)
    got = mcf.mc_int8_matmul(pack(a, sa), pack(b, sb), K, dtype=torch.float32)
    rows = np.concatenate([np.arange(0, M, 97), [M - 1]])
    assert np.array_equal(host(got[torch.from_numpy(rows).cuda()]), product(a[rows], sa[rows], b, sb, None, "float32"))


def test_long_weight(mcf):
    """Offsets past 32 bits in the weight and in the result."""
    import torch

    N, K = 530000, 4100  # 2^31 bytes of codes and more
    codes = torch.zeros(N, 4224, dtype=torch.int8, device="cuda")
    scales = torch.ones(N, device="cuda")
    g = np.random.default_rng(2)
    b, sb = operand(g, 50, K)
    codes[-50:, :K] = dev(b)
    scales[-50:] = dev(sb)
    for M in (1, 40):
        a, sa = operand(g, M, K)
        y = mcf.mc_int8_matmul(pack(a, sa), (codes, scales), K, dtype=torch.float32)
        assert np.array_equal(host(y[:, -50:]), product(a, sa, b, sb, None, "float32")) and not bool(y[:, :-50].any())
    del y
    M, K = 4100, 100
    (a, sa), w = operand(g, M, K), codes[:, :128].contiguous()
    w[-50:, :K] = dev(b[:, :K])
    w[-50:, K:] = 0
    y = mcf.mc_int8_matmul(pack(a, sa), (w, scales), K, dtype=torch.bfloat16)
    assert np.array_equal(host(y[-30:, -50:]), product(a[-30:], sa[-30:], b[:, :K], sb, None, "bfloat16"))
