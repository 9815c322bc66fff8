"""Infinities and NaN in the MXFP4 calls: the same row has the same result whatever the number of
rows beside it and whichever kernel takes them."""
import numpy as np
import pytest

import mx4_reference as ref
from test_gpu_mx4 import DTYPES, dev, host, mcf, plain, random_mx4  # noqa: F401 (mcf: the fixture)

pytestmark = pytest.mark.gpu

ROWS = [1, 3, 10, 17, 40, 70, 300]


def no_zeros(codes, nc, rows, n):
    """The same tensor with the zeros of its first n columns replaced by 0.5 (-0.5)."""
    nib = np.stack((codes & 15, codes >> 4), -1).reshape(nc, rows, -1)
    part = nib[:, :, :n]
    part[(part & 7) == 0] |= 1
    return (nib[..., 0::2] + 16 * nib[..., 1::2]).astype(np.uint8)


def weight(g, O, I, wide):
    """One component with no zero elements; `wide`: blocks 60 binades apart in every row."""
    codes, scales = random_mx4(g, 1, O, I)
    if wide:
        scales[:, ::2] = np.where(scales[:, ::2] > 0, 67, 0)
        scales[:, 1::2] = np.where(scales[:, 1::2] > 0, 127, 0)
    codes = no_zeros(codes, 1, O, I)
    return codes, scales, ref.dequantize(codes, scales, I)[0]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", ROWS)
@pytest.mark.parametrize("wide", [False, True])
def test_infinite_input(mcf, dtype, T, wide):
    """y of a row with one infinity: the infinity times the weight's column, IEEE's result."""
    O, I = 70, 200
    g = np.random.default_rng(T)
    codes, scales, w = weight(g, O, I, wide)
    W = dev(codes), dev(scales)
    clean = plain(g, T, I, "float16")
    want = host(mcf.mc_mx4_linear_fwd(dev(clean, dtype), W))
    for value, column in ((np.inf, 7), (-np.inf, I - 1)):
        x = clean.copy()
        x[T // 2, column] = value
        y = host(mcf.mc_mx4_linear_fwd(dev(x, dtype), W))
        assert np.array_equal(y[T // 2], np.sign(w[:, column]) * value)
        keep = np.arange(T) != T // 2
        assert np.array_equal(y[keep], want[keep])
    x = clean.copy()
    x[T // 2, 5] = np.nan
    y = host(mcf.mc_mx4_linear_fwd(dev(x, dtype), W))
    assert np.isnan(y[T // 2]).all() and np.isfinite(np.delete(y, T // 2, 0)).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1, 9, 70, 300])
def test_infinite_gradient(mcf, dtype, T):
    """An infinity in dY: dX and db are IEEE's, dW too in the 16-bit formats; in binary32 its row of dW
    is not finite (NaN where the product of the whole numbers is an infinity).  Nothing else changes."""
    O, I = 70, 200
    g = np.random.default_rng(T)
    codes, scales, w = weight(g, O, I, False)
    W = dev(codes), dev(scales)
    x, clean = plain(g, T, I, "float16"), plain(g, T, O, "float16")
    x[np.abs(x) < 2.0 ** -10] = 1.0
    want = [host(v) for v in mcf.mc_mx4_linear_bwd(dev(x, dtype), W, dev(clean, dtype))]
    t, o = T // 2, 33
    clean[t, o] = np.inf
    dX, dW, db = (host(v) for v in mcf.mc_mx4_linear_bwd(dev(x, dtype), W, dev(clean, dtype)))
    assert np.array_equal(dX[t], np.sign(w[o]) * np.inf)
    assert np.array_equal(np.delete(dX, t, 0), np.delete(want[0], t, 0))
    if dtype == "float32":
        assert not np.isfinite(dW[o]).any()
    else:
        assert np.array_equal(dW[o], np.sign(x[t]) * np.inf)
    assert np.array_equal(np.delete(dW, o, 0), np.delete(want[1], o, 0))
    assert db[o] == np.inf and np.array_equal(np.delete(db, o), np.delete(want[2], o))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", ROWS)
def test_nan_blocks(mcf, dtype, T):
    """A block that stands for NaN: its column of the product, its rows of a left operand, and the
    block's columns of dX, and no others."""
    import torch

    O, I, bad, at = 70, 300, 11, 160
    g = np.random.default_rng(T)
    w = g.normal(size=(O, I)).astype(np.float32)
    w[bad, at + 3] = np.nan
    W = mcf.mc_mx4_quantize(dev(w))
    x = plain(g, T, I, dtype)
    cols = np.arange(O) != bad
    y = host(mcf.mc_mx4_linear_fwd(dev(x, dtype), W))
    assert np.isnan(y[:, bad]).all() and np.isfinite(y[:, cols]).all()
    a = x.astype(np.float32)
    A = mcf.mc_mx4_quantize(dev(a))
    y = host(mcf.mc_mx4_matmul(A, W, I, dtype=getattr(torch, dtype)))
    assert np.isnan(y[:, bad]).all() and np.isfinite(y[:, cols]).all()
    a[T // 2, at] = np.inf
    clean = mcf.mc_mx4_quantize(dev(g.normal(size=(O, I)).astype(np.float32)))
    y = host(mcf.mc_mx4_matmul(mcf.mc_mx4_quantize(dev(a)), clean, I, dtype=getattr(torch, dtype)))
    assert np.isnan(y[T // 2]).all() and np.isfinite(np.delete(y, T // 2, 0)).all()
    dX, _, _ = mcf.mc_mx4_linear_bwd(dev(x, dtype), W, dev(plain(g, T, O, dtype), dtype), dw=False, db=False)
    inside = (np.arange(I) >= at) & (np.arange(I) < at + 32)
    assert np.isnan(host(dX)[:, inside]).all() and np.isfinite(host(dX)[:, ~inside]).all()


@pytest.mark.parametrize("T", ROWS)
@pytest.mark.parametrize("bits", [0x7F800001, 0x7FC00000, 0xFF80FFFF])
def test_every_nan_is_one(mcf, T, bits):
    """binary32 NaN whose upper 16 bits are those of an infinity."""
    O, I = 70, 200
    g = np.random.default_rng(T)
    codes, scales, _ = weight(g, O, I, False)
    x, dY = plain(g, T, I, "float32").astype(np.float32), plain(g, T, O, "float32").astype(np.float32)
    x.view(np.uint32)[T // 2, 9] = bits
    dY.view(np.uint32)[T // 2, 9] = bits
    W = dev(codes), dev(scales)
    y = host(mcf.mc_mx4_linear_fwd(dev(x), W))
    dX, dW, db = (host(v) for v in mcf.mc_mx4_linear_bwd(dev(x), W, dev(dY)))
    for got in (y, dX):
        assert np.isnan(got[T // 2]).all() and np.isfinite(np.delete(got, T // 2, 0)).all()
    assert np.isnan(dW[9]).all() and np.isnan(dW[:, 9]).all() and np.isnan(db[9])
    assert np.isfinite(np.delete(np.delete(dW, 9, 0), 9, 1)).all() and np.isfinite(np.delete(db, 9)).all()
