"""What the tests on small integers cannot see in the MXFP4 products: the low pieces of wide inputs,
the smallest numbers, operands at odd addresses, reductions of nothing over large results.

Every sum here is one that binary32 holds exactly in any order (integers, or multiples of one power of
two, below 2^24 of them in magnitude, few numbers in a row), so results equal the exact sum rounded
once to the format, and a piece that is lost or counted twice shows."""
import numpy as np
import pytest

import mx4_reference as ref
from test_gpu_mx4 import DTYPES, dev, host, mcf, plain, random_mx4, values64  # noqa: F401

pytestmark = pytest.mark.gpu


def sparse(g, rows, n, bits, count, columns=None):
    """Odd integers of `bits` bits of both signs, `count` of them in a row, at `columns` if given."""
    x = np.zeros((rows, n))
    where = np.arange(n) if columns is None else np.asarray(columns)
    pick = where[g.integers(0, len(where), (rows, count))]
    value = g.integers(2 ** (bits - 2), 2 ** (bits - 1), (rows, count)) * 2 + 1
    np.put_along_axis(x, pick, value * g.choice([-1.0, 1.0], (rows, count)), 1)
    return x


def small_weight(g, nc, rows, n):
    """Elements 0, 0.5, 1, 1.5, 2 with a scale of 1."""
    codes, scales = random_mx4(g, nc, rows, n, 127, 128)
    nib = np.stack((codes & 15, codes >> 4), -1).reshape(nc, rows, -1)
    nib = np.where((nib & 7) > 4, nib & 11, nib)
    return (nib[..., 0::2] + 16 * nib[..., 1::2]).astype(np.uint8), scales


BITS = {"float16": 11, "bfloat16": 8, "float32": 19}  # 19: three bfloat16 pieces


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nc", [1, 2])
@pytest.mark.parametrize("T, O, I", [(1, 33, 500), (4, 40, 2100), (9, 50, 300), (17, 130, 256), (65, 200, 640),
                                     (300, 520, 300), (1030, 520, 1024), (4096, 4096, 2048)])
def test_linear_low_pieces(mcf, dtype, nc, T, O, I):
    """3 numbers of 19 bits times at most 4: below 2^23 halves."""
    import torch

    g = np.random.default_rng(T + nc)
    x, W = sparse(g, T, I, BITS[dtype], 3), tuple(map(dev, small_weight(g, nc, O, I)))
    got = mcf.mc_mx4_linear_fwd(dev(x, dtype), W)
    want = dev(x) @ values64(W, I).t()
    assert torch.equal(got.double(), want.to(got.dtype).double())


@pytest.mark.parametrize("nc", [1, 2, 3])
@pytest.mark.parametrize("T, O, I", [(17, 70, 512), (70, 130, 512), (300, 520, 1280), (4096, 4096, 2048)])
def test_binary16_low_pieces_of_wide_rows(mcf, nc, T, O, I):
    """The tiles' two-piece form: numbers of 11 bits where the weight's are 60 binades below their row's
    largest scale, zeros where the large ones are.  With several components every one but the last has
    its small blocks empty, so that the last alone makes the result."""
    import torch

    g = np.random.default_rng(T + nc)
    codes, scales = small_weight(g, nc, O, I)
    big = np.arange(I // 128) % 2 == 0
    scales[:, big], scales[:, ~big] = 177, 117
    codes.reshape(nc, O, I // 128, 64)[:nc - 1, :, ~big] = 0
    columns = np.flatnonzero(np.repeat(~big, 128))
    x = sparse(g, T, I, 11, 3, columns)
    W = dev(codes), dev(scales)
    got = mcf.mc_mx4_linear_fwd(dev(x, "float16"), W)
    want = dev(x) @ values64(W, I).t()
    assert float(want.abs().max()) > 0
    assert torch.equal(got.double(), want.half().double())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, O, I", [(60, 50, 70), (200, 130, 300), (1030, 257, 129), (2048, 1024, 1024)])
def test_backward_low_pieces(mcf, dtype, T, O, I):
    """dX from wide dY, dW from wide dY and from wide x, all three numbers a row of the reduction."""
    import torch

    g = np.random.default_rng(T)
    W = tuple(map(dev, small_weight(g, 1, O, I)))
    ones = g.choice([-1.0, 1.0], (T, I))
    wide = sparse(g, T, O, BITS[dtype], 3)
    dX, _, _ = mcf.mc_mx4_linear_bwd(dev(ones, dtype), W, dev(wide, dtype), dw=False, db=False)
    assert torch.equal(dX.double(), (dev(wide) @ values64(W, I)).to(dX.dtype).double())
    for x, dY in ((ones, sparse(g, O, T, BITS[dtype], 3).T), (sparse(g, I, T, BITS[dtype], 3).T, g.choice([-1.0, 1.0], (T, O)))):
        _, dW, _ = mcf.mc_mx4_linear_bwd(dev(x, dtype), W, dev(dY, dtype), dx=False, db=False)
        assert torch.equal(dW.double(), (dev(dY).t() @ dev(x)).to(dW.dtype).double())
    # both of two pieces: 11 bits each, or 8
    x, dY = sparse(g, I, T, min(11, BITS[dtype]), 3).T, sparse(g, O, T, min(11, BITS[dtype]), 3).T
    if dtype != "float16":  # 2^22 is past binary16's range
        _, dW, _ = mcf.mc_mx4_linear_bwd(dev(x, dtype), W, dev(dY, dtype), dx=False, db=False)
        assert torch.equal(dW.double(), (dev(dY).t() @ dev(x)).to(dW.dtype).double())


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T", [1, 3, 10, 40, 70, 300])
def test_smallest_numbers(mcf, dtype, T):
    """A weight at the bottom of its range (2^-128 and up, subnormal bfloat16 numbers) against large
    inputs, and inputs at the bottom of bfloat16's range against a large weight."""
    import torch

    O, I = 70, 160
    g = np.random.default_rng(T)
    codes, scales = random_mx4(g, 1, O, I, 0, 1)  # all scales 2^-127
    W = dev(codes), dev(scales)
    x = g.integers(-8, 9, (T, I)) * 2.0 ** 100
    got = mcf.mc_mx4_linear_fwd(dev(x, dtype), W)
    assert torch.equal(got.double(), (dev(x) @ values64(W, I).t()).to(got.dtype).double())
    dY = g.integers(-8, 9, (T, O)) * 2.0 ** 100
    dX, _, _ = mcf.mc_mx4_linear_bwd(dev(x, dtype), W, dev(dY, dtype), dw=False, db=False)
    assert torch.equal(dX.double(), (dev(dY) @ values64(W, I)).to(dX.dtype).double())
    W = dev(codes), dev(np.where(np.arange(8).reshape(1, 2, 1, 4) < 5, 227, 0).astype(np.uint8) + 0 * scales)
    x = g.integers(-8, 9, (T, I)) * 2.0 ** -133
    got = mcf.mc_mx4_linear_fwd(torch.from_numpy(x).to(getattr(torch, dtype)).cuda(), W)
    assert torch.equal(got.double(), (dev(x) @ values64(W, I).t()).to(got.dtype).double())


@pytest.mark.parametrize("M", [1, 40, 70, 300])
def test_smallest_numbers_product(mcf, M):
    """Scales at both ends of the range in one product of two MXFP4 tensors."""
    import torch

    g = np.random.default_rng(M)
    A, B = random_mx4(g, 1, M, 160, 0, 1), random_mx4(g, 1, 50, 160, 227, 228)
    A, B = tuple(map(dev, A)), tuple(map(dev, B))
    got = mcf.mc_mx4_matmul(A, B, 160, dtype=torch.float32)
    assert torch.equal(got.double(), values64(A, 160) @ values64(B, 160).t())


def moved(t):
    """The same contents one element past an aligned address."""
    import torch

    room = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    out = room[1:].view(t.shape)
    out.copy_(t)
    assert out.data_ptr() % 16 != 0 and out.is_contiguous()
    return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, O, I", [(1, 40, 256), (4, 40, 256), (12, 40, 256), (40, 130, 256), (70, 130, 512), (300, 520, 384)])
def test_addresses(mcf, dtype, T, O, I):
    """Plain operands aligned to their element only give the bits of aligned ones."""
    import torch

    g = np.random.default_rng(T)
    w = torch.randn(O, I, device="cuda").to(getattr(torch, dtype))
    W = mcf.mc_mx4_quantize(w, nc=2)
    V = mcf.mc_mx4_quantize(moved(w), nc=2)
    assert torch.equal(W[0], V[0]) and torch.equal(W[1], V[1])
    out = moved(torch.zeros_like(w))
    mcf.mc_mx4_dequantize(*W, I, dtype=w.dtype, out=out)
    assert torch.equal(out, mcf.mc_mx4_dequantize(*W, I, dtype=w.dtype))
    x, b, dY = (dev(plain(g, *s, dtype), dtype) for s in ((T, I), (1, O), (T, O)))
    b = b[0].clone()
    want = mcf.mc_mx4_linear_fwd(x, W, b)
    assert torch.equal(mcf.mc_mx4_linear_fwd(moved(x), W, moved(b), out=moved(torch.zeros_like(want))), want)
    for got, ref_ in zip(mcf.mc_mx4_linear_bwd(moved(x), W, moved(dY)), mcf.mc_mx4_linear_bwd(x, W, dY)):
        assert torch.equal(got, ref_)
