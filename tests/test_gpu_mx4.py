"""MXFP4 tensors on the GPU against plain binary64 forms: quantisation byte for byte, reading
back, products, the linear layer and its gradients.

Tolerances of the products: a sum of L exact products, taken in binary32 in any order, is
within L 2^-24 sum|a||b| of the sum (first order), and the result is rounded once to its
format.  Products whose every partial sum is a binary32 number must come out exactly, whatever
the order: those tests are for the indexing."""
import numpy as np
import pytest

import mx4_reference as ref

pytestmark = pytest.mark.gpu

U = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8, "float32": 2.0 ** -24}
DTYPES = ["float16", "bfloat16", "float32"]


@pytest.fixture(scope="module")
def mcf():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2207_08867_amd as m

    m.lib()
    return m


def dev(a, dtype=None):
    import torch

    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(getattr(torch, dtype))


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def rounded(a, dtype):
    """a rounded to dtype, as binary64."""
    import torch

    return torch.from_numpy(np.ascontiguousarray(a)).to(getattr(torch, dtype)).double().numpy()


def spread(g, rows, n, dtype):
    """Values over many binades, with ties, zeros of both signs, and blocks of one kind."""
    v = g.normal(size=(rows, n)) * np.exp2(g.integers(-12, 12, size=(rows, 1)))
    pick = g.integers(0, 8, size=(rows, n))
    v = np.where(pick == 0, np.exp2(g.integers(-14, 14, size=(rows, n))) * g.choice([-5.0, -2.5, 1.25, 1.75, 3.5, 7.0], size=(rows, n)), v)
    v = np.where(pick == 1, 0.0, v)
    v = np.where(pick == 2, -0.0, v)
    v = np.where(pick == 3, g.choice([-1, 1], size=(rows, n)) * np.exp2(-24.0), v)
    if rows > 2:
        v[1] = 0.0
    return rounded(v, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nc", [1, 2, 4])
@pytest.mark.parametrize("rows, n", [(1, 1), (3, 31), (2, 32), (5, 33), (1, 127), (7, 128), (3, 129), (2, 1000),
                                     (1, 4096), (130, 260)])
def test_quantize_bytes(mcf, dtype, nc, rows, n):
    x = spread(np.random.default_rng(rows * n + nc), rows, n, dtype)
    codes, scales = mcf.mc_mx4_quantize(dev(x, dtype), nc=nc)
    want = ref.quantize(x[None], nc)
    assert np.array_equal(host(scales), want[1])
    assert np.array_equal(host(codes), want[0])
    back = mcf.mc_mx4_dequantize(codes, scales, n, dtype=dev(x, dtype).dtype)
    parts = ref.dequantize(*want, n).astype(np.float32)
    total = parts[-1]
    for p in parts[-2::-1]:
        total = total + p
    assert np.array_equal(host(back), rounded(total, dtype))


def test_quantize_extremes(mcf):
    """binary32 values at both ends of the range, infinities and NaN."""
    g = np.random.default_rng(5)
    x = np.zeros((8, 96), np.float32)
    x[0] = np.ldexp(g.uniform(1, 2, 96), -149 + g.integers(0, 30, 96))  # subnormal numbers
    x[1] = g.choice([-1, 1], 96) * np.float32(3.4028235e38) * g.uniform(0.1, 1, 96).astype(np.float32)
    x[2] = np.ldexp(g.normal(size=96), -125)
    x[3, :32], x[3, 32:64], x[3, 64:] = 1.0, 2.0, 3.0
    x[3, 5], x[3, 40] = np.inf, np.nan
    x[4, 33] = -np.inf
    x[5, 7] = np.float32(np.finfo(np.float32).tiny)
    x[6, 50] = np.ldexp(1.0, -149)
    x[7] = 6.0
    for nc in (1, 3):
        codes, scales = mcf.mc_mx4_quantize(dev(x), nc=nc)
        want = ref.quantize(x[None], nc)
        assert np.array_equal(host(scales), want[1])
        assert np.array_equal(host(codes), want[0])
    back = host(mcf.mc_mx4_dequantize(codes, scales, 96, dtype=dev(x).dtype))
    assert np.isnan(back[3, :64]).all() and not np.isnan(back[3, 64:]).any()
    assert np.isnan(back[4, 32:64]).all() and not back[4, :32].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nc_in", [2, 3, 4])
def test_quantize_planes(mcf, dtype, nc_in):
    """MC inputs: the planes' sum decides, also where it is a tie but for the last plane."""
    g = np.random.default_rng(nc_in)
    v = g.normal(size=(9, 200))
    planes = []
    for _ in range(nc_in):
        planes.append(rounded(v, dtype))
        v = v - planes[-1]
    x = np.stack(planes)
    x[0, 4] = rounded(g.choice([1.25, 2.5, -3.5, 5.0, 6.0], 200), dtype)  # ties of a scale of 1
    x[0, 4, ::32] = 6.0
    x[1:, 4] = 0.0
    x[nc_in - 1, 4] = rounded(g.choice([-1, 0, 1], 200) * 2.0 ** -24, dtype)
    x[1, 5, 3] = np.inf
    x[0, 6] = rounded(np.full(200, 60000.0), dtype)  # equal planes: sums past binary16's range
    x[1:, 6] = x[0, 6]
    codes, scales = mcf.mc_mx4_quantize(dev(x, dtype), nc=3, x_mc=True)
    want = ref.quantize(x, 3)
    assert np.array_equal(host(scales), want[1])
    assert np.array_equal(host(codes), want[0])


def test_quantize_planes_past_binary32(mcf):
    """binary32 planes whose sum passes the largest binary32 number."""
    x = np.full((2, 1, 40), 3e38, np.float32)
    x[:, 0, 3] = -3.4e38
    codes, scales = mcf.mc_mx4_quantize(dev(x), nc=2, x_mc=True)
    want = ref.quantize(x, 2)
    assert np.array_equal(host(scales), want[1]) and np.array_equal(host(codes), want[0])


def test_leading_shapes_and_empty(mcf):
    import torch

    x = torch.randn(2, 3, 70, device="cuda")
    codes, scales = mcf.mc_mx4_quantize(x, nc=2)
    assert codes.shape == (2, 2, 3, 64) and scales.shape == (2, 1, 2, 3, 4)
    flat = mcf.mc_mx4_quantize(x.reshape(6, 70), nc=2)
    assert torch.equal(flat[0].reshape(codes.shape), codes) and torch.equal(flat[1].reshape(scales.shape), scales)
    assert mcf.mc_mx4_dequantize(codes, scales, 70, dtype=torch.float16).shape == (2, 3, 70)
    one = mcf.mc_mx4_quantize(x[0, 0].clone())
    assert one[0].shape == (1, 64) and mcf.mc_mx4_dequantize(*one, 70, dtype=torch.float32).shape == (70,)
    for shape in ((0, 70), (3, 0)):
        c, s = mcf.mc_mx4_quantize(torch.empty(shape, device="cuda"))
        assert mcf.mc_mx4_dequantize(c, s, shape[1], dtype=torch.float32).shape == shape


def random_mx4(g, nc, rows, n, lo=121, hi=130):
    """Random codes and scales, zeros past n."""
    G = ref.groups(n)
    code = g.integers(0, 16, (nc, rows, G * 128))
    code[:, :, n:] = 0
    codes = (code[..., 0::2] + 16 * code[..., 1::2]).astype(np.uint8)
    scales = g.integers(lo, hi, (nc, G, rows, 4)).astype(np.uint8)
    flat = scales.transpose(0, 2, 1, 3).reshape(nc, rows, G * 4).copy()
    flat[:, :, -(-n // 32):] = 0
    return codes, np.ascontiguousarray(flat.reshape(nc, rows, G, 4).transpose(0, 2, 1, 3))


def close(got, want, size, terms, dtype, what):
    bound = terms * 2.0 ** -24 * size + U[dtype] * np.abs(want) * 1.01 + 2.0 ** -24
    worst = np.max(np.abs(got - want) / bound) if got.size else 0.0
    assert worst <= 1.0, f"{what}: {worst} of the bound"


SIZES = [(1, 1, 1), (1, 16, 128), (1, 33, 1000), (3, 50, 70), (16, 17, 129), (17, 40, 300), (33, 100, 128), (64, 64, 256),
         (65, 130, 31), (100, 99, 784), (129, 257, 513), (260, 300, 640), (1, 5, 5000), (300, 8, 2050)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("a_nc, b_nc", [(1, 1), (1, 2), (3, 2)])
@pytest.mark.parametrize("M, N, K", SIZES)
def test_matmul(mcf, dtype, a_nc, b_nc, M, N, K):
    g = np.random.default_rng(M + N + K)
    A, B = random_mx4(g, a_nc, M, K), random_mx4(g, b_nc, N, K)
    got = host(mcf.mc_mx4_matmul(tuple(map(dev, A)), tuple(map(dev, B)), K, dtype=dev(np.zeros(1), dtype).dtype))
    a, b = ref.dequantize(*A, K), ref.dequantize(*B, K)
    size = np.abs(a).sum(0) @ np.abs(b).sum(0).T
    close(got, a.sum(0) @ b.sum(0).T, size, K * a_nc * b_nc, dtype, f"{M}x{N}x{K}")


@pytest.mark.parametrize("M, N, K", SIZES + [(512, 768, 1024), (2000, 1000, 130)])
def test_matmul_exact_sums(mcf, M, N, K):
    """Scales of 1: every partial sum is a multiple of 1/4 below 2^22, so binary32 holds it."""
    g = np.random.default_rng(M * N + K)
    A, B = random_mx4(g, 1, M, K, 127, 128), random_mx4(g, 2, N, K, 127, 128)
    got = host(mcf.mc_mx4_matmul(tuple(map(dev, A)), tuple(map(dev, B)), K, dtype=dev(np.zeros(1), "float32").dtype))
    assert np.array_equal(got, ref.dequantize(*A, K).sum(0) @ ref.dequantize(*B, K).sum(0).T)


def plain(g, rows, n, dtype):
    x = g.normal(size=(rows, n))
    x[g.random((rows, n)) < 0.02] *= 50.0
    return rounded(x, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nc", [1, 2, 4])
@pytest.mark.parametrize("T, O, I", SIZES)
def test_linear(mcf, dtype, nc, T, O, I):
    g = np.random.default_rng(T + O + I + nc)
    x, W, b = plain(g, T, I, dtype), random_mx4(g, nc, O, I), plain(g, 1, O, dtype)[0]
    w = ref.dequantize(*W, I)
    tx, tw, tb = dev(x, dtype), tuple(map(dev, W)), dev(b, dtype)
    size = np.abs(x) @ np.abs(w).sum(0).T
    want = x @ w.sum(0).T
    pieces = {"float16": 2, "bfloat16": 1, "float32": 3}[dtype]
    close(host(mcf.mc_mx4_linear_fwd(tx, tw)), want, size, I * nc * pieces, dtype, "y")
    close(host(mcf.mc_mx4_linear_fwd(tx, tw, tb)), want + b, size + np.abs(b), I * nc * pieces + 1, dtype, "y + b")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, O, I", SIZES + [(400, 520, 1024), (1100, 300, 260)])
def test_linear_exact_sums(mcf, dtype, T, O, I):
    g = np.random.default_rng(T * O + I)
    x, W = g.integers(-8, 9, (T, I)).astype(np.float64), random_mx4(g, 1, O, I, 127, 128)
    got = host(mcf.mc_mx4_linear_fwd(dev(x, dtype), tuple(map(dev, W))))
    assert np.array_equal(got, rounded(x @ ref.dequantize(*W, I).sum(0).T, dtype))


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_linear_wide_scales(mcf, dtype):
    """Scales over the format's range against inputs at the other end."""
    g = np.random.default_rng(3)
    O, I = 20, 256
    W = random_mx4(g, 1, O, I, 30, 31)
    W[1][:, :, 1::2] = 200
    W[1][:, :, 0::2] = 3
    w = ref.dequantize(*W, I).sum(0)
    for T in (2, 70):
        x = rounded(g.normal(size=(T, I)) * 2.0 ** -60, dtype)
        got = host(mcf.mc_mx4_linear_fwd(dev(x, dtype), tuple(map(dev, W))))
        want = x @ w.T
        assert np.all(np.abs(got - want) <= 3 * I * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T) + U[dtype] * np.abs(want) + 2.0 ** -126)


def test_linear_nonfinite_rows_stay_apart(mcf):
    """An infinity or NaN in one row of x leaves the other rows as they are."""
    import torch

    g = np.random.default_rng(8)
    for T in (3, 40, 300):
        x = plain(g, T, 200, "float32")
        W = tuple(map(dev, random_mx4(g, 1, 48, 200)))
        clean = mcf.mc_mx4_linear_fwd(dev(x, "float16"), W)
        x[T // 2, 7], x[T // 2, 199] = np.inf, np.nan
        dirty = mcf.mc_mx4_linear_fwd(dev(x, "float16"), W)
        keep = torch.arange(T, device="cuda") != T // 2
        assert torch.equal(clean[keep], dirty[keep]) and torch.isnan(dirty[T // 2]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nc", [1, 2, 3])
@pytest.mark.parametrize("T, O, I", [(1, 1, 1), (1, 64, 128), (7, 33, 70), (64, 50, 129), (100, 99, 784), (130, 260, 300),
                                     (513, 40, 31), (300, 300, 257)])
def test_backward(mcf, dtype, nc, T, O, I):
    g = np.random.default_rng(T + O + I)
    x, dY, W = plain(g, T, I, dtype), plain(g, T, O, dtype), random_mx4(g, nc, O, I)
    w = ref.dequantize(*W, I)
    tx, tw, ty = dev(x, dtype), tuple(map(dev, W)), dev(dY, dtype)
    dX, dW, db = mcf.mc_mx4_linear_bwd(tx, tw, ty)
    close(host(dX), dY @ w.sum(0), np.abs(dY) @ np.abs(w).sum(0), 3 * O * nc, dtype, "dX")
    # three pieces a side leave out products of 2^-26 |x||dY| each: one more unit of the sum's bound
    close(host(dW), dY.T @ x, np.abs(dY).T @ np.abs(x), 6 * T + 1, dtype, "dW")
    close(host(db), dY.sum(0), np.abs(dY).sum(0), T, dtype, "db")
    for k, flags in enumerate(((True, False, False), (False, True, False), (False, False, True))):
        part = mcf.mc_mx4_linear_bwd(tx, tw, ty, dx=flags[0], dw=flags[1], db=flags[2])
        assert all((p is None) == (not f) for p, f in zip(part, flags))
        assert np.array_equal(host(part[k]), host((dX, dW, db)[k]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, O, I", [(5, 40, 70), (200, 130, 300), (512, 384, 512), (1030, 257, 129)])
def test_backward_by_differences(mcf, dtype, T, O, I):
    """y is linear in x, so on integers (y(x + e) - y(x)) . dY is dX's directional product
    exactly; dW and db likewise by linearity in the weight, read through exact sums."""
    g = np.random.default_rng(T)
    x, dY = g.integers(-3, 4, (T, I)).astype(float), g.integers(-2, 3, (T, O)).astype(float)
    W = random_mx4(g, 1, O, I, 127, 128)
    tw = tuple(map(dev, W))
    dX, dW, db = (host(v) for v in mcf.mc_mx4_linear_bwd(dev(x, "float32"), tw, dev(dY, "float32")))
    e = g.integers(-2, 3, (T, I)).astype(float)
    lift = host(mcf.mc_mx4_linear_fwd(dev(x + e, "float32"), tw)) - host(mcf.mc_mx4_linear_fwd(dev(x, "float32"), tw))
    assert (lift * dY).sum() == (dX * e).sum()
    w2 = random_mx4(g, 1, O, I, 127, 128)
    step = ref.dequantize(*w2, I)[0] - ref.dequantize(*W, I)[0]
    b = g.integers(-3, 4, O).astype(float)
    lift = host(mcf.mc_mx4_linear_fwd(dev(x, "float32"), tuple(map(dev, w2)), dev(b, "float32"))) \
        - host(mcf.mc_mx4_linear_fwd(dev(x, "float32"), tw))
    assert (lift * dY).sum() == (dW * step).sum() + (db * b).sum()
    got = mcf.mc_mx4_linear_bwd(dev(x, dtype), tw, dev(dY, dtype))
    for a, b in zip(got, (dX, dW, db)):
        assert np.array_equal(host(a), rounded(b, dtype))


def test_empty_products(mcf):
    import torch

    W = mcf.mc_mx4_quantize(torch.randn(6, 40, device="cuda"))
    x = torch.randn(4, 40, device="cuda")
    assert mcf.mc_mx4_linear_fwd(x[:0], W).shape == (0, 6)
    none = mcf.mc_mx4_quantize(torch.empty(6, 0, device="cuda"))
    b = torch.randn(6, device="cuda")
    assert torch.equal(mcf.mc_mx4_linear_fwd(x[:, :0].contiguous(), none, b), b.expand(4, 6))
    assert not mcf.mc_mx4_matmul(mcf.mc_mx4_quantize(x[:, :0].contiguous()), none, 0, dtype=torch.float32).any()
    dX, dW, db = mcf.mc_mx4_linear_bwd(x[:0], W, torch.empty(0, 6, device="cuda"))
    assert dX.shape == (0, 40) and not dW.any() and not db.any()
    empty = mcf.mc_mx4_quantize(torch.empty(0, 40, device="cuda"))
    dX, dW, db = mcf.mc_mx4_linear_bwd(x, empty, torch.empty(4, 0, device="cuda"))
    assert not dX.any() and dW.shape == (0, 40) and db.shape == (0,)


def test_refusals(mcf):
    import torch

    x, W = torch.randn(4, 40, device="cuda"), mcf.mc_mx4_quantize(torch.randn(6, 40, device="cuda"))
    with pytest.raises(TypeError):
        mcf.mc_mx4_quantize(x.double())
    with pytest.raises(ValueError):
        mcf.mc_mx4_quantize(x.t())
    with pytest.raises(ValueError):
        mcf.mc_mx4_quantize(x, nc=5)
    with pytest.raises(ValueError):
        mcf.mc_mx4_quantize(x.cpu())
    with pytest.raises(ValueError):
        mcf.mc_mx4_dequantize(*W, 200, dtype=torch.float32)
    with pytest.raises(ValueError):
        mcf.mc_mx4_linear_fwd(torch.randn(4, 200, device="cuda"), W)
    with pytest.raises(ValueError):
        mcf.mc_mx4_linear_fwd(x, W, torch.randn(5, device="cuda"))
    with pytest.raises(ValueError):
        mcf.mc_mx4_linear_fwd(x, W, torch.randn(6, device="cuda").half())
    with pytest.raises(TypeError):
        mcf.mc_mx4_linear_fwd(x, (W[0].int(), W[1]))
    with pytest.raises(ValueError):
        mcf.mc_mx4_linear_fwd(x, (W[0][:, ::2], W[1]))
    with pytest.raises(ValueError):
        mcf.mc_mx4_linear_bwd(x, W, torch.randn(4, 7, device="cuda"))
    with pytest.raises(ValueError):
        mcf.mc_mx4_matmul(W, W, 300, dtype=torch.float32)
    if mcf.mc_mx4_linear_bwd_workspace(torch.float32, 1, 4, 40, 6):
        with pytest.raises(ValueError):
            mcf.mc_mx4_linear_bwd(x, W, torch.randn(4, 6, device="cuda"),
                                  workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_side_stream(mcf):
    """Calls run on the caller's current stream."""
    import torch

    x = torch.randn(64, 512, device="cuda").half()
    W = mcf.mc_mx4_quantize(torch.randn(96, 512, device="cuda").half())
    want = mcf.mc_mx4_linear_fwd(x, W)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = torch.zeros_like(x)
        for _ in range(20):
            y = y + x / 32
        y = y * 0 + x
        got = mcf.mc_mx4_linear_fwd(y, W)
    s.synchronize()
    assert torch.equal(got, want)


def test_many_elements(mcf):
    """More than 2^31 elements: offsets in 64 bits; sampled rows against the same rows alone."""
    import torch

    rows, n = 70001, 32768
    x = torch.randn(1, n, device="cuda").half().expand(rows, n).contiguous()
    pick = [0, 1, 35000, 65535, 65536, rows - 1]
    for i in pick:
        x[i] = torch.randn(n, device="cuda").half()
    codes, scales = mcf.mc_mx4_quantize(x)
    back = mcf.mc_mx4_dequantize(codes, scales, n, dtype=torch.float16)
    alone = mcf.mc_mx4_quantize(x[pick].contiguous())
    assert torch.equal(codes[:, pick], alone[0]) and torch.equal(scales[:, :, pick], alone[1])
    assert torch.equal(back[pick], mcf.mc_mx4_dequantize(*alone, n, dtype=torch.float16))


def values64(W, n):
    """The numbers of an MXFP4 tensor on the GPU, summed over its components, in binary64."""
    import torch

    codes, scales = W[0].long(), W[1].permute(0, 2, 1, 3).double()
    nib = torch.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], codes.shape[1], -1, 32)
    mag = torch.tensor(ref.MAGNITUDES, device="cuda")[nib & 7] * (1.0 - 2.0 * (nib >> 3))
    return (mag * torch.exp2(scales - 127.0).flatten(2).unsqueeze(-1)).flatten(2).sum(0)[:, :n]


@pytest.mark.parametrize("M, N, K", [(4099, 4100, 4224), (2100, 8200, 2049), (520, 5000, 8192), (8200, 70, 1000)])
def test_large_products_exact_sums(mcf, M, N, K):
    """The largest tiles, their ragged edges and the products in slices: integer operands whose every
    partial sum binary32 holds (36 K < 2^22 quarters), so all orders give the same."""
    import torch

    g = np.random.default_rng(M + K)
    A, B = (tuple(map(dev, random_mx4(g, 1, r, K, 127, 128))) for r in (M, N))
    a, b = values64(A, K), values64(B, K)
    assert torch.equal(mcf.mc_mx4_matmul(A, B, K, dtype=torch.float32).double(), a @ b.t())
    x = torch.from_numpy(g.integers(-4, 5, (M, K)).astype(np.float32)).cuda()
    want = x.double() @ b.t()
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        assert torch.equal(mcf.mc_mx4_linear_fwd(x.to(dtype), B).double(), want.to(dtype).double()), dtype
    dY = torch.from_numpy(g.integers(-2, 3, (M, N)).astype(np.float32)).cuda()
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        dX, dW, db = mcf.mc_mx4_linear_bwd(x.to(dtype), B, dY.to(dtype))
        assert torch.equal(dX.double(), (dY.double() @ b).to(dtype).double()), dtype
        assert torch.equal(dW.double(), (dY.double().t() @ x.double()).to(dtype).double()), dtype
        assert torch.equal(db.double(), dY.double().sum(0).to(dtype).double()), dtype


@pytest.mark.parametrize("dtype", DTYPES)
def test_results_repeat(mcf, dtype):
    """The same bits from one call to the next."""
    import torch

    W = mcf.mc_mx4_quantize(torch.randn(300, 1000, device="cuda"), nc=2)
    x = torch.randn(500, 1000, device="cuda").to(getattr(torch, dtype))
    first = mcf.mc_mx4_linear_fwd(x, W)
    for _ in range(3):
        assert torch.equal(mcf.mc_mx4_linear_fwd(x, W), first)


@pytest.mark.parametrize("below", [0, 35, 36, 37, 60, 120])
@pytest.mark.parametrize("T, O, I", [(70, 130, 256), (300, 520, 640)])
def test_binary16_layer_of_wide_rows(mcf, below, T, O, I):
    """Blocks far below the largest one of their weight row, where x is zero at the large ones: the
    small ones alone make the result, exactly, whatever lies between them."""
    import torch

    g = np.random.default_rng(below)
    codes, scales = random_mx4(g, 1, O, I, 117, 118)
    small = 117
    big = np.arange(0, I // 128) % 2 == 0  # every second group is large in all four blocks
    scales[:, big] = min(small + below, 254)
    scales[:, ~big, O // 2] = 0  # a row whose small blocks are the least there is, with no numbers in them
    codes.reshape(1, O, I // 128, 64)[:, O // 2, ~big] = 0
    x = g.integers(-4, 5, (T, I)).astype(np.float64)
    x.reshape(T, I // 128, 128)[:, big] = 0.0
    W = dev(codes), dev(scales)
    got = mcf.mc_mx4_linear_fwd(dev(x, "float16"), W)
    want = torch.from_numpy(x).cuda() @ values64(W, I).t()
    assert torch.equal(got.double(), want.half().double())
    b = torch.randn(O, device="cuda").half()
    got = mcf.mc_mx4_linear_fwd(dev(x, "float16"), W, b)
    assert (got.double() - (want + b.double())).abs().max() <= 2.0 ** -11 * (want.abs().max() + 8)


def test_binary16_layer_keeps_nan_blocks(mcf):
    """A weight block that stands for NaN makes its column NaN and no other."""
    import torch

    x = torch.randn(100, 300, device="cuda").half()
    w = torch.randn(90, 300, device="cuda")
    w[7, 40] = float("nan")
    y = mcf.mc_mx4_linear_fwd(x, mcf.mc_mx4_quantize(w))
    assert torch.isnan(y[:, 7]).all()
    keep = torch.arange(90, device="cuda") != 7
    assert torch.isfinite(y[:, keep]).all()


def test_more_rows_than_one_launch(mcf):
    """Past 2^21 workgroups they go out in several launches: the same rows over and over."""
    import torch

    part, times, n = 1100003, 31, 5
    x = torch.randn(part, n, device="cuda").bfloat16()
    codes, scales = mcf.mc_mx4_quantize(x)
    back = mcf.mc_mx4_dequantize(codes, scales, n, dtype=torch.bfloat16)
    many = x.repeat(times, 1)
    assert many.shape[0] > 2 ** 25
    got_codes, got_scales = mcf.mc_mx4_quantize(many)
    for i in range(times):
        rows = slice(i * part, (i + 1) * part)
        assert torch.equal(got_codes[:, rows], codes) and torch.equal(got_scales[:, :, rows], scales)
    got = mcf.mc_mx4_dequantize(got_codes, got_scales, n, dtype=torch.bfloat16)
    assert torch.equal(got.view(times, part, n), back.expand(times, part, n))


def test_linear_of_more_rows_than_one_staging_launch(mcf):
    """A binary16 x of more than 2^32 padded elements, with sums that binary16 holds exactly."""
    import torch

    T, n, out = 2 ** 20, 4100, 3
    some = torch.randint(-1, 2, (1024, n), device="cuda").half()
    x = some.repeat(T // 1024, 1)
    pick = [0, 1, 1016801, 1016802, T - 1]  # the second launch begins in row 2^32 / 4224
    for i in pick:
        x[i] = torch.randint(-1, 2, (n,), device="cuda").half()
    w = torch.randint(-1, 2, (out, n), device="cuda").half()
    y = mcf.mc_mx4_linear_fwd(x, mcf.mc_mx4_quantize(w))
    exact = some.double().cpu() @ w.double().cpu().T
    picked = x[pick].double().cpu() @ w.double().cpu().T
    assert float(max(exact.abs().max(), picked.abs().max())) <= 2048
    assert torch.equal(y[pick].cpu(), picked.half())
    same = y.view(T // 1024, 1024, out) == exact.half().cuda()
    same.view(T, out)[pick] = True
    assert bool(same.all())
