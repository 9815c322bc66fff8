"""The RMS norm of a residual stream, its 8-bit output and its gradients, and 8-bit quantisation, on the GPU
against plain binary64 forms.

The stream behind the addition and the codes are fixed functions of the input and must come out exactly.
Tolerances: everything else is binary64 until it is rounded to binary32 and from there to the format,
so a value is within |v| (2^-24 + U) of its own, and sums of n terms in binary64 add n 2^-53 of the
terms' magnitudes.  (y of a plain 16-bit row is a binary32 product with a rounded factor first: 2^-23, where a
hundredth of U is 2^-18 or more.)  dw's sums of a workgroup's rows are kept in binary32 each: 2^-24 of the magnitudes."""
import numpy as np
import pytest

import lm_reference as ref
from lm_reference import DTYPES, TINY, U, dev, host, rounded

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def mcf():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2207_08867_amd as m

    m.lib()
    return m


def tensors(seed, rows, n, nc, dtype, add):
    g = np.random.default_rng(seed)
    size = np.exp2(g.integers(-6, 7, size=(rows, 1)))
    h = rounded(size * g.normal(size=(rows, n)), dtype)[None]
    for c in range(1, nc):
        h = np.concatenate([h, rounded(h[0:1] * 2.0 ** (-12.0 * c) * g.normal(size=(1, rows, n)), dtype)])
    x = rounded(size * g.normal(size=(rows, n)), dtype) if add else None
    w = rounded(1 + 0.5 * g.normal(size=n), dtype)
    return h, x, w


def same_stream(got, want):
    got = host(got)
    assert np.array_equal(got, want, equal_nan=True), np.argwhere(got != want)[:4]


def check_plain(got, y, dtype):
    got = host(got)
    bound = np.abs(y) * (U[dtype] + 2.0 ** -24) * 1.01 + 2 * TINY[dtype]
    assert np.all(np.abs(got - y) <= bound), (np.abs(got - y) / bound).max()


def check_int8(pair, p, r, n):
    codes, scales = host(pair[0]), host(pair[1])
    c, s = ref.quantize(p, r)
    pitch = (n + 127) // 128 * 128
    assert codes.shape == (*c.shape[:-1], pitch) and not codes[..., n:].any()
    assert np.array_equal(codes[..., :n], c), np.argwhere(codes[..., :n] != c)[:4]
    assert np.array_equal(np.isnan(scales), np.isnan(s))
    ok = ~np.isnan(s)
    assert np.all(np.abs(scales[ok] - s[ok]) <= s[ok] * 2.0 ** -24 * 1.01 + 2.0 ** -150)


SIZES = [(1, 1), (3, 7), (5, 8), (17, 16), (37, 100), (300, 128), (9, 129), (5, 500), (4, 513), (3, 1000), (2, 2048),
         (3, 2049), (5, 4096), (2, 4100), (3, 8191), (2, 8200), (2, 16384), (2, 16400), (2, 40001), (41, 200), (40, 256)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nc", [1, 2, 3])
@pytest.mark.parametrize("rows, n", SIZES)
def test_forward(mcf, dtype, nc, rows, n):
    import torch

    for add in (False, True):
        h, x, w = tensors(rows + n, rows, n, nc, dtype, add)
        new, v = ref.stream(h, x, dtype)
        r = ref.inverse_rms(v, EPS)
        for weight in (None, w):
            p = v if weight is None else v * weight
            args = dev(h, dtype), None if weight is None else dev(weight, dtype)
            kw = dict(x=None if x is None else dev(x, dtype), eps=EPS, h_mc=True)
            y, stream = mcf.mc_rmsnorm_fwd(*args, **kw)
            pair, stream8 = mcf.mc_rmsnorm_int8(*args, **kw)
            same_stream(stream, new)
            same_stream(stream8, new)
            check_plain(y, p * r, dtype)
            check_int8(pair, p, r, n)
            if add:  # in place
                hp = args[0].clone()
                y2, back = mcf.mc_rmsnorm_fwd(hp, args[1], h_out=hp, **kw)
                assert back is hp and torch.equal(hp, stream) and torch.equal(y2, y)
        if not add:
            check_int8(mcf.mc_int8_quantize(dev(h, dtype), x_mc=True), v, 1.0, n)
            if nc == 1:
                y1, s1 = mcf.mc_rmsnorm_fwd(dev(h[0], dtype), eps=EPS)
                assert torch.equal(y1, mcf.mc_rmsnorm_fwd(dev(h, dtype), eps=EPS, h_mc=True)[0]) and s1.shape == (rows, n)


@pytest.mark.parametrize("dtype", DTYPES)
def test_ties_and_zeros(mcf, dtype):
    """Rows of small whole numbers, whose quotients are ties again and again; rows of zeros."""
    g = np.random.default_rng(3)
    v = g.integers(-20, 21, size=(40, 254)).astype(float)
    v[:, 0] = 127.0 * np.exp2(g.integers(0, 3, size=40))  # 127 p / m has halves
    v[5] = 0.0
    v[6] = -0.0
    w = np.exp2(g.integers(-3, 4, size=254))
    check_int8(mcf.mc_int8_quantize(dev(v, dtype)), v, 1.0, 254)
    check_int8(mcf.mc_rmsnorm_int8(dev(v, dtype), dev(w, dtype), eps=EPS)[0], v * w, ref.inverse_rms(v, EPS), 254)
    y, _ = mcf.mc_rmsnorm_fwd(dev(v, dtype), dev(w, dtype), eps=EPS)
    check_plain(y, v * w * ref.inverse_rms(v, EPS), dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_extremes(mcf, dtype):
    """The largest and smallest numbers of the format, infinities and NaN; eps of zero."""
    big = {"float16": 65504.0, "bfloat16": 3.3895314e38, "float32": 3.4028235e38}[dtype]
    low = {"float16": 2.0 ** -24, "bfloat16": 2.0 ** -133, "float32": 2.0 ** -149}[dtype]
    g = np.random.default_rng(4)
    v = g.normal(size=(8, 200))
    v[0] = rounded(big * g.uniform(-1, 1, 200), dtype)
    v[1] = low * g.integers(-9, 10, size=200)
    v[2, 50], v[3, 60], v[4, 70], v[4, 71] = np.inf, np.nan, -np.inf, np.inf
    v = rounded(v, dtype)
    w = rounded(np.where(np.arange(200) % 2, 1.5, big if dtype != "float16" else 100.0), dtype)
    for weight in (None, w):
        with np.errstate(all="ignore"):
            p = v if weight is None else v * weight
            r = ref.inverse_rms(v, EPS)
        pair, _ = mcf.mc_rmsnorm_int8(dev(v, dtype), None if weight is None else dev(weight, dtype), eps=EPS)
        check_int8(pair, p, r, 200)
    check_int8(mcf.mc_int8_quantize(dev(v, dtype)), v, 1.0, 200)
    y, _ = mcf.mc_rmsnorm_fwd(dev(v[:2], dtype), eps=0.0)
    check_plain(y, v[:2] * ref.inverse_rms(v[:2], 0.0), dtype)
    y, _ = mcf.mc_rmsnorm_fwd(dev(v[3:4], dtype), eps=EPS)
    assert np.isnan(host(y)).all()
    # the addition passes the format's range: an infinite stream with nothing in its low plane
    h = np.stack([np.full((1, 200), big), np.zeros((1, 200))])
    new, _ = ref.stream(h, np.full((1, 200), big), dtype)
    if dtype != "float16":
        assert np.isinf(new[0]).all() and not new[1].any()
    _, got = mcf.mc_rmsnorm_fwd(dev(h, dtype), x=dev(np.full((1, 200), big), dtype), eps=EPS, h_mc=True)
    same_stream(got, new)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [0, 1, 5, 127, 128, 1000, 20000])
def test_quantize_and_read_back(mcf, dtype, n):
    g = np.random.default_rng(n)
    x = rounded(g.normal(size=(2, 3, n)) * np.exp2(g.integers(-9, 9, size=(2, 3, 1))), dtype)
    codes, scales = mcf.mc_int8_quantize(dev(x, dtype))
    assert codes.shape == (2, 3, (n + 127) // 128 * 128) and scales.shape == (2, 3)
    check_int8((codes, scales), x, 1.0, n)
    for out in DTYPES:
        import torch

        got = mcf.mc_int8_dequantize(codes, scales, n, dtype=getattr(torch, out))
        want = host(codes)[..., :n].astype(np.float32) * host(scales).astype(np.float32)[..., None]
        assert np.array_equal(host(got), rounded(want, out))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nc", [1, 2])
@pytest.mark.parametrize("rows, n", [(1, 1), (3, 7), (700, 40), (513, 64), (9, 129), (5, 513), (1100, 1000), (3, 2049),
                                     (4, 4100), (530, 4096), (3, 8200), (2, 16384), (5, 16400), (2, 40001), (9000, 200),
                                     (2100, 600), (300, 5000)])
def test_gradients(mcf, dtype, nc, rows, n):
    import torch

    h, _, w = tensors(rows * n, rows, n, nc, dtype, False)
    g = np.random.default_rng(7)
    dy, later = rounded(g.normal(size=(rows, n)), dtype), rounded(g.normal(size=(rows, n)), dtype)
    v = ref.planes_sum(h)
    r = ref.inverse_rms(v, EPS)
    th, tdy, tlater = dev(h, dtype), dev(dy, dtype), dev(later, dtype)
    for weight, gr in ((w, later), (None, None)):
        dh, dw = ref.norm_bwd(v, weight, dy, gr, EPS)
        tw = None if weight is None else dev(weight, dtype)
        got_h, got_w = mcf.mc_rmsnorm_bwd(th, tw, tdy, dh=None if gr is None else tlater, eps=EPS, h_mc=True)
        p = np.abs(dy if weight is None else weight * dy)
        terms = r * (p + np.abs(v) * r * r * (np.abs(v) * p).sum(-1, keepdims=True) / n) + (0 if gr is None else np.abs(gr))
        bound = np.abs(dh) * (U[dtype] + 2.0 ** -24) * 1.01 + (n + 20) * 2.0 ** -52 * terms + 2 * TINY[dtype]
        assert np.all(np.abs(host(got_h) - dh) <= bound), (np.abs(host(got_h) - dh) / bound).max()
        size = (np.abs(dy * v) * r).sum(0)
        bound = np.abs(dw) * (U[dtype] + 2.0 ** -24) * 1.01 + (2.0 ** -24 * 1.01 + (n + rows) * 2.0 ** -52) * size + 2 * TINY[dtype]
        assert np.all(np.abs(host(got_w) - dw) <= bound), (np.abs(host(got_w) - dw) / bound).max()
        # each alone has the same bits
        a, none = mcf.mc_rmsnorm_bwd(th, tw, tdy, dh=None if gr is None else tlater, eps=EPS, h_mc=True, dw=False)
        assert none is None and torch.equal(a, got_h)
        none, b = mcf.mc_rmsnorm_bwd(th, tw, tdy, eps=EPS, h_mc=True, dx=False)
        assert none is None and torch.equal(b, got_w)


def test_gradients_by_differences(mcf):
    """Differences of the library's own forward pass in binary32.  A step of 2^-7 of the unit leaves
    its third derivative's part, below 2^-14 of the gradient's size here, and 2 2^-24 |y| 2^7 of rounding per
    output; the loss is summed in binary64."""
    g = np.random.default_rng(11)
    rows, n, step = 2, 24, 2.0 ** -7
    v, w, dy = (g.normal(size=s).astype(np.float32) for s in ((rows, n), n, (rows, n)))
    dh, dw = mcf.mc_rmsnorm_bwd(dev(v), dev(w), dev(dy), eps=1e-3)

    def loss(v, w):
        y, _ = mcf.mc_rmsnorm_fwd(dev(v), dev(w), eps=1e-3)
        return (host(y) * dy).sum()

    tol = 24 * 2.0 ** -24 * 4 * 4 / step + 2.0 ** -12 * 8
    for i in range(n):
        e = np.zeros_like(v)
        e[1, i] = step
        assert abs((loss(v + e, w) - loss(v - e, w)) / (2 * step) - host(dh)[1, i]) < tol
        e = np.zeros_like(w)
        e[i] = step
        assert abs((loss(v, w + e) - loss(v, w - e)) / (2 * step) - host(dw)[i]) < tol


def test_no_rows(mcf):
    import torch

    h = torch.empty(0, 300, device="cuda")
    y, s = mcf.mc_rmsnorm_fwd(h)
    assert y.shape == (0, 300) and s is h
    (codes, scales), _ = mcf.mc_rmsnorm_int8(h)
    assert codes.shape == (0, 384) and scales.shape == (0,)
    for n in (300, 20000):
        h = torch.empty(0, n, device="cuda")
        dh, dw = mcf.mc_rmsnorm_bwd(h, None, h)
        assert dh.shape == (0, n) and dw.shape == (n,) and not dw.any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nc", [1, 2])
@pytest.mark.parametrize("n", [5, 200, 1000, 1023, 4096, 5000, 20000])
def test_a_row_alone(mcf, dtype, nc, n):
    """A row's results have the same bits alone, among few and among many."""
    import torch

    h, x, w = (dev(t, dtype) for t in tensors(n, 300, n, nc, dtype, True))
    (codes, scales), stream = mcf.mc_rmsnorm_int8(h, w, x=x, eps=EPS, h_mc=True)
    y, _ = mcf.mc_rmsnorm_fwd(h, w, x=x, eps=EPS, h_mc=True)
    dx, _ = mcf.mc_rmsnorm_bwd(stream, w, x, eps=EPS, h_mc=True)
    for lo, hi in ((7, 8), (120, 137)):
        a, b = h[:, lo:hi].contiguous(), x[lo:hi].contiguous()
        (c, s), st = mcf.mc_rmsnorm_int8(a, w, x=b, eps=EPS, h_mc=True)
        assert torch.equal(c, codes[lo:hi]) and torch.equal(s, scales[lo:hi]) and torch.equal(st, stream[:, lo:hi])
        assert torch.equal(mcf.mc_rmsnorm_fwd(a, w, x=b, eps=EPS, h_mc=True)[0], y[lo:hi])
        assert torch.equal(mcf.mc_rmsnorm_bwd(st, w, b, eps=EPS, h_mc=True)[0], dx[lo:hi])


def test_many_short_rows(mcf):
    """More rows than one launch takes."""
    import torch

    rows, n = (1 << 21) + 77, 3
    h = torch.randn(rows, n, device="cuda").bfloat16()
    y, _ = mcf.mc_rmsnorm_fwd(h, eps=EPS)
    (codes, scales), _ = mcf.mc_rmsnorm_int8(h, eps=EPS)
    for lo in (0, (1 << 21) - 40, rows - 100):
        v = host(h[lo:lo + 100])
        r = ref.inverse_rms(v, EPS)
        check_plain(y[lo:lo + 100], v * r, "bfloat16")
        check_int8((codes[lo:lo + 100], scales[lo:lo + 100]), v, r, n)
    dy = torch.randn(rows, n, device="cuda").bfloat16()
    dh, dw = mcf.mc_rmsnorm_bwd(h, None, dy, eps=EPS)
    v = h.double()
    r = ((v * v).mean(-1, keepdim=True) + EPS).rsqrt()
    want = (dy.double() * v * r)
    assert bool(((dw.double() - want.sum(0)).abs() <= want.sum(0).abs() * 2.0 ** -7.9 + 2.0 ** -23 * want.abs().sum(0)).all())


def test_long_tensor(mcf):
    """Offsets past 32 bits: 2^31 elements and more."""
    import torch

    rows, n = 262200, 8200
    h = torch.zeros(rows, n, device="cuda", dtype=torch.bfloat16)
    g = np.random.default_rng(5)
    v = rounded(g.normal(size=(3, n)), "bfloat16")
    h[-3:] = dev(v, "bfloat16")
    pair, _ = mcf.mc_rmsnorm_int8(h, eps=EPS)
    check_int8((pair[0][-3:], pair[1][-3:]), v, ref.inverse_rms(v, EPS), n)
    assert not bool(pair[1][:-3].any())
    y, _ = mcf.mc_rmsnorm_fwd(h, eps=EPS)
    check_plain(y[-3:], v * ref.inverse_rms(v, EPS), "bfloat16")
    back = mcf.mc_int8_dequantize(*pair, n, dtype=torch.bfloat16, out=y)
    want = host(pair[0][-3:])[:, :n].astype(np.float32) * host(pair[1][-3:]).astype(np.float32)[:, None]
    assert np.array_equal(host(back[-3:]), rounded(want, "bfloat16"))
    del back, pair
    dh, dw = mcf.mc_rmsnorm_bwd(h, None, y, eps=EPS)
    want_h, want_w = ref.norm_bwd(v, None, host(y[-3:]), None, EPS)
    assert np.all(np.abs(host(dw) - want_w) <= np.abs(want_w) * 2.0 ** -7.9 + 2.0 ** -22 * (np.abs(host(y[-3:]) * v)).sum(0))
    assert np.all(np.abs(host(dh[-3:]) - want_h) <= np.abs(want_h) * 2.0 ** -7.9 + 1e-9)
