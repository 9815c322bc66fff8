"""The distillation loss from a teacher's top logits and its gradient on the GPU, against a plain
binary64 form and against differences of the loss.

Tolerances.  With d the largest |z - m| / T that counts (exp of less than -100 is nothing), the
argument of an exponential is off by at most 4 d 2^-24 and its value by as much, relatively; a
sum of n terms adds at most (n / 64 + 32) 2^-24 (64 lanes or more add apart, then join).  So q is
within e_q = (4 d + V / 64 + 32) 2^-24 of its value, p within e_p alike, a loss within
T^2 (sum p |log p - log q| e_p + e_p + e_q + 4 2^-24 sum p (|log p| + |log q|)), and a gradient
within |g| T (q e_q + p e_p) plus its rounding to the format."""
import numpy as np
import pytest

import mx4_reference as ref
from test_gpu_mx4 import DTYPES, U, dev, host, rounded

pytestmark = pytest.mark.gpu

TINY = {"float16": 2.0 ** -25, "bfloat16": 2.0 ** -133, "float32": 2.0 ** -126}


@pytest.fixture(scope="module")
def mcf():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2207_08867_amd as m

    m.lib()
    return m


def batch(seed, rows, V, k, dtype, nc=1):
    g = np.random.default_rng(seed)
    z = np.stack([rounded(3.0 * g.normal(size=(rows, V)), dtype)] +
                 [rounded(2.0 ** (-8 * c) * g.normal(size=(rows, V)), dtype) for c in range(1, nc)])
    t = rounded(3.0 * g.normal(size=(rows, k)), dtype)
    ids = np.stack([g.permutation(V)[:k] if V >= k else g.integers(0, V, k) for _ in range(rows)]).astype(np.int32)
    up = g.uniform(-1, 1, rows).astype(np.float32)
    return z, ids.reshape(rows, k), t, up


def check(mcf, z, ids, t, g, T, dtype):
    """All three calls against the plain form; returns their results."""
    planes = z if z.ndim == 3 else z[None]
    total = planes[-1].astype(np.float32)
    for p in planes[-2::-1]:
        total = total + p.astype(np.float32)
    rows, V = total.shape
    loss, dz = ref.distill(total, ids, t, g, T)
    tz = dev(planes if planes.shape[0] > 1 else planes[0], dtype)
    args = tz, dev(ids), dev(t, dtype)
    tg = dev(g)
    l1, stats = mcf.mc_distill_fwd(*args, temperature=T)
    d1 = mcf.mc_distill_bwd(*args, stats, tg, temperature=T)
    l2, d2 = mcf.mc_distill_fwd_bwd(*args, tg, temperature=T)
    assert l1.shape == (rows,) and d1.shape == (rows, V) and d1.dtype == tz.dtype
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        top = np.max(np.where(np.isfinite(total), total, -1e30), -1, keepdims=True)
        q = np.exp((total - top) / T)
        q = q / np.maximum(q.sum(-1, keepdims=True), 1e-300)
        e = (4 * 100 + max(V, ids.shape[1]) / 64 + 32) * 2.0 ** -24
        zs = np.abs(np.where(np.isfinite(total), total - top, 0)).max(-1) / T
        ts = np.abs(np.where(np.isfinite(t), t, 0)).max(-1) / T * 2 if t.shape[1] else np.zeros(rows)
        size = zs + ts + np.log(V) + 8
    lossb = T * T * (size * (e + 4 * 2.0 ** -24) + 2 * e)
    gradb = np.abs(g)[:, None] * T * (q + 1.0 * (np.abs(dz) > 0)) * e
    # the p of an entry is at most |dz| / (|g| T) + q
    gradb = np.minimum(gradb, (np.abs(dz) + 2 * np.abs(g)[:, None] * T * q) * e) + U[dtype] * np.abs(dz) * 1.01 + TINY[dtype]
    for name, got in (("fwd", host(l1)), ("fused", host(l2))):
        same = (got == loss) | (np.isnan(got) & np.isnan(loss))
        assert np.all(same | (np.abs(got - loss) <= lossb)), (name, got, loss)
    for name, got in (("bwd", host(d1)), ("fused", host(d2))):
        bad = ~((np.abs(got - dz) <= gradb) | (np.isnan(got) & np.isnan(dz)))
        assert not bad.any(), (name, np.argwhere(bad)[:4], got[bad][:4], dz[bad][:4])
    return l1, d1, l2, d2


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1.0, 2.5])
@pytest.mark.parametrize("rows, V, k", [(1, 1, 1), (3, 7, 4), (5, 100, 8), (300, 257, 5), (2, 512, 64), (3, 513, 3),
                                        (4, 2049, 16), (2, 8192, 32), (3, 8193, 32), (2, 32768, 64), (260, 8200, 7),
                                        (257, 33001, 12), (1, 131071, 100), (3, 4100, 1024)])
def test_rows(mcf, dtype, T, rows, V, k):
    z, ids, t, g = batch(rows + V, rows, V, k, dtype)
    check(mcf, z, ids, t, g, T, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nc", [2, 3, 4])
@pytest.mark.parametrize("rows, V", [(5, 300), (3, 9000), (260, 9001)])
def test_mc_logits(mcf, dtype, nc, rows, V):
    z, ids, t, g = batch(nc, rows, V, 6, dtype, nc)
    check(mcf, z, ids, t, g, 1.5, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 600, 9000])
def test_masks_and_padding(mcf, dtype, V):
    """Unused entries, rows with none, masked logits, entries that the student has masked,
    duplicates, the type's lowest value as a mask, NaN and infinities."""
    rows, k = 14, 8
    z, ids, t, g = batch(V, rows, V, k, dtype)
    z = z[0]
    low = rounded(np.array([{"float16": -65504.0, "bfloat16": -3.3895314e38, "float32": -3.4028235e38}[dtype]]), dtype)[0]
    ids[0, 3:] = -1
    ids[1, :] = -1  # no entry
    ids[2, 1], ids[2, 2] = V, 2 ** 31 - 1  # outside the vocabulary
    t[3, 2:5] = -np.inf
    t[4, :] = -np.inf  # none above -inf
    z[5, V // 2:] = -np.inf
    ids[5] = np.arange(k)
    z[6, ids[6, 0]] = -np.inf  # the loss is infinite
    t[7, 1] = -np.inf
    z[7, ids[7, 1]] = -np.inf  # p = 0 there: no contribution
    ids[8, 1] = ids[8, 0]
    ids[8, 5] = ids[8, 0]
    z[9, 1:] = low
    z[10, :] = -np.inf  # nothing left: q = 0, the loss infinite
    z[11, 3] = np.nan
    t[12, 2] = np.nan
    z[13, :] = low
    loss, dz = ref.distill(z, ids, t, g, 1.0)
    loss[11] = np.nan
    dz[11] = np.nan
    args = dev(z, dtype), dev(ids), dev(t, dtype)
    l1, stats = mcf.mc_distill_fwd(*args)
    d1 = mcf.mc_distill_bwd(*args, stats, dev(g))
    l2, d2 = mcf.mc_distill_fwd_bwd(*args, dev(g))
    rowset = [r for r in range(rows) if r not in (11, 12)]
    for l, d in ((l1, d1), (l2, d2)):
        l, d = host(l), host(d)
        assert l[1] == 0 and l[4] == 0 and not d[1].any() and not d[4].any()
        assert l[6] == np.inf and l[10] == np.inf
        assert np.isnan(l[11]) and np.isnan(l[12]) and np.isnan(d[11]).any() and np.isnan(d[12]).any()
        assert np.allclose(l[rowset], loss[rowset], rtol=2e-5, atol=2e-5)
        assert np.allclose(d[rowset], dz[rowset], rtol=2e-5 + 2 * U[dtype], atol=2e-5 + 2 * U[dtype])


def test_no_entries_and_no_rows(mcf):
    import torch

    z = torch.randn(3, 50, device="cuda")
    ids, t = torch.empty(3, 0, dtype=torch.int32, device="cuda"), torch.empty(3, 0, device="cuda")
    loss, dz = mcf.mc_distill_fwd_bwd(z, ids, t)
    assert not loss.any() and not dz.any()
    loss, stats = mcf.mc_distill_fwd(z[:0], ids[:0], t[:0])
    assert loss.shape == (0,) and mcf.mc_distill_bwd(z[:0], ids[:0], t[:0], stats).shape == (0, 50)


@pytest.mark.parametrize("V", [300, 20000])
@pytest.mark.parametrize("T", [1.0, 3.0])
def test_gradient_by_differences(mcf, V, T):
    """sum dz d against (L(z + h d) - L(z - h d)) / 2 h along d in {-1, 0, 1}: the third
    derivative of a log-sum-exp along such a d is at most T^-3, so the difference's error is at
    most T^2 h^2 / (6 T^3), and the losses' own error e gives e / h."""
    rows, k, h = 6, 10, 2.0 ** -5
    z, ids, t, g = batch(V, rows, V, k, "float32")
    z = z[0]
    d = np.random.default_rng(1).integers(-1, 2, z.shape).astype(float)
    _, dz = mcf.mc_distill_fwd_bwd(dev(z, "float32"), dev(ids), dev(t, "float32"), temperature=T)
    up, _ = mcf.mc_distill_fwd(dev(z + h * d, "float32"), dev(ids), dev(t, "float32"), temperature=T)
    down, _ = mcf.mc_distill_fwd(dev(z - h * d, "float32"), dev(ids), dev(t, "float32"), temperature=T)
    slope = (host(up) - host(down)) / (2 * h)
    e = T * T * 40 * (4 * 100 + V / 64 + 32) * 2.0 ** -24
    # z +- h d is rounded to binary32: at most 2^-21 of a logit below 16, for every logit
    assert np.all(np.abs((host(dz) * d).sum(-1) - slope) <= h * h / (6 * T) + e / h + T * 2.0 ** -21 / h)


def test_refusals(mcf):
    import torch

    z, ids, t = torch.randn(3, 50, device="cuda"), torch.zeros(3, 2, dtype=torch.int32, device="cuda"), torch.randn(3, 2, device="cuda")
    with pytest.raises(TypeError):
        mcf.mc_distill_fwd(z, ids.long(), t)
    with pytest.raises(TypeError):
        mcf.mc_distill_fwd(z.double(), ids, t.double())
    with pytest.raises(ValueError):
        mcf.mc_distill_fwd(z, ids, t.half())
    with pytest.raises(ValueError):
        mcf.mc_distill_fwd(z, ids[:2], t)
    with pytest.raises(ValueError):
        mcf.mc_distill_fwd(z, ids, t, temperature=0.0)
    with pytest.raises(ValueError):
        mcf.mc_distill_fwd(z, ids, t, temperature=float("nan"))
    with pytest.raises(ValueError):
        mcf.mc_distill_fwd_bwd(z, ids, t, torch.ones(3, device="cuda").half())
    with pytest.raises(ValueError):
        mcf.mc_distill_fwd_bwd(z, ids, t, out=z)
    with pytest.raises(ValueError):
        mcf.mc_distill_bwd(z, ids, t, torch.zeros(3, device="cuda"))
    with pytest.raises(ValueError):
        mcf.mc_distill_fwd(torch.randn(50, 3, device="cuda").t(), ids, t)
    many = torch.zeros(3, 1025, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        mcf.mc_distill_fwd(z, many, torch.zeros(3, 1025, device="cuda"))


def test_graph_replays(mcf):
    """Captured once and replayed with new contents, the eager calls' results every time."""
    import torch

    z, ids, t, g = batch(3, 40, 20000, 8, "bfloat16")
    tz, tids, tt, tg = dev(z[0], "bfloat16"), dev(ids), dev(t, "bfloat16"), dev(g)
    x = torch.randn(40, 256, device="cuda").bfloat16()
    W = mcf.mc_mx4_quantize(torch.randn(20000, 256, device="cuda").bfloat16())

    def step():
        y = mcf.mc_mx4_linear_fwd(x, W)
        loss, dz = mcf.mc_distill_fwd_bwd(y, tids, tt, tg)
        return (loss, dz) + mcf.mc_mx4_linear_bwd(x, W, dz)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        x.copy_(torch.randn(40, 256, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_many_logits(mcf):
    """More than 2^31 logits: sampled rows against the same rows alone."""
    import torch

    rows, V, k = 16500, 131072, 4
    z = torch.empty(rows, V, device="cuda", dtype=torch.bfloat16)
    z[:] = torch.randn(V, device="cuda").bfloat16()
    pick = [0, 5, 8191, 16384, rows - 1]
    for i in pick:
        z[i] = torch.randn(V, device="cuda").bfloat16()
    ids = torch.randint(0, V, (rows, k), device="cuda", dtype=torch.int32)
    t = torch.randn(rows, k, device="cuda").bfloat16()
    loss, stats = mcf.mc_distill_fwd(z, ids, t)
    dz = mcf.mc_distill_bwd(z, ids, t, stats)
    for i in pick:
        l, d = mcf.mc_distill_fwd_bwd(z[i:i + 1], ids[i:i + 1], t[i:i + 1])
        assert torch.allclose(l, loss[i:i + 1], rtol=1e-5, atol=1e-5)
        assert (d.float() - dz[i:i + 1].float()).abs().max() <= 2.0 ** -7 * d.float().abs().max()


def test_more_rows_than_one_launch(mcf):
    """Past 2^21 rows the workgroups go out in several launches: the same rows over and over."""
    import torch

    part, times = 70001, 31
    z = torch.randn(part, 5, device="cuda").half()
    ids = torch.randint(0, 5, (part, 2), device="cuda", dtype=torch.int32)
    t = torch.randn(part, 2, device="cuda").half()
    loss, stats = mcf.mc_distill_fwd(z, ids, t)
    _, dz = mcf.mc_distill_fwd_bwd(z, ids, t)
    many = [v.repeat(times, 1) for v in (z, ids, t)]
    assert many[0].shape[0] > 2 ** 21
    got_loss, got_stats = mcf.mc_distill_fwd(*many)
    assert torch.equal(got_loss.view(times, part), loss.expand(times, part))
    assert torch.equal(got_stats.view(times, part, 2), stats.expand(times, part, 2))
    got_loss, got = mcf.mc_distill_fwd_bwd(*many)
    assert torch.equal(got_loss.view(times, part), loss.expand(times, part))
    assert torch.equal(got.view(times, part, 5), dz.expand(times, part, 5))
    assert torch.equal(mcf.mc_distill_bwd(*many, got_stats), got)
