"""Log probabilities of given tokens, entropy, top alternatives and their gradient on the GPU against
plain binary64 forms and against differences.  Alternatives must come out exactly.

Tolerances, e = 2^-24.  With d = (m - z) / T, a term exp(-d) has a relative error of (2 d + 2) e: the difference
and the product are rounded, the exponential is off by a unit in the last place.  A sum of s terms over 64 elements
a thread, then joined in at most 32 steps, adds 96 e, and what chunks are joined with 4 more.  So
  err(L) <= rest / (1 + rest) (2 avg(d) + 106) e + 4 e L,
avg over the terms of the rest, weighted by them; B = sum q d has the terms' (2 d + 6) e, weighted by q d, and 106 e and
the sum's own; log q = -d - L adds 4 d e and its rounding.  The gradient's q has (2 d + 8) e and err(L)."""
import numpy as np
import pytest

import lm_reference as ref
from lm_reference import DTYPES, TINY, U, dev, host, rounded

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


@pytest.fixture(scope="module")
def mcf():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2207_08867_amd as m

    m.lib()
    return m


def near(got, want, bound, what):
    # a value past binary32's range (the difference of its largest number and its lowest) rounds to infinity
    with np.errstate(invalid="ignore"):
        want = np.where(np.abs(want) >= (2 - 2.0 ** -24) * 2.0 ** 127, np.sign(want) * np.inf, want)
        ok = (got == want) | (np.isnan(got) & np.isnan(want)) | (np.abs(got - want) <= bound)
    assert ok.all(), (what, np.argwhere(~ok)[:4], got[~ok][:4], want[~ok][:4])


def total(planes):
    s = planes[-1].astype(np.float32)
    for p in planes[-2::-1]:
        s = p.astype(np.float32) + s
    return s.astype(np.float64)


def check(mcf, z, ids, k, T, dtype, g=None, gh=None):
    """Both calls against the plain form; rows of finite or -inf logits.  Returns the results."""
    planes = z if z.ndim == 3 else z[None]
    s = total(planes)
    rows, V = s.shape
    want_g = np.ones(ids.shape) if g is None else g
    logp, ent, logq, dz = ref.logprobs(s, ids, T, want_g, gh)
    tz = dev(planes if len(planes) > 1 else planes[0], dtype)
    tids = dev(ids.astype(np.int32))
    out = mcf.mc_logprobs_fwd(tz, tids, top=k, temperature=T)
    got_p, got_h, top_ids, top_logp, stats = out
    got_z = mcf.mc_logprobs_bwd(tz, tids, stats, None if g is None else dev(g.astype(np.float32)),
                                None if gh is None else dev(gh.astype(np.float32)), temperature=T)
    assert got_z.dtype == tz.dtype and got_z.shape == (rows, V)
    with np.errstate(all="ignore"):
        q = np.exp(logq)
        some = np.isfinite(s.max(-1))
        d = np.where(q > 0, (s.max(-1, keepdims=True) - s) / T, 0.0)
        L = np.where(some, -np.where(some[:, None], logq, 0).max(-1), 0.0)
        qd = (q * d).sum(-1)
        rest = -np.expm1(-L)  # the share of the others: 1 - exp(-L) is 0 in binary64 for a sure row
        avg = np.where(qd > 0, qd / np.maximum(rest, 1e-300), 0.0)
        eL = rest * (2 * np.minimum(avg, 104) + 106) * E * 1.1 + 4 * E * L
        avg2 = np.where(qd > 0, (q * d * d).sum(-1) / np.maximum(qd, 1e-300), 0.0)
        eB = qd * ((2 * avg2 + 112) * E * 1.1 + eL + 4 * E)
        dt = np.where(np.isfinite(logq), -logq - L[:, None], 0.0)
    eP = eL[:, None] + 4 * E * dt + E * np.abs(np.where(np.isfinite(logq), logq, 0.0))
    used = (ids >= 0) & (ids < V)
    at = np.where(used, ids, 0)
    near(host(got_p), logp, np.take_along_axis(eP, at, 1) * 1.01 + 1e-38, "logp")
    near(host(got_h), ent, (eL + eB + E * ent) * 1.01 + 1e-38, "entropy")
    if k:
        want = ref.top(s, k)
        assert np.array_equal(host(top_ids), want), np.argwhere(host(top_ids) != want)[:4]
        at = np.maximum(want, 0)
        near(host(top_logp), np.where(want < 0, -np.inf, np.take_along_axis(logq, at, 1)),
             np.take_along_axis(eP, at, 1) * 1.01 + 1e-38, "top")
    else:
        assert top_ids.shape == (rows, 0) and top_logp.shape == (rows, 0)
    G = np.where(used, want_g, 0.0)
    size = np.abs(G.sum(-1, keepdims=True)) + np.abs(G).sum(-1, keepdims=True) * (ids.shape[1] + 2) * E
    slope = np.zeros((rows, 1)) if gh is None else np.abs(gh)[:, None]
    lq = np.where(q > 0, np.abs(np.where(np.isfinite(logq), logq, 0.0) + ent[:, None]), 0.0)
    e_slope = np.where(q > 0, eB[:, None] + eL[:, None] + 4 * E * dt + 4 * E * (ent[:, None] + dt + lq), 0.0)
    bound = q / T * ((size + slope * lq) * ((2 * dt + 12) * E + eL[:, None]) + slope * e_slope)
    bound += q / T * np.abs(G).sum(-1, keepdims=True) * (ids.shape[1] + 2) * E
    for i in range(ids.shape[1]):
        np.add.at(bound, (np.arange(rows), np.where(used[:, i], ids[:, i], 0)), np.abs(G[:, i]) / T * (ids.shape[1] + 4) * E)
    near(host(got_z), dz, bound * 1.05 + (np.abs(dz) + bound) * U[dtype] * 1.01 + TINY[dtype] * 2 + 1e-38, "dz")
    return (*out, got_z)


def batch(seed, rows, V, given, dtype, nc=1):
    g = np.random.default_rng(seed)
    z = np.stack([rounded(3.0 * g.normal(size=(rows, V)), dtype)] +
                 [rounded(2.0 ** (-8 * c) * g.normal(size=(rows, V)), dtype) for c in range(1, nc)])
    ids = g.integers(0, V, size=(rows, given))
    ids[g.random(size=ids.shape) < 0.1] = -1
    return z, ids, g.uniform(-1, 1, size=(rows, given)).astype(np.float32), g.uniform(-1, 1, rows).astype(np.float32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1.0, 0.7])
@pytest.mark.parametrize("rows, V, given, k", [(1, 1, 1, 1), (3, 2, 2, 5), (3, 7, 1, 0), (5, 100, 3, 8), (300, 257, 1, 5), (2, 512, 4, 128),
                                               (3, 513, 1, 64), (4, 2049, 2, 20), (256, 4100, 1, 20), (2, 8192, 1, 32), (3, 8193, 1, 128),
                                               (2, 32768, 5, 64), (257, 9000, 1, 1), (256, 16390, 2, 7), (256, 32769, 1, 128),
                                               (257, 70000, 1, 20), (1, 131071, 1, 100), (3, 4100, 1024, 3), (2, 40, 0, 0),
                                               (3, 1000, 12, 128), (2, 32768, 1, 128), (2, 1000, 65, 64), (2, 200, 9, 100),
                                               (66, 100000, 1, 128), (2, 5001, 2, 128), (2, 12001, 2, 64), (2, 20001, 10, 64), (2, 28001, 2, 128),
                                               (130, 34003, 1, 30), (64, 42001, 1, 64), (64, 49999, 1, 64), (64, 65001, 1, 64)])
def test_rows(mcf, dtype, T, rows, V, given, k):
    z, ids, g, gh = batch(rows + V, rows, V, given, dtype)
    check(mcf, z, ids, k, T, dtype, g, gh)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nc", [2, 3, 4])
@pytest.mark.parametrize("rows, V", [(5, 300), (3, 9000), (260, 9001)])
def test_mc_logits(mcf, dtype, nc, rows, V):
    z, ids, g, gh = batch(nc, rows, V, 2, dtype, nc)
    check(mcf, z, ids, 20, 1.5, dtype, g, gh)


def test_defaults(mcf):
    """No upstream gradients given: ones for the tokens, none for the entropy."""
    z, ids, _, _ = batch(3, 6, 900, 2, "float32")
    check(mcf, z, ids, 3, 1.0, "float32")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 600, 9000])
def test_masks_and_special_tokens(mcf, dtype, V):
    low = rounded(np.array([{"float16": -65504.0, "bfloat16": -3.3895314e38, "float32": -3.4028235e38}[dtype]]), dtype)[0]
    z, ids, g, gh = batch(V, 10, V, 4, dtype)
    z = z[0]
    z[0, V // 2:] = -np.inf  # a masked half
    ids[0] = [0, V - 1, V // 2, 1]  # tokens in it
    z[1] = -np.inf  # nothing left
    z[2, 3:] = -np.inf  # fewer logits than alternatives
    z[3] = low  # masks of the lowest value alone
    z[4, V // 3:] = low
    z[5, 1:] = low
    z[5, 0] = -low  # the format's whole range
    ids[6] = [7, 7, 7, -1]  # one token several times
    ids[7] = [-1, V, 2 ** 31 - 1, -2 ** 31]  # none
    z[8] = 0.0  # all alike
    z[8, ::2] = -0.0
    z[9, 5] = z[9].max() + (30.0 if dtype == "float32" else 16.0)  # a row that is sure
    ids[9] = [5, 0, 1, 5]
    z = rounded(z, dtype)  # what the call is given
    for T in (1.0, 0.7, 3.0):
        check(mcf, z, ids, 20, T, dtype, g, gh)
        check(mcf, z, ids, 0, T, dtype, g, None)


def test_sure_rows_keep_relative_accuracy(mcf):
    """log q of the largest logit far below binary32's step at one."""
    for V in (50, 5000, 20000, 40000):
        z = np.full((2, V), -40.0, np.float32)
        z[0, 17], z[1, V - 1] = 3.0, 0.0
        ids = np.array([[17], [V - 1]])
        logp, ent, ids_, lp, _, _ = check(mcf, z, ids, 1, 1.0, "float32", np.ones((2, 1), np.float32), np.ones(2, np.float32))
        for r, d in enumerate((43.0, 40.0)):
            want = -np.log1p((V - 1) * np.exp(-d))
            assert abs(host(logp)[r, 0] - want) <= 3e-5 * abs(want) and host(lp)[r, 0] == host(logp)[r, 0]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [300, 3000, 20000, 40001])
@pytest.mark.parametrize("rows", [3, 256])
def test_top_orders(mcf, dtype, V, rows):
    """Rows in ascending and descending order, steps of equal logits, all alike, the largest side by side,
    signed zeros: the order by logit, then index."""
    if rows > 3 and V < 9000:
        pytest.skip("rows of one workgroup either way")
    j = np.arange(V)
    kinds = [j / V * 8, -j / V * 8, j // 64 * 0.5, -(j // 100) * 0.25, np.zeros(V), np.where(j % 2, 0.0, -0.0),
             np.where((j >= V // 2) & (j < V // 2 + 300), 5.0, -1.0), (j * 7919 % 13).astype(float),
             np.where(j < V - 3, -np.inf, 1.0)]
    for k in (1, 64, 128):
        for i in range(0, len(kinds), 3):
            z = rounded(np.stack([kinds[(i + r) % len(kinds)] for r in range(min(rows, 3))]), dtype)
            z = np.concatenate([z] * ((rows + 2) // 3))[:rows]
            got = mcf.mc_logprobs_fwd(dev(z, dtype), dev(np.zeros((rows, 1), np.int32)), top=k)
            want = ref.top(z, k)
            assert np.array_equal(host(got[2]), want), (k, i, np.argwhere(host(got[2]) != want)[:4])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [60, 5000, 20000, 40000])
def test_non_finite(mcf, dtype, V):
    """NaN and +inf: NaN everywhere and no alternatives; the rows beside them are whole."""
    z, ids, g, gh = batch(V, 6, V, 2, dtype)
    z = z[0]
    ids[:, 0], ids[:, 1] = 3, -1
    clean = check(mcf, z, ids, 9, 1.0, dtype, g, gh)
    bad = z.copy()
    bad[0, V - 1], bad[1, 7], bad[3, 0] = np.nan, np.inf, np.nan
    bad[3, 1:] = -np.inf
    bad[4, V // 2] = np.inf
    bad[4, 5:9] = np.nan
    tz, tids = dev(bad, dtype), dev(ids.astype(np.int32))
    logp, ent, top_ids, top_logp, stats = mcf.mc_logprobs_fwd(tz, tids, top=9)
    dz = mcf.mc_logprobs_bwd(tz, tids, stats, dev(g), dev(gh))
    for r in (0, 1, 3, 4):
        assert np.isnan(host(logp)[r, 0]) and host(logp)[r, 1] == 0.0 and np.isnan(host(ent)[r])
        assert (host(top_ids)[r] == -1).all() and np.isnan(host(top_logp)[r]).all() and np.isnan(host(dz)[r]).all()
    for r in (2, 5):
        for a, b in zip((logp, ent, top_ids, top_logp, stats, dz), clean):
            assert np.array_equal(host(a)[r], host(b)[r])


def test_gradient_by_differences(mcf):
    """Differences of the library's own forward pass in binary32: a step of 2^-6 leaves 2^-12 of third
    derivatives, the outputs (below 8) are within 2^-20, over 2 2^-6."""
    z, ids, g, gh = batch(5, 2, 30, 3, "float32")
    ids[0] = [4, 4, 9]
    z, step, T = z[0], 2.0 ** -6, 1.5

    def value(z):
        logp, ent, _, _, stats = mcf.mc_logprobs_fwd(dev(z, "float32"), dev(ids.astype(np.int32)), temperature=T)
        return (g * host(logp)).sum(-1) + gh * host(ent), stats

    dz = host(mcf.mc_logprobs_bwd(dev(z, "float32"), dev(ids.astype(np.int32)), value(z)[1], dev(g), dev(gh), temperature=T))
    for j in range(30):
        e = np.zeros_like(z)
        e[:, j] = step
        diff = (value(rounded(z + e, "float32"))[0] - value(rounded(z - e, "float32"))[0]) / (2 * step)
        assert np.all(np.abs(diff - dz[:, j]) < 2.0 ** -10 + 4 * 2.0 ** -20 / step)


def test_no_rows(mcf):
    import torch

    z, ids = torch.empty(0, 50, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda")
    logp, ent, ti, tl, stats = mcf.mc_logprobs_fwd(z, ids, top=4)
    assert logp.shape == (0, 2) and ent.shape == (0,) and ti.shape == tl.shape == (0, 4) and stats.shape == (0, 3)
    assert mcf.mc_logprobs_bwd(z, ids, stats).shape == (0, 50)


def test_many_short_rows(mcf):
    """More rows than one launch takes."""
    import torch

    rows, V = (1 << 21) + 5, 6
    z = torch.randn(rows, V, device="cuda")
    ids = torch.randint(0, V, (rows, 1), device="cuda", dtype=torch.int32)
    logp, ent, ti, tl, stats = mcf.mc_logprobs_fwd(z, ids, top=2)
    dz = mcf.mc_logprobs_bwd(z, ids, stats)
    want = torch.log_softmax(z.double(), -1)
    assert bool(((logp[:, 0].double() - want.gather(1, ids.long())[:, 0]).abs() < 1e-5).all())
    # among millions of rows some have equal logits, whose order torch's topk leaves open
    assert torch.equal(ti.long(), torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :2])
    assert bool(((dz.double() + want.exp() - torch.nn.functional.one_hot(ids[:, 0].long(), V)).abs() < 1e-5).all())


@pytest.mark.parametrize("rows, V", [(65800, 32768), (40, 53687100)])
def test_long_tensor(mcf, rows, V):
    """Offsets past 32 bits, rows in one workgroup and in many."""
    import torch

    z = torch.full((rows, V), -30.0, device="cuda", dtype=torch.bfloat16)
    g = np.random.default_rng(6)
    at = np.sort(g.choice(V, 500, replace=False))
    v = rounded(3 * g.normal(size=500), "bfloat16")
    z[-1, torch.from_numpy(at).cuda()] = dev(v, "bfloat16")
    ids = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    ids[-1] = int(at[-1])
    logp, ent, ti, tl, stats = mcf.mc_logprobs_fwd(z, ids, top=20)
    order = np.argsort(-v, kind="stable")[:20]
    assert np.array_equal(host(ti)[-1], at[order])
    m = v.max()
    S = np.exp(v - m).sum() + (V - 500) * np.exp(-30.0 - m)
    assert np.abs(host(tl)[-1] - (v[order] - m - np.log(S))).max() < 2e-5
    dz = mcf.mc_logprobs_bwd(z, ids, stats)
    q = np.exp(v - m) / S
    want = -q
    want[-1] += 1
    got = host(dz[-1, torch.from_numpy(at).cuda()])
    assert np.all(np.abs(got - want) <= np.abs(want) * 2.0 ** -7.9 + 1e-7)
    assert abs(float(dz[0, 1])) <= 1.01 / V
