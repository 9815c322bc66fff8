"""The gradient of the log probabilities at the token of a row that is sure of it: g (1 - q) with 1 - q far below
binary32's step at one, to a relative bound.

A row has its largest logit d above all V - 1 others, so L = log(1 + s), s = (V - 1) exp(-d).  With e = 2^-24: s has a
relative error of (2 d + 106) e (test_gpu_logprobs.py counts it), L, 1 - q = 1 - exp(-L) and the entropy's part
B = d s / (1 + s) 8 e beside it, a sum of n upstream gradients n e relative to their magnitudes, the products and the
difference 8 e more, the format half a step."""
import numpy as np
import pytest

from lm_reference import DTYPES, TINY, U, dev, host
from test_gpu_logprobs import mcf  # noqa: F401

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [50, 1000, 5000, 9000, 40000])
@pytest.mark.parametrize("ids", [[0], [0, 0, -1], [0, 1, 0], [0] * 12, [0, 2, 2, 0, -1, 5, 0, 0, 9, 0]])
def test_sure_token(mcf, dtype, V, ids):  # noqa: F811
    """ids: 0 for the sure token, others as they are (places beside it), -1 for none."""
    g = np.random.default_rng(V + len(ids))
    depth, T = np.array([14.0, 20.0, 28.0, 40.0]), 0.5
    at = np.array([0, V - 1, V // 2, 7])  # of the sure token
    z = np.zeros((4, V)) - depth[:, None] * T
    z[np.arange(4), at] = 0.0
    ids = np.array(ids)
    places = np.where(ids == 0, at[:, None], np.where(ids < 0, -1, (at[:, None] + ids) % V)).astype(np.int32)
    up = g.uniform(0.5, 1.0, size=places.shape).astype(np.float32)
    uh = g.uniform(-1, 1, size=4).astype(np.float32)
    tz, tids = dev(z, dtype), dev(places)
    stats = mcf.mc_logprobs_fwd(tz, tids, temperature=T)[-1]
    s = (V - 1) * np.exp(-depth)
    q, B = 1.0 / (1.0 + s), depth * s / (1.0 + s)
    own = np.where(places == at[:, None], up, 0.0).astype(np.float64).sum(-1)
    others = np.where((places >= 0) & (places != at[:, None]), up, 0.0).astype(np.float64).sum(-1)
    for gh in (None, uh):
        dz = host(mcf.mc_logprobs_bwd(tz, tids, stats, dev(up), None if gh is None else dev(gh), temperature=T))
        h = 0.0 if gh is None else gh.astype(np.float64)
        parts = [own * s / (1.0 + s), -q * others, -q * h * B]
        want = sum(parts) / T
        size = sum(np.abs(p) for p in parts) / T
        bound = size * (2 * depth + 106 + 8 + len(ids) + 8) * E * 1.01
        got = dz[np.arange(4), at]
        ok = np.abs(got - want) <= bound + (np.abs(want) + bound) * U[dtype] * 1.01 + TINY[dtype] * 2
        assert ok.all(), (gh is not None, got, want, bound)
