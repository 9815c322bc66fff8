"""The distillation loss where finite masks, or a small temperature, put a logarithm past binary32's range
and the loss inside it.  Tolerances as in test_gpu_distill."""
import numpy as np
import pytest

import mx4_reference as ref
from test_gpu_distill import TINY, batch, mcf  # noqa: F401 (mcf: the fixture)
from test_gpu_mx4 import DTYPES, U, dev, host, rounded

pytestmark = pytest.mark.gpu

LOWEST = {"float16": -65504.0, "bfloat16": -3.3895314e38, "float32": -3.4028235e38}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 600, 9000])
@pytest.mark.parametrize("T", [0.25, 0.5, 1.0, 4.0])
def test_lowest_value_masks(mcf, dtype, V, T):
    """Logits masked by the type's lowest value where the teacher has an entry: the loss is p T |lowest|
    to within rounding, a finite number wherever binary32 holds it, at every temperature.  Of the size
    of a loss without masks: |z| < 27, |t| < 15, log V + 10 < 20."""
    rows, k = 6, 8
    z, ids, t, g = batch(V, rows, V, k, dtype)
    z = z[0]
    low = rounded(np.array([LOWEST[dtype]]), dtype)[0]
    z[0, ids[0, 0]] = low
    z[1, ids[1, :3]] = low
    z[2, 1:] = low
    z[3, :] = low
    z[4, ids[4]] = low
    args = dev(z, dtype), dev(ids), dev(t, dtype)
    with np.errstate(over="ignore"):
        loss, dz = ref.distill(z, ids, t, g, T)
        held = np.abs(loss) <= 3.4028235e38
    l1, stats = mcf.mc_distill_fwd(*args, temperature=T)
    l2, d2 = mcf.mc_distill_fwd_bwd(*args, dev(g), temperature=T)
    e = (4 * 100 + V / 64 + 36) * 2.0 ** -24
    for got in (host(l1), host(l2)):
        assert np.all(np.isinf(got[~held]))
        assert np.all(np.abs(got - loss)[held] <= (e * np.abs(loss) + e * (60 * T + 30 * T * T))[held]), (got, loss)
    for got in (host(d2), host(mcf.mc_distill_bwd(*args, stats, dev(g), temperature=T))):
        bound = (np.abs(dz) + 2 * np.abs(g)[:, None] * T) * e + U[dtype] * np.abs(dz) * 1.01 + TINY[dtype]
        assert np.all(np.abs(got - dz) <= bound)


def test_small_temperature(mcf):
    """(z - m) / T passes binary32's range, T^2 times it does not: the loss is T (m - z) nearly."""
    T = 1e-30
    z = np.array([[0.0, -1e10, 3.0], [2.0, 1.0, -1e20]], np.float32)
    ids, t = np.array([[1], [2]], np.int32), np.array([[0.5], [0.5]], np.float32)
    loss, _ = mcf.mc_distill_fwd(dev(z), dev(ids), dev(t), temperature=T)
    want = T * (z.max(-1).astype(np.float64) - z[[0, 1], [1, 2]])
    assert np.all(np.abs(host(loss) - want) <= 1e-5 * want)
