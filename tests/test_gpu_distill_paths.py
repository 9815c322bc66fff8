"""The distillation loss by length class: rows enough for a workgroup each, kept in registers or read
again, MC logits, and long results element by element.  Tolerances as in test_gpu_distill."""
import numpy as np
import pytest

import mx4_reference as ref
from test_gpu_distill import TINY, batch, check, mcf  # noqa: F401 (mcf: the fixture)
from test_gpu_mx4 import DTYPES, U, dev, host, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, V, k", [(256, 20001, 7), (256, 32768, 64), (256, 70001, 5), (257, 65536, 70), (256, 131071, 5)])
def test_one_workgroup_rows(mcf, dtype, rows, V, k):
    """Rows enough for a workgroup each: 512 threads, 1024 threads, rows kept and rows read again."""
    z, ids, t, g = batch(rows + V, rows, V, k, dtype)
    check(mcf, z, ids, t, g, 1.0, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [33000, 2049])
def test_one_workgroup_rows_of_mc_logits(mcf, dtype, V):
    z, ids, t, g = batch(V, 256, V, 6, dtype, 2)
    check(mcf, z, ids, t, g, 1.5, dtype)


@pytest.mark.parametrize("rows, V, dtype", [(16500, 131072, "bfloat16"), (9000, 250000, "float32")])
def test_long_results_element_by_element(mcf, rows, V, dtype):
    """More than 2^31 logits; sampled rows against binary64, every element to its own tolerance."""
    import torch

    k = 4
    g = np.random.default_rng(V)
    z = torch.empty(rows, V, device="cuda", dtype=getattr(torch, dtype))
    z[:] = dev(3.0 * g.normal(size=V), dtype)
    pick = [0, 5, rows // 2, rows - 1]
    for i in pick:
        z[i] = dev(3.0 * g.normal(size=V), dtype)
    ids = g.integers(0, V, (rows, k)).astype(np.int32)
    t = rounded(3.0 * g.normal(size=(rows, k)), dtype)
    up = g.uniform(-1, 1, rows).astype(np.float32)
    args = z, dev(ids), dev(t, dtype)
    loss, dz = ref.distill(host(z[pick]), ids[pick], t[pick], up[pick], 1.0)
    e = (4 * 100 + V / 64 + 32) * 2.0 ** -24
    p_plus_q = np.abs(dz) + 2 * np.abs(up[pick])[:, None] * np.exp(host(z[pick]) - np.log(np.exp(host(z[pick])).sum(-1, keepdims=True)))
    bound = p_plus_q * e + U[dtype] * np.abs(dz) * 1.01 + TINY[dtype]
    l1, stats = mcf.mc_distill_fwd(*args)
    d1 = mcf.mc_distill_bwd(*args, stats, dev(up))
    assert np.all(np.abs(host(d1[pick]) - dz) <= bound)
    del d1
    l2, d2 = mcf.mc_distill_fwd_bwd(*args, dev(up))
    assert np.all(np.abs(host(d2[pick]) - dz) <= bound)
    for got in (l1, l2):
        assert np.all(np.abs(host(got[pick]) - loss) <= 95 * e + 3e-5)
