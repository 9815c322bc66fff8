"""The gradient of the distillation loss at large temperatures, with logits and entries of the temperature's size,
which binary32 and bfloat16 hold.  Tolerances as in test_gpu_distill.  The loss itself has T^2, which passes binary32's range at 2^64."""
import numpy as np
import pytest

import mx4_reference as ref
from test_gpu_distill import TINY, mcf  # noqa: F401 (mcf: the fixture)
from test_gpu_mx4 import U, dev, host, rounded

pytestmark = pytest.mark.gpu

LARGEST = {"bfloat16": (2 - 2.0 ** -7) * 2.0 ** 127, "float32": (2 - 2.0 ** -23) * 2.0 ** 127}


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T", [2.0 ** 63, 2.0 ** 64, 2.0 ** 65, 1e31, 1e36, 1e38])
@pytest.mark.parametrize("rows, V, k", [(3, 7, 2), (4, 300, 8), (3, 5000, 70), (2, 9000, 5), (256, 9000, 5), (2, 40000, 20)])
def test_large(mcf, dtype, T, rows, V, k):  # noqa: F811
    T = float(np.float32(T))
    g = np.random.default_rng(V + k)
    most = LARGEST[dtype]
    z, t = (rounded(np.clip(3.0 * T * g.normal(size=s), -most, most), dtype) for s in ((rows, V), (rows, k)))
    z[0, :3] = most, -most, -np.inf
    t[-1, 0], t[-1, 1] = most, -most
    ids = np.stack([g.permutation(V)[:k] for _ in range(rows)]).astype(np.int32)
    up = (g.uniform(-1, 1, rows) / T).astype(np.float32)
    args = dev(z, dtype), dev(ids), dev(t, dtype)
    with np.errstate(over="ignore", invalid="ignore"):
        _, dz = ref.distill(z, ids, t, up, T)
        m = z.max(-1, keepdims=True)
        w = np.exp((z - m) / T)
    s = w.sum(-1, keepdims=True)
    e = (4 * 100 + V / 64 + 32) * 2.0 ** -24
    _, stats = mcf.mc_distill_fwd(*args, temperature=T)
    assert np.array_equal(host(stats)[:, 0], m[:, 0]) and np.all(np.abs(host(stats)[:, 1] - s[:, 0]) <= s[:, 0] * e)
    bound = (np.abs(dz) + 2 * np.abs(up)[:, None].astype(np.float64) * T * w / s) * e
    bound += U[dtype] * np.abs(dz) * 1.01 + TINY[dtype]
    for got in (mcf.mc_distill_fwd_bwd(*args, dev(up), temperature=T)[1],
                mcf.mc_distill_bwd(*args, stats, dev(up), temperature=T)):
        assert np.all(np.abs(host(got) - dz) <= bound)
