"""The log probabilities and their gradient at the ends of the temperatures that the calls take, with logits of the
temperature's size, which binary32 and bfloat16 hold: against the plain binary64 form, to the bounds of the ordinary
temperatures (test_gpu_logprobs.py).  What those count holds here as well: a difference of scaled logits is rounded once, the
factor's two terms hold log2(e) / T to 2^-48, and what scaling rounds away is below 2^-126 of a quotient."""
import numpy as np
import pytest

from lm_reference import dev, host, rounded
from test_gpu_logprobs import check, mcf  # noqa: F401

pytestmark = pytest.mark.gpu

LARGEST = {"bfloat16": (2 - 2.0 ** -7) * 2.0 ** 127, "float32": (2 - 2.0 ** -23) * 2.0 ** 127}


def logits(seed, rows, V, T, dtype):
    """Rows of logits of T's size within the format's range, the last one with both ends of it and -inf."""
    g = np.random.default_rng(seed)
    z = T * 3.0 * g.normal(size=(rows, V))
    z = rounded(np.clip(z, -LARGEST[dtype], LARGEST[dtype]), dtype)
    if V > 2:
        z[-1, 0], z[-1, 1], z[-1, 2] = LARGEST[dtype], -LARGEST[dtype], -np.inf
    return z, g


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T", [2.0 ** 63, 2.0 ** 64, 2.0 ** 65, 1e30, 1e33, 1e36, 1e37, 1e38, 3.4028e38])
@pytest.mark.parametrize("rows, V, given, k", [(2, 3, 1, 3), (3, 300, 3, 9), (2, 1000, 12, 5), (2, 9000, 2, 20),
                                               (3, 40001, 1, 20)])
def test_large(mcf, dtype, T, rows, V, given, k):  # noqa: F811
    both(mcf, dtype, T, rows, V, given, k)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T", [2.0 ** 64, 1e38])
def test_many_long_rows(mcf, dtype, T):  # noqa: F811
    both(mcf, dtype, T, 260, 33001, 9, 0)


def both(mcf, dtype, T, rows, V, given, k):  # noqa: F811
    T = float(np.float32(T))
    z, g = logits(rows + V, rows, V, T, dtype)
    ids = g.integers(0, V, size=(rows, given))
    # gradients of T's size too, so that dz, which has 1 / T, is not lost in the format; sums of them hold in binary32
    size = min(T, 1e36)
    up = (size * g.uniform(-1, 1, size=(rows, given))).astype(np.float32)
    uh = (0.1 * size * g.uniform(-1, 1, size=rows)).astype(np.float32)
    check(mcf, z, ids, k, T, dtype, up, uh)
    check(mcf, z, ids, 0, T, dtype, up, None)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_flat(mcf, dtype):  # noqa: F811
    """Ordinary logits at a temperature that makes all tokens alike, masks of -inf apart."""
    g = np.random.default_rng(1)
    z = rounded(3.0 * g.normal(size=(3, 5000)), dtype)
    z[1, 100:] = -np.inf
    ids = g.integers(0, 5000, size=(3, 2))
    for T in (1e19, 1e20, 1e30, 1e38):
        _, ent, _, top_logp, _, _ = check(mcf, z, ids, 4, float(np.float32(T)), dtype)
        for r, n in enumerate((5000, 100, 5000)):
            assert abs(host(ent)[r] - np.log(n)) < 1e-5 and np.all(np.abs(host(top_logp)[r] + np.log(n)) < 1e-5)


@pytest.mark.parametrize("T", [2.0 ** -100, 1e-30, 1e-20])
@pytest.mark.parametrize("V", [3, 1000, 9000])
def test_small(mcf, T, V):  # noqa: F811
    """Logits of a small temperature's size; gradients of it, since dz has 1 / T."""
    T = float(np.float32(T))
    z, g = logits(V, 2, V, T, "float32")
    z[-1, :2] = T
    ids = g.integers(0, V, size=(2, 3))
    check(mcf, z, ids, 3, T, "float32", (T * g.uniform(-1, 1, size=(2, 3))).astype(np.float32),
          (T * g.uniform(-1, 1, size=2)).astype(np.float32))


def test_most_likely_token(mcf):  # noqa: F811
    """Logits 0, -T and -2 T: the same numbers at every temperature."""
    want = -np.log1p(np.exp(-1.0) + np.exp(-2.0))
    for T in (1.0, 1e6, 2.0 ** 64, 1e30, 1e36, 1e37, 1.6e38):
        T = float(np.float32(T))
        z = dev(np.array([[0.0, -T, -2.0 * T]]), "float32")
        logp = mcf.mc_logprobs_fwd(z, dev(np.zeros((1, 1), np.int32)), temperature=T)[0]
        assert abs(host(logp)[0, 0] - want) < 2e-6, T
