"""The pairs of pieces that dW of a binary32 MXFP4 layer leaves out, and what that costs.

A number is split into three bfloat16 pieces, each what is left rounded to nearest.  The second is at
most 2^-8 of the number's power of two, the third 2^-17, so the pairs (1, 2) and (2, 1) are at most
2^-25 of |x||dY| each, the pair (2, 2) 2^-34: together just above 2^-24, half a unit in the last place
of the largest binary32 number at or above the product."""
import numpy as np
import pytest

LEFT_OUT = 2.0 ** -24 + 2.0 ** -34
WORST = np.float32(1.0038986206)  # 1 + 2^-8 - 2^-17: the largest pieces there are


def pieces(x):
    import torch

    out, r = [], torch.from_numpy(np.atleast_1d(np.asarray(x, np.float32)))
    for _ in range(3):
        out.append(r.bfloat16())
        r = r - out[-1].float()
    assert not r.any()
    return [p.double().numpy() for p in out]


def test_bound():
    g = np.random.default_rng(0)
    x = np.concatenate([[WORST], g.uniform(1, 2, 200000), np.nextafter(np.float32(1), np.float32(2)) + 2.0 ** -8 * g.uniform(0, 1, 200000)])
    p = pieces(x)
    x = np.asarray(x, np.float32).astype(np.float64)
    power = np.exp2(np.floor(np.log2(x)))
    assert np.all(np.abs(p[1]) <= 2.0 ** -8 * power) and np.all(np.abs(p[2]) <= 2.0 ** -17 * power)
    out = 2 * np.abs(p[1] * p[2]) + p[2] ** 2
    assert np.all(out <= LEFT_OUT * x * x)
    assert abs(p[1][0] * p[2][0]) > 2.0 ** -25.1 * x[0] ** 2 and out[0] > 2.0 ** -24.1 * x[0] ** 2


@pytest.mark.gpu
def test_worst_numbers():
    """Six kept products in one binary32 accumulator and the result's rounding add at most 7 2^-24 of the sum
    of magnitudes, at most 1 + 2^-6 of |x||dY|."""
    import torch

    import paper_2207_08867_amd as mcf

    x, dY = torch.full((1, 70), float(WORST), device="cuda"), torch.full((1, 40), float(WORST), device="cuda")
    W = mcf.mc_mx4_quantize(torch.zeros(40, 70, device="cuda"))
    _, dW, _ = mcf.mc_mx4_linear_bwd(x, W, dY, dx=False, db=False)
    exact = float(WORST) * float(WORST)
    assert float((dW.double() - exact).abs().max()) <= (LEFT_OUT + 7 * 2.0 ** -24 * (1 + 2.0 ** -6)) * exact
