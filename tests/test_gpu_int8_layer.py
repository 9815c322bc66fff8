"""The 8-bit layer of one and two rows on both sides of the rule that quantises them in the product's launch or ahead of
it: the numbers of the quantisation and the product either way, a row's the same alone and beside another."""
import numpy as np
import pytest

from lm_reference import dev, rounded
from test_gpu_int8 import mcf, operand, pack  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("inp, out", [(100, 4096), (100, 4097), (130, 8192), (130, 8193), (4095, 8200), (4096, 8193),
                                      (4096, 32768), (4100, 32769), (16385, 40), (32768, 60), (32769, 60), (33, 131072)])
def test_few_rows(mcf, dtype, inp, out):  # noqa: F811
    import torch

    g = np.random.default_rng(inp + out)
    W = pack(*operand(g, out, inp))
    x = dev(rounded(g.normal(size=(2, inp)), dtype), dtype)
    b = dev(rounded(g.normal(size=out), dtype), dtype)
    want = mcf.mc_int8_matmul(mcf.mc_int8_quantize(x), W, inp, b, dtype=x.dtype)
    assert torch.equal(mcf.mc_int8_linear_fwd(x, W, b), want)
    for r in range(2):
        assert torch.equal(mcf.mc_int8_linear_fwd(x[r:r + 1].contiguous(), W, b), want[r:r + 1])
