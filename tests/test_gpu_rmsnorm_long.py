"""The gradients of a norm whose rows are longer than one launch of the sum over workgroups takes (2^27 elements;
a single launch would come to 2^32 threads at 2^28)."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [(1 << 27) + 64, (1 << 28) + 77])
def test_gradients_of_long_rows(n):
    """Every element: dh and dw are rounded from binary64 (dw through one binary32 sum a workgroup), so within
    half a step of bfloat16 and, relative, 2^-22."""
    import torch

    import paper_2207_08867_amd as mcf

    gen = torch.Generator(device="cuda").manual_seed(n)
    h, dy = (torch.randn(1, n, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = (1 + 0.1 * torch.randn(n, generator=gen, device="cuda")).to(torch.bfloat16)
    dh, dw = mcf.mc_rmsnorm_bwd(h, w, dy, eps=1e-5)
    step = 1 << 24
    pieces = [slice(lo, min(lo + step, n)) for lo in range(0, n, step)]
    square = sum(h[0, p].double().square().sum() for p in pieces)
    inner = sum((h[0, p].double() * w[p].double() * dy[0, p].double()).sum() for p in pieces)
    r = (square / n + 1e-5) ** -0.5
    for p in pieces:
        v, d, u = h[0, p].double(), dy[0, p].double(), w[p].double()
        want = r * (u * d - v * (r * r * inner / n))
        assert bool(((dh[0, p].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -22) + 1e-12).all()), p
        want = d * v * r
        assert bool(((dw[p].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -22) + 1e-12).all()), p
