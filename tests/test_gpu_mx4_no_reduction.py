"""Products over nothing, of results whose smallest tiles are 2^24 workgroups, 2^32 threads: zeros."""
import pytest

pytestmark = pytest.mark.gpu

M, N = 2 ** 20, 2 ** 16  # 2^36 binary16 results


@pytest.fixture()
def result():
    import torch

    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 140 * 2 ** 30:
        pytest.skip("needs 128 GiB")
    yield torch.empty(M, N, dtype=torch.float16, device="cuda")
    torch.cuda.empty_cache()


def none(rows):
    import torch

    return (torch.empty(1, rows, 0, dtype=torch.uint8, device="cuda"), torch.empty(1, 0, rows, 4, dtype=torch.uint8, device="cuda"))


def all_zero(t):
    return not any(bool(part.any()) for part in t.view(64, -1))


def test_product(result):
    import paper_2207_08867_amd as mcf

    result.fill_(1.0)
    mcf.mc_mx4_matmul(none(M), none(N), 0, dtype=result.dtype, out=result)
    assert all_zero(result)


def test_layer(result):
    import torch

    import paper_2207_08867_amd as mcf

    result.fill_(1.0)
    b = torch.randn(N, device="cuda").half()
    mcf.mc_mx4_linear_fwd(torch.empty(M, 0, dtype=torch.float16, device="cuda"), none(N), b, out=result)
    assert all(torch.equal(part, b.expand_as(part)) for part in result.view(1024, -1, N))
