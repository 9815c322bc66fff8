"""Outputs and workspaces of exactly the stated sizes between marked bytes: the calls write all of the
outputs and nothing outside."""
import pytest

pytestmark = pytest.mark.gpu

MARK = 0xA5
EDGE = 4096


@pytest.fixture(scope="module")
def mcf():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2207_08867_amd as m

    m.lib()
    return m


class Room:
    """A tensor of marked bytes with EDGE marked bytes on both sides."""

    def __init__(self, shape, dtype, align=16):
        import torch

        self.bytes = torch.empty(0, dtype=dtype).element_size()
        for s in shape:
            self.bytes *= s
        self.raw = torch.full((2 * EDGE + self.bytes + align,), MARK, dtype=torch.uint8, device="cuda")
        self.at = EDGE + (-(self.raw.data_ptr() + EDGE)) % 16 + (align % 16)
        self.tensor = self.raw[self.at:self.at + self.bytes].view(dtype).view(shape)

    def check(self):
        assert bool((self.raw[:self.at] == MARK).all()) and bool((self.raw[self.at + self.bytes:] == MARK).all())


def rooms(*specs):
    return [Room(*s) for s in specs]


DTYPES = ["float16", "bfloat16", "float32"]
SIZES = [(1, 1, 1), (1, 33, 1000), (3, 50, 70), (16, 17, 129), (17, 40, 300), (33, 99, 127), (65, 130, 31), (129, 257, 513), (300, 8, 2050),
         (1031, 1029, 260)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, O, I", SIZES)
def test_layer_and_product(mcf, dtype, T, O, I):
    import torch

    dt = getattr(torch, dtype)
    x, w, dY = torch.randn(T, I, device="cuda").to(dt), torch.randn(O, I, device="cuda").to(dt), torch.randn(T, O, device="cuda").to(dt)
    G, nc = (I + 127) // 128, 2
    q = rooms(((nc, O, 64 * G), torch.uint8), ((nc, G, O, 4), torch.uint8))
    W = mcf.mc_mx4_quantize(w, nc=nc, out=tuple(r.tensor for r in q))
    A = mcf.mc_mx4_quantize(x)
    assert all(torch.equal(a, b) for a, b in zip(W, mcf.mc_mx4_quantize(w, nc=nc)))
    back = Room((O, I), dt)
    mcf.mc_mx4_dequantize(*W, I, dtype=dt, out=back.tensor)
    ws = Room((mcf.mc_mx4_linear_fwd_workspace(dt, nc, T, I, O),), torch.uint8)
    y = Room((T, O), dt, 16 + dt.itemsize)
    mcf.mc_mx4_linear_fwd(x, W, out=y.tensor, workspace=ws.tensor)
    assert torch.equal(y.tensor, mcf.mc_mx4_linear_fwd(x, W))
    wp = Room((mcf.mc_mx4_matmul_workspace(dt, T, O, I, 1, nc),), torch.uint8)
    p = Room((T, O), dt, 16 + dt.itemsize)
    mcf.mc_mx4_matmul(A, W, I, dtype=dt, out=p.tensor, workspace=wp.tensor)
    assert torch.equal(p.tensor, mcf.mc_mx4_matmul(A, W, I, dtype=dt))
    wb = Room((mcf.mc_mx4_linear_bwd_workspace(dt, nc, T, I, O),), torch.uint8)
    grads = rooms(((T, I), dt, 16 + dt.itemsize), ((O, I), dt, 16 + dt.itemsize), ((O,), dt, 16 + dt.itemsize))
    codes, scales = W
    stream = torch.cuda.current_stream().cuda_stream
    code = {"float16": mcf.MCF_F16, "bfloat16": mcf.MCF_BF16, "float32": mcf.MCF_F32}[dtype]
    assert mcf.lib().mc_mx4_linear_bwd(code, nc, T, I, O, x.data_ptr(), codes.data_ptr(), scales.data_ptr(), dY.data_ptr(),
                                       *(g.tensor.data_ptr() for g in grads), wb.tensor.data_ptr(), wb.bytes, stream) == 0
    for g, want in zip(grads, mcf.mc_mx4_linear_bwd(x, W, dY)):
        assert torch.equal(g.tensor, want)
    for r in (*q, back, ws, y, wp, p, wb, *grads):
        r.check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, V", [(1, 1), (3, 7), (2, 8193), (5, 1025), (4, 20001), (256, 8195), (256, 16390), (256, 33001), (256, 131071)])
def test_distillation(mcf, dtype, rows, V):
    import torch

    dt, k = getattr(torch, dtype), min(V, 5)
    z, t = torch.randn(rows, V, device="cuda").to(dt), torch.randn(rows, k, device="cuda").to(dt)
    ids = torch.stack([torch.arange(k, device="cuda") * (V // k) for _ in range(rows)]).int()
    ws = Room((mcf.mc_distill_workspace(rows, V),), torch.uint8)
    dz = Room((rows, V), dt, 16 + dt.itemsize)
    loss, out = mcf.mc_distill_fwd_bwd(z, ids, t, out=dz.tensor, workspace=ws.tensor)
    want = mcf.mc_distill_fwd_bwd(z, ids, t)
    assert torch.equal(loss, want[0]) and torch.equal(out, want[1])
    d2 = Room((rows, V), dt, 16 + dt.itemsize)
    _, stats = mcf.mc_distill_fwd(z, ids, t, workspace=ws.tensor)
    mcf.mc_distill_bwd(z, ids, t, stats, out=d2.tensor)
    assert bool(torch.isfinite(d2.tensor.float()).all())
    for r in (ws, dz, d2):
        r.check()
