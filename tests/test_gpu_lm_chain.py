"""The norm, the 8-bit products and the log probabilities as they are used: one after the other, on another
stream, in a captured graph, with outputs and workspaces of exactly the stated sizes, and with the
distillation loss that reads the alternatives."""
import numpy as np
import pytest

import lm_reference as ref
from lm_reference import DTYPES, dev, host, rounded
from test_gpu_mx4_bounds import Room

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mcf():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2207_08867_amd as m

    m.lib()
    return m


def model(mcf, hidden, vocab, dtype):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(1)
    dt = getattr(torch, dtype)
    w = torch.randn(vocab, hidden, generator=gen, device="cuda") / hidden ** 0.5 * 3.0
    return (1 + 0.1 * torch.randn(hidden, generator=gen, device="cuda")).to(dt), mcf.mc_int8_quantize(w.to(dt))


def score(mcf, h, x, norm, W, ids, n, top):
    (codes, scales), h = mcf.mc_rmsnorm_int8(h, norm, x=x)
    z = mcf.mc_int8_matmul((codes, scales), W, n, dtype=h.dtype)
    return (h, z, *mcf.mc_logprobs_fwd(z, ids, top=top))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, hidden, vocab", [(1, 256, 9000), (5, 100, 333), (70, 512, 2000)])
def test_chain(mcf, dtype, rows, hidden, vocab):
    """Hidden states to log probabilities, against the plain forms of the same steps; a row has the
    same bits alone and among others."""
    import torch

    norm, W = model(mcf, hidden, vocab, dtype)
    g = np.random.default_rng(rows)
    h, x = (rounded(g.normal(size=(rows, hidden)), dtype) for _ in range(2))
    ids = g.integers(0, vocab, size=(rows, 2)).astype(np.int32)
    out = score(mcf, dev(h, dtype), dev(x, dtype), norm, W, dev(ids), hidden, 8)
    new, v = ref.stream(h[None], x, dtype)
    assert np.array_equal(host(out[0]), new[0])
    c, s = ref.quantize(v * host(norm), ref.inverse_rms(v, 1e-6))
    z = (c.astype(np.float64) @ host(W[0])[:, :hidden].astype(np.float64).T) * s[:, None] * host(W[1])
    assert np.all(np.abs(host(out[1]) - z) <= np.abs(z) * (2.0 ** -22 + {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}.get(dtype, 0)) + 2.0 ** -24)
    logp, entropy, logq, _ = ref.logprobs(host(out[1]), ids, 1.0)
    assert np.abs(host(out[2]) - logp).max() < 1e-4 and np.abs(host(out[3]) - entropy).max() < 1e-4
    assert np.array_equal(host(out[4]), ref.top(host(out[1]), 8))
    alone = score(mcf, dev(h[-1:], dtype), dev(x[-1:], dtype), norm, W, dev(ids[-1:]), hidden, 8)
    for a, b in zip(alone[:2], out[:2]):
        assert torch.equal(a[0], b[-1])


def test_alternatives_teach(mcf):
    """The alternatives are the entries that the distillation loss reads; the loss of the logits
    they were taken from is the divergence that the kept ones leave."""
    import torch

    z = 3.0 * torch.randn(6, 3000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    _, _, ids, logp, _ = mcf.mc_logprobs_fwd(z, torch.empty(6, 0, dtype=torch.int32, device="cuda"), top=32)
    loss, _ = mcf.mc_distill_fwd_bwd(z, ids, logp)
    q = torch.softmax(z.double(), -1)
    kept = q.gather(1, ids.long())
    p = kept / kept.sum(-1, keepdim=True)
    want = (p * (p.log() - kept.log())).sum(-1)
    assert torch.allclose(loss.double(), want, atol=1e-5)


def test_training_step(mcf):
    """Norm, 4-bit layer, log probabilities and the way back, against binary64 autograd on the numbers
    the weight stands for."""
    import torch

    gen = torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn(40, 256, generator=gen, device="cuda")
    w = 1 + 0.2 * torch.randn(256, generator=gen, device="cuda")
    W = mcf.mc_mx4_quantize(torch.randn(500, 256, generator=gen, device="cuda") / 16, nc=2)
    ids = torch.randint(0, 500, (40, 1), generator=gen, device="cuda", dtype=torch.int32)
    g, gh = torch.randn(40, 1, generator=gen, device="cuda"), torch.randn(40, generator=gen, device="cuda")
    y, _ = mcf.mc_rmsnorm_fwd(h, w)
    z = mcf.mc_mx4_linear_fwd(y, W)
    logp, ent, _, _, stats = mcf.mc_logprobs_fwd(z, ids)
    dz = mcf.mc_logprobs_bwd(z, ids, stats, g, gh)
    dy, _, _ = mcf.mc_mx4_linear_bwd(y, W, dz, dw=False, db=False)
    dh, dw = mcf.mc_rmsnorm_bwd(h, w, dy)
    hd, wd = h.double().cpu().requires_grad_(), w.double().cpu().requires_grad_()
    Wd = mcf.mc_mx4_dequantize(*W, 256, dtype=torch.float32).double().cpu()
    yd = hd * torch.rsqrt(hd.square().mean(-1, keepdim=True) + 1e-6) * wd
    lq = torch.log_softmax(yd @ Wd.t(), -1)
    loss = (g.double().cpu() * lq.gather(1, ids.long().cpu())).sum() + (gh.double().cpu() * -(lq.exp() * lq).sum(-1)).sum()
    loss.backward()
    # products of 500 and 256 terms in binary32: 2^-24 times a thousand, of sums of magnitudes below ten
    assert torch.allclose(dh.double().cpu(), hd.grad, atol=2e-4) and torch.allclose(dw.double().cpu(), wd.grad, atol=2e-3)


def test_streams(mcf):
    """Work on another stream than the default one, two calls at once with their own workspaces."""
    import torch

    norm, W = model(mcf, 256, 9000, "float16")
    g = np.random.default_rng(0)
    h, x = (dev(rounded(g.normal(size=(40, 256)), "float16"), "float16") for _ in range(2))
    ids = dev(g.integers(0, 9000, size=(40, 2)).astype(np.int32))
    want = score(mcf, h, x, norm, W, ids, 256, 8)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(score(mcf, h, x, norm, W, ids, 256, 8))
    torch.cuda.synchronize()
    for out in outs:
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_graph(mcf):
    """The chain and the gradients captured once and replayed on new inputs, with eager work in between."""
    import torch

    norm, W = model(mcf, 512, 9000, "bfloat16")
    h, x = torch.empty(300, 512, device="cuda", dtype=torch.bfloat16), torch.empty(300, 512, device="cuda", dtype=torch.bfloat16)
    ids = torch.zeros(300, 1, dtype=torch.int32, device="cuda")

    def step():
        out = score(mcf, h, x, norm, W, ids, 512, 8)
        y = mcf.mc_int8_linear_fwd(x, W)
        dz = mcf.mc_logprobs_bwd(out[1], ids, out[-1])
        return (*out, y, dz, *mcf.mc_rmsnorm_bwd(out[0], norm, x))

    def fill(i):
        gen = torch.Generator(device="cuda").manual_seed(i)
        h.copy_(torch.randn(300, 512, generator=gen, device="cuda"))
        x.copy_(torch.randn(300, 512, generator=gen, device="cuda"))
        ids.copy_(torch.randint(0, 9000, (300, 1), generator=gen, device="cuda"))

    fill(0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(1, 5):
        fill(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, n, O", [(1, 1, 1), (1, 129, 33), (3, 1000, 70), (33, 127, 99), (129, 513, 257), (600, 40, 31),
                                        (200, 8200, 64), (2, 16400, 40)])
def test_bounds(mcf, dtype, rows, n, O):
    """Outputs at odd addresses and workspaces between marked bytes: all of the outputs is written, nothing
    outside."""
    import torch

    dt = getattr(torch, dtype)
    odd = 16 + dt.itemsize
    h, x = (torch.randn(2, rows, n, device="cuda").to(dt) for _ in range(2))
    x = x[0].contiguous()
    w = torch.randn(n, device="cuda").to(dt)
    P = (n + 127) // 128 * 128
    rooms = dict(h=Room((2, rows, n), dt, odd), y=Room((rows, n), dt, odd), c=Room((rows, P), torch.int8),
                 s=Room((rows,), torch.float32, 20), back=Room((rows, n), dt, odd))
    y, new = mcf.mc_rmsnorm_fwd(h, w, x=x, h_mc=True, h_out=rooms["h"].tensor, out=rooms["y"].tensor)
    want = mcf.mc_rmsnorm_fwd(h, w, x=x, h_mc=True)
    assert torch.equal(y, want[0]) and torch.equal(new, want[1])
    pair, _ = mcf.mc_rmsnorm_int8(h, w, x=x, h_mc=True, out=(rooms["c"].tensor, rooms["s"].tensor))
    for a, b in zip(pair, mcf.mc_rmsnorm_int8(h, w, x=x, h_mc=True)[0]):
        assert torch.equal(a, b)
    mcf.mc_int8_dequantize(*pair, n, dtype=dt, out=rooms["back"].tensor)
    dy = torch.randn(rows, n, device="cuda").to(dt)
    want = mcf.mc_rmsnorm_bwd(h, w, dy, h_mc=True)
    rooms["ws"] = Room((mcf.mc_rmsnorm_bwd_workspace(dt, rows, n),), torch.uint8)
    rooms["dh"], rooms["dw"] = Room((rows, n), dt, odd), Room((n,), dt, odd)
    code = {"float16": mcf.MCF_F16, "bfloat16": mcf.MCF_BF16, "float32": mcf.MCF_F32}[dtype]
    stream = torch.cuda.current_stream().cuda_stream
    assert mcf.lib().mc_rmsnorm_bwd(code, 2, rows, n, h.data_ptr(), w.data_ptr(), dy.data_ptr(), None, 1e-6,
                                    rooms["dh"].tensor.data_ptr(), rooms["dw"].tensor.data_ptr(),
                                    rooms["ws"].tensor.data_ptr(), rooms["ws"].bytes, stream) == 0
    assert torch.equal(rooms["dh"].tensor, want[0]) and torch.equal(rooms["dw"].tensor, want[1])
    W = mcf.mc_int8_quantize(torch.randn(O, n, device="cuda"))
    rooms["wp"], rooms["p"] = Room((mcf.mc_int8_matmul_workspace(dt, rows, O, n),), torch.uint8), Room((rows, O), dt, odd)
    mcf.mc_int8_matmul(pair, W, n, dtype=dt, out=rooms["p"].tensor, workspace=rooms["wp"].tensor)
    assert torch.equal(rooms["p"].tensor, mcf.mc_int8_matmul(pair, W, n, dtype=dt))
    rooms["wl"], rooms["l"] = Room((mcf.mc_int8_linear_fwd_workspace(dt, rows, n, O),), torch.uint8), Room((rows, O), dt, odd)
    mcf.mc_int8_linear_fwd(x, W, out=rooms["l"].tensor, workspace=rooms["wl"].tensor)
    assert torch.equal(rooms["l"].tensor, mcf.mc_int8_linear_fwd(x, W))
    for r in rooms.values():
        r.check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, V", [(1, 1), (3, 7), (2, 8193), (5, 1025), (4, 20001), (256, 8195), (256, 16390), (256, 33001)])
def test_bounds_logprobs(mcf, dtype, rows, V):
    import torch

    dt, top = getattr(torch, dtype), 9
    z = torch.randn(rows, V, device="cuda").to(dt)
    ids = torch.randint(0, V, (rows, 3), device="cuda", dtype=torch.int32)
    f32, i32 = torch.float32, torch.int32
    outs = [Room((rows, 3), f32, 20), Room((rows,), f32, 20), Room((rows, top), i32, 20), Room((rows, top), f32, 20),
            Room((rows, 3), f32, 20)]
    ws, dz = Room((mcf.mc_logprobs_workspace(rows, V, top),), torch.uint8), Room((rows, V), dt, 16 + dt.itemsize)
    code = {"float16": mcf.MCF_F16, "bfloat16": mcf.MCF_BF16, "float32": mcf.MCF_F32}[dtype]
    stream = torch.cuda.current_stream().cuda_stream
    want = mcf.mc_logprobs_fwd(z, ids, top=top)
    assert mcf.lib().mc_logprobs_fwd(code, 1, rows, V, 3, top, z.data_ptr(), ids.data_ptr(), 1.0, ws.tensor.data_ptr(),
                                     ws.bytes, *(o.tensor.data_ptr() for o in outs), stream) == 0
    for o, v in zip(outs, want):
        assert torch.equal(o.tensor, v)
    mcf.mc_logprobs_bwd(z, ids, want[-1], out=dz.tensor)
    assert torch.equal(dz.tensor, mcf.mc_logprobs_bwd(z, ids, want[-1]))
    for r in (*outs, ws, dz):
        r.check()
