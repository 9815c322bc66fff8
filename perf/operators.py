"""Cases of the operators on microscaled 4-bit tensors and of the distillation loss.

Two families, which a low-precision training step or a server uses one after the other:

* MXFP4 tensors: blocks of 32 elements along a row, each element an E2M1 number (0, 0.5, 1,
  1.5, 2, 3, 4, 6 and their negatives), the block's scale a power of two (E8M0).  A tensor
  has nc components, each the MXFP4 rounding of what the components before it leave.
  Quantisation and reading back, the product of two such tensors, the linear layer of a plain
  input with such a weight, and that layer's gradients.
* Distillation from a teacher's top logits: the divergence of the student's softmax over the
  whole vocabulary from the teacher's softmax over its k kept logits, and its gradient.

``run`` computes a case in elementary torch operations in 32 bits, or through the library
where ``own`` is true; ``exact`` computes it in 64 bits by other steps.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}
BLOCK = 32
DEVICE = "cuda"


def listed():
    return [
        # One token's activations written as 4-bit numbers and read back: the latency of two small calls.
        dict(name="quant_token", kind="quant", dtype="f16", nc_in=1, nc=1, rows=1, n=4096),
        # A layer's binary16 two-component master weight, odd in both sizes, into two 4-bit components.
        dict(name="quant_weight", kind="quant", dtype="f16", nc_in=2, nc=2, rows=4099, n=4097),
        # A decoding step of eight sequences with quantised activations.
        dict(name="mm_decode", kind="matmul", dtype="bf16", nc_a=1, nc_b=1, M=8, N=4096, K=4096),
        # Ragged sizes, a two-component weight, results in binary32.
        dict(name="mm_odd", kind="matmul", dtype="f32", nc_a=1, nc_b=2, M=777, N=1023, K=1025),
        # The benchmark's matrix size in 4-bit operands: the largest product.
        dict(name="mm_large", kind="matmul", dtype="bf16", nc_a=1, nc_b=1, M=8192, N=8192, K=8192),
        # One token through a layer: the weight is read once, and latency counts.
        dict(name="lin_token", kind="linear", dtype="f16", nc=1, batch=1, inp=4096, out=4096, bias=True),
        # A prompt of 4096 tokens through the same layer.
        dict(name="lin_prompt", kind="linear", dtype="bf16", nc=1, batch=4096, inp=4096, out=4096, bias=False),
        # A small binary32 layer on an odd batch, two components.
        dict(name="lin_odd", kind="linear", dtype="f32", nc=2, batch=100, inp=784, out=99, bias=True),
        # The gradients of that small layer: a latency-bound training step.
        dict(name="bwd_odd", kind="backward", dtype="f32", nc=2, batch=100, inp=784, out=99),
        # The gradients of the benchmark's binary16 layer.
        dict(name="bwd_layer", kind="backward", dtype="f16", nc=1, batch=4096, inp=1024, out=1024),
        # Few rows over a long odd vocabulary, loss and gradient in two calls.
        dict(name="distill_few", kind="distill", dtype="f32", nc=1, rows=4, vocab=131071, k=32, temperature=2.0,
             fused=False),
        # A training batch's rows, loss and gradient in one call.
        dict(name="distill_batch", kind="distill", dtype="bf16", nc=1, rows=4096, vocab=32768, k=64, temperature=1.0,
             fused=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quant", "matmul", "linear", "linear", "backward", "distill"])
    dtype = rng.choice(["f16", "bf16", "f32"])
    if kind == "quant":
        rows, n = _log(rng, 1, 8192), _log(rng, 1, 8192)
        return dict(kind=kind, dtype=dtype, nc_in=rng.choice([1, 1, 2]) if dtype == "f16" else 1,
                    nc=rng.choice([1, 1, 2, 3]), rows=rows, n=n)
    if kind == "matmul":
        return dict(kind=kind, dtype=dtype, nc_a=rng.choice([1, 1, 1, 2]), nc_b=rng.choice([1, 1, 2]),
                    M=_log(rng, 1, 4096), N=_log(rng, 16, 8192), K=_log(rng, 32, 8192))
    if kind == "linear":
        batch = _log(rng, 1, 64) if rng.random() < 0.5 else _log(rng, 64, 4096)
        return dict(kind=kind, dtype=dtype, nc=rng.choice([1, 1, 1, 2, 3]), batch=batch, inp=_log(rng, 32, 8192),
                    out=_log(rng, 16, 8192), bias=rng.choice([False, True]))
    if kind == "backward":
        return dict(kind=kind, dtype=dtype, nc=rng.choice([1, 1, 2]), batch=_log(rng, 1, 4096), inp=_log(rng, 32, 4096),
                    out=_log(rng, 16, 4096))
    vocab = _log(rng, 100, 131072)
    rows = _log(rng, 1, max(2, min(8192, (1 << 27) // vocab)))
    return dict(kind=kind, dtype=dtype, nc=rng.choice([1, 1, 2]) if dtype == "f16" else 1, rows=rows, vocab=vocab,
                k=min(vocab, _log(rng, 1, 128)), temperature=rng.choice([1.0, 1.5, 2.0, 4.0]),
                fused=rng.choice([False, True]))


# --- the plain forms -------------------------------------------------------------------

def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _quantize(x, nc):
    """x: binary32 (rows, n) -> codes (nc, rows, 64 G), scales (nc, G, rows, 4), G groups of
    four blocks covering a row, zeros past its end.  The scale of a block is 2^(floor(log2 of
    its largest magnitude) - 2), at least 2^-127; the elements are rounded to nearest, ties
    to even, at most 6."""
    rows, n = x.shape
    groups = (n + 4 * BLOCK - 1) // (4 * BLOCK)
    r = torch.nn.functional.pad(x, (0, groups * 4 * BLOCK - n)).reshape(rows, groups * 4, BLOCK)
    codes, scales = [], []
    for _ in range(nc):
        _, e = torch.frexp(r.abs().amax(-1, keepdim=True))
        top = torch.where(r.abs().amax(-1, keepdim=True) > 0, e - 3, torch.full_like(e, -127)).clamp(min=-127)
        y = r * _power(-top)
        a = y.abs()
        code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int()
                + (a >= 3.5).int() + (a > 5.0).int()) + 8 * (y < 0).int()
        pairs = code.reshape(*code.shape[:-1], BLOCK // 2, 2)
        codes.append((pairs[..., 0] + 16 * pairs[..., 1]).to(torch.uint8).reshape(rows, 64 * groups))
        scales.append((top + 127).to(torch.uint8).reshape(rows, groups, 4).transpose(0, 1).contiguous())
        r = r - _values(code) * _power(top)
    return torch.stack(codes), torch.stack(scales)


def _power(e):
    """2^e in binary32, -127 <= e <= 127, from its bits (2^-127 is subnormal)."""
    return torch.where(e > -127, (e.int() + 127) << 23, torch.full_like(e, 1 << 22, dtype=torch.int32)).view(torch.float32)


def _values(code):
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    return table[(code & 7).long()] * (1.0 - 2.0 * (code >> 3).float())


def _dequantize(codes, scales, n):
    """Binary32 values (rows, n): the sum of the components, the smallest first."""
    total = None
    for c, s in zip(reversed(codes.unbind(0)), reversed(scales.unbind(0))):
        c, s = c.int(), s.transpose(0, 1).int()
        v = _values(torch.stack((c & 15, c >> 4), -1).flatten(-2).reshape(*s.shape, BLOCK))
        v = (v * _power(s - 127).unsqueeze(-1)).flatten(1)[:, :n]
        total = v if total is None else total + v
    return total


def _distill_teacher(ids, t, temperature, dtype):
    """The teacher's probabilities over its kept entries, 0 at the unused ones."""
    used = ids >= 0
    u = torch.where(used, t.to(dtype) / temperature, torch.full_like(t, -math.inf, dtype=dtype))
    top = u.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    w = torch.exp(u - top)
    total = w.sum(-1, keepdim=True)
    p = torch.where(total > 0, w / total, torch.zeros_like(w))
    return p, torch.where(p > 0, u - top - torch.log(total), torch.zeros_like(p))


def _distill(z, ids, t, g, temperature):
    """loss = T^2 sum_i p_i (log p_i - log q_i); gradient g T (q - p), 0 for a row with no
    teacher entry."""
    p, logp = _distill_teacher(ids, t, temperature, torch.float32)
    logits = z.float().sum(0) / temperature
    logits = logits - logits.amax(-1, keepdim=True)
    e = torch.exp(logits)
    total = e.sum(-1, keepdim=True)
    where = ids.clamp(min=0).long()
    logq = torch.gather(logits, 1, where) - torch.log(total)
    loss = temperature ** 2 * torch.where(p > 0, p * (logp - logq), torch.zeros_like(p)).sum(-1)
    d = e / total * (p.sum(-1, keepdim=True) > 0)
    d.scatter_add_(1, where, -p)
    return loss, d * (temperature * g).unsqueeze(-1)


# --- inputs ----------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE)


def _split(x, nc, dtype):
    """nc components of `dtype` by successive rounding."""
    parts = []
    for _ in range(nc):
        parts.append(x.to(dtype))
        x = x - parts[-1].float()
    return torch.stack(parts)


def _weight(gen, out, inp, nc):
    """A layer's weight: rows of unequal size, a few large columns."""
    w = _normal(gen, out, inp) * (0.5 + torch.rand(out, 1, generator=gen, device=DEVICE)) / math.sqrt(inp)
    w = w * torch.where(torch.rand(1, inp, generator=gen, device=DEVICE) < 0.01, 8.0, 1.0)
    return _quantize(w, nc)


def prepare(case, seed):
    gen = _generator(seed)
    dtype = DTYPES[case["dtype"]]
    state = {"case": case}
    kind = case["kind"]
    if kind == "quant":
        x = _normal(gen, case["rows"], case["n"])
        x = x * torch.where(torch.rand(case["rows"], case["n"], generator=gen, device=DEVICE) < 0.002, 20.0, 1.0)
        state["x"] = _split(x, case["nc_in"], dtype)
    elif kind == "matmul":
        state["a"] = _quantize(_normal(gen, case["M"], case["K"]), case["nc_a"])
        state["b"] = _weight(gen, case["N"], case["K"], case["nc_b"])
    elif kind in ("linear", "backward"):
        state["x"] = _normal(gen, case["batch"], case["inp"]).to(dtype)
        state["w"] = _weight(gen, case["out"], case["inp"], case["nc"])
        if kind == "linear":
            state["bias"] = (0.1 * _normal(gen, case["out"])).to(dtype) if case["bias"] else None
        else:
            state["dy"] = (_normal(gen, case["batch"], case["out"]) / math.sqrt(case["out"])).to(dtype)
    else:
        rows, vocab, k = case["rows"], case["vocab"], case["k"]
        z = 2.0 * _normal(gen, rows, vocab)
        # the end of the vocabulary is not in use: its logits are masked
        masked = vocab // 64
        if masked:
            z[:, vocab - masked:] = -math.inf
        teacher = z + 0.7 * _normal(gen, rows, vocab)
        top, ids = torch.topk(teacher, min(k, vocab - masked), dim=-1)
        top = torch.nn.functional.pad(top, (0, k - top.shape[1]), value=-math.inf)
        ids = torch.nn.functional.pad(ids, (0, k - ids.shape[1]), value=-1)
        # a teacher keeps up to k logits a row; a few rows (prompt positions) keep none
        kept = torch.randint(1, k + 1, (rows, 1), generator=gen, device=DEVICE)
        kept = torch.where(torch.rand(rows, 1, generator=gen, device=DEVICE) < 0.05, torch.zeros_like(kept), kept)
        unused = torch.arange(k, device=DEVICE).unsqueeze(0) >= kept
        state["ids"] = torch.where(unused, torch.full_like(ids, -1), ids).to(torch.int32)
        state["t"] = torch.where(unused, torch.full_like(top, -math.inf), top).to(dtype)
        if case["nc"] > 1:
            z = torch.where(z == -math.inf, torch.full_like(z, -30000.0), z)
        state["z"] = _split(z, case["nc"], dtype)
        state["g"] = (0.5 + torch.rand(rows, generator=gen, device=DEVICE)) / rows
    return state


# --- one pass --------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(state):
    case = state["case"]
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    if kind == "quant":
        # the planes' sum, the smallest first
        x = state["x"].float()
        total = x[-1]
        for c in range(x.shape[0] - 2, -1, -1):
            total = x[c] + total
        codes, scales = _quantize(total, case["nc"])
        return _dequantize(codes, scales, case["n"]).to(dtype)
    if kind == "matmul":
        a, b = _dequantize(*state["a"], case["K"]), _dequantize(*state["b"], case["K"])
        return (a @ b.t()).to(dtype)
    if kind == "linear":
        y = state["x"].float() @ _dequantize(*state["w"], case["inp"]).t()
        return (y if state["bias"] is None else y + state["bias"].float()).to(dtype)
    if kind == "backward":
        w, x, dy = _dequantize(*state["w"], case["inp"]), state["x"].float(), state["dy"].float()
        return (dy @ w).to(dtype), (dy.t() @ x).to(dtype), dy.sum(0).to(dtype)
    loss, dz = _distill(state["z"], state["ids"], state["t"], state["g"], case["temperature"])
    return loss, dz.to(dtype)


def _run_own(state):
    import paper_2207_08867_amd as mcf

    case = state["case"]
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    if kind == "quant":
        codes, scales = mcf.mc_mx4_quantize(state["x"], nc=case["nc"], x_mc=True)
        return mcf.mc_mx4_dequantize(codes, scales, case["n"], dtype=dtype)
    if kind == "matmul":
        return mcf.mc_mx4_matmul(state["a"], state["b"], case["K"], dtype=dtype)
    if kind == "linear":
        return mcf.mc_mx4_linear_fwd(state["x"], state["w"], state["bias"])
    if kind == "backward":
        return mcf.mc_mx4_linear_bwd(state["x"], state["w"], state["dy"])
    z, ids, t, g, temperature = state["z"], state["ids"], state["t"], state["g"], case["temperature"]
    if case["fused"]:
        return mcf.mc_distill_fwd_bwd(z, ids, t, g, temperature=temperature)
    loss, stats = mcf.mc_distill_fwd(z, ids, t, temperature=temperature)
    return loss, mcf.mc_distill_bwd(z, ids, t, stats, g, temperature=temperature)


# --- what a pass cannot do without -----------------------------------------------------

def work(case):
    kind, size = case["kind"], SIZE[case["dtype"]]
    if kind == "quant":
        elems = case["rows"] * case["n"]
        packed = 17 * case["nc"] * case["rows"] * _blocks(case["n"])
        return {"bytes": (case["nc_in"] + 1) * size * elems + 2 * packed, "flops": 4 * case["nc"] * elems}
    if kind == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": 17 * _blocks(K) * (case["nc_a"] * M + case["nc_b"] * N) + size * M * N,
                "flops": 2 * case["nc_a"] * case["nc_b"] * M * N * K}
    if kind in ("linear", "backward"):
        T, I, O = case["batch"], case["inp"], case["out"]
        weight = 17 * case["nc"] * O * _blocks(I)
        if kind == "linear":
            return {"bytes": size * (T * I + T * O + (O if case["bias"] else 0)) + weight,
                    "flops": 2 * case["nc"] * T * I * O}
        return {"bytes": size * (2 * T * I + T * O + O * I + O) + weight, "flops": 2 * (case["nc"] + 1) * T * I * O}
    R, V, k = case["rows"], case["vocab"], case["k"]
    return {"bytes": R * V * size * (case["nc"] + 1) + R * k * (4 + size) + 8 * R, "flops": 6 * R * V}


# --- the definitions in 64 bits --------------------------------------------------------

def _decode64(codes, scales, n):
    """Components' sum in binary64 from the bits: E2M1 with exponent bias 1, E8M0 with bias 127."""
    nibble = torch.empty(*codes.shape, 2, dtype=torch.int64, device=codes.device)
    nibble[..., 0] = codes.long() % 16
    nibble[..., 1] = codes.long() // 16
    nibble = nibble.flatten(-2)
    expo, mant = (nibble % 8) // 2, (nibble % 2).double()
    mag = torch.where(expo == 0, 0.5 * mant, (1.0 + 0.5 * mant) * 2.0 ** (expo - 1).double())
    mag = torch.where(nibble >= 8, -mag, mag)
    unit = (2.0 ** (scales.permute(0, 2, 1, 3).double() - 127.0)).flatten(2).repeat_interleave(BLOCK, -1)
    return (mag * unit).sum(0)[:, :n]


def _round64(x, nc):
    """The sum of nc successive MXFP4 roundings of binary64 values, in binary64."""
    n = x.shape[-1]
    r = torch.zeros(*x.shape[:-1], _blocks(n) * BLOCK, dtype=torch.float64, device=x.device)
    r[..., :n] = x
    r = r.unflatten(-1, (-1, BLOCK))
    total = torch.zeros_like(r)
    for _ in range(nc):
        peak = r.abs().amax(-1, keepdim=True)
        unit = 2.0 ** (torch.floor(torch.log2(peak.clamp(min=2.0 ** -126))) - 2.0).clamp(min=-127.0)
        # the spacing of the magnitudes is half a unit below 2, one below 4, two from there on
        step = unit * torch.where(r.abs() < 2 * unit, 0.5, torch.where(r.abs() < 4 * unit, 1.0, 2.0)).double()
        q = torch.minimum(torch.round(r.abs() / step) * step, 6 * unit) * torch.sign(r)
        total = total + q
        r = r - q
    return total.flatten(-2)[..., :n]


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "quant":
        return _round64(state["x"].double().sum(0), case["nc"])
    if kind == "matmul":
        return torch.matmul(_decode64(*state["a"], case["K"]), _decode64(*state["b"], case["K"]).transpose(0, 1))
    if kind == "linear":
        y = torch.matmul(state["x"].double(), _decode64(*state["w"], case["inp"]).transpose(0, 1))
        return y if state["bias"] is None else y + state["bias"].double()
    if kind == "backward":
        w, x, dy = _decode64(*state["w"], case["inp"]), state["x"].double(), state["dy"].double()
        return torch.matmul(dy, w), torch.matmul(dy.transpose(0, 1), x), dy.sum(0)
    T = case["temperature"]
    losses, grads = [], []
    step = max(1, (1 << 25) // case["vocab"])
    for a in range(0, case["rows"], step):
        z, ids, t = state["z"][:, a:a + step].double().sum(0), state["ids"][a:a + step], state["t"][a:a + step].double()
        logq = torch.log_softmax(z / T, -1)
        kept = ids >= 0
        p = torch.zeros_like(t)
        some = kept.any(-1)
        p[some] = torch.softmax(torch.where(kept, t / T, torch.full_like(t, -math.inf))[some], -1)
        at = torch.where(kept, ids, torch.zeros_like(ids)).long()
        picked = torch.where(p > 0, torch.gather(logq, 1, at), torch.zeros_like(p))
        losses.append(T * T * (torch.special.xlogy(p, p) - p * picked).sum(-1))
        full = torch.zeros_like(z).scatter_add(1, at, p)
        grads.append(T * state["g"][a:a + step].double().unsqueeze(-1)
                     * (torch.exp(logq) * some.unsqueeze(-1) - full))
    return torch.cat(losses), torch.cat(grads)
