"""Plain binary64 forms of the RMS norm, of 8-bit tensors and of the log probabilities of tokens, in
numpy, and what their tests share."""
import numpy as np

# half a unit in the last place, relative to the value, and half the smallest number's distance
U = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8, "float32": 2.0 ** -24}
TINY = {"float16": 2.0 ** -25, "bfloat16": 2.0 ** -134, "float32": 2.0 ** -150}
DTYPES = ["float16", "bfloat16", "float32"]


def rounded(x, dtype):
    """binary64 values through binary32 to the format, as binary64."""
    import torch

    with np.errstate(over="ignore"):
        return torch.from_numpy(np.asarray(x, np.float64).astype(np.float32)).to(getattr(torch, dtype)).double().numpy()


def dev(x, dtype=None):
    import torch

    t = torch.from_numpy(np.ascontiguousarray(x))
    if dtype is not None:
        t = t.float().to(getattr(torch, dtype))
    return t.cuda()


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def planes_sum(planes):
    s = planes[-1]
    for p in planes[-2::-1]:
        s = s + p
    return s


def split(s, nc, dtype):
    planes = []
    for _ in range(nc):
        planes.append(rounded(s, dtype))
        with np.errstate(invalid="ignore"):
            s = np.where(np.isinf(planes[-1]), 0.0, s - planes[-1])
    return np.stack(planes)


def stream(h, x, dtype):
    """(the new planes, their sum)."""
    if x is None:
        return h, planes_sum(h)
    with np.errstate(invalid="ignore"):
        new = split(planes_sum(h) + x, h.shape[0], dtype)
    return new, planes_sum(new)


def inverse_rms(v, eps):
    return 1.0 / np.sqrt((v * v).sum(-1, keepdims=True) / v.shape[-1] + eps)


def quantize(p, r=1.0):
    """(codes, scales in binary64) of rows p; NaN scales and zero codes where the scale is not finite."""
    with np.errstate(all="ignore"):
        m = np.abs(p).max(-1, keepdims=True) if p.shape[-1] else np.zeros((*p.shape[:-1], 1))
        bad = ~np.isfinite(p).all(-1, keepdims=True)
        scale = np.where(bad, np.nan, m * r / 127.0)
        bad = ~np.isfinite(scale.astype(np.float32))
        codes = np.rint((127.0 * p) / np.where(m > 0, m, 1.0))
    return np.where(bad, 0, codes).astype(np.int8), np.where(bad, np.nan, scale)[..., 0]


def norm_bwd(v, w, dy, g, eps):
    r = inverse_rms(v, eps)
    p = dy if w is None else w * dy
    dh = r * (p - v * (r * r * (v * p).sum(-1, keepdims=True) / v.shape[-1]))
    return dh if g is None else dh + g, (dy * v * r).sum(0)


def logprobs(z, ids, T, g=None, gh=None):
    """(log probabilities, entropy, log q, gradient) of finite or -inf logits."""
    rows, V = z.shape
    with np.errstate(all="ignore"):
        top = z.max(-1, keepdims=True)
        some = np.isfinite(top)
        u = np.where(some, (z - np.where(some, top, 0.0)) / T, -np.inf)
        logq = np.where(some, u - np.log1p(np.maximum(np.exp(u).sum(-1, keepdims=True) - 1.0, 0.0)), -np.inf)
        # sure rows: the sum of all but one largest
        rest = np.where(np.arange(V) == u.argmax(-1)[:, None], 0.0, np.exp(u)).sum(-1, keepdims=True)
        logq = np.where(some, u - np.log1p(rest), logq)
        q = np.exp(logq)
        entropy = np.where(q > 0, -q * np.where(q > 0, logq, 0.0), 0.0).sum(-1)
    used = (ids >= 0) & (ids < V)
    at = np.where(used, ids, 0)
    logp = np.where(used, np.take_along_axis(logq, at, 1), 0.0)
    grad = None
    if g is not None:
        g = np.where(used, g, 0.0)
        slope = np.where(q > 0, np.where(q > 0, logq, 0.0) + entropy[:, None], 0.0)
        grad = -q * (g.sum(-1, keepdims=True) + (0.0 if gh is None else gh[:, None] * slope))
        for i in range(ids.shape[1]):
            np.add.at(grad, (np.arange(rows), at[:, i]), np.where(some[:, 0], g[:, i], 0.0))
        grad = np.where(some, grad / T, 0.0)
    return logp, entropy, logq, grad


def top(z, k):
    """The first k indices in the order (z descending, index ascending); -1 past the last above -inf."""
    order = np.argsort(-z, axis=-1, kind="stable")[:, :k]
    order = np.where(np.take_along_axis(z, order, 1) > -np.inf, order, -1)
    return np.pad(order, ((0, 0), (0, k - order.shape[1])), constant_values=-1)
