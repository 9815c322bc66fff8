"""Plain numpy forms, in binary64, of the MXFP4 tensors and of the distillation loss, written
from their definitions in include/mcf.h.  They share no code with the library."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def groups(n):
    return -(-n // 128)


def round_e2m1(y):
    """|y| to the index of the nearest E2M1 magnitude, ties to the even index, at most 7."""
    a = np.minimum(np.abs(y), 6.0)
    hi = np.searchsorted(MAGNITUDES, a).clip(0, 7)  # first magnitude >= a
    lo = np.maximum(hi - 1, 0)
    dlo, dhi = a - MAGNITUDES[lo], MAGNITUDES[hi] - a
    pick_lo = (dlo < dhi) | ((dlo == dhi) & (lo % 2 == 0))
    return np.where((MAGNITUDES[hi] == a) | ~pick_lo, hi, lo)


def quantize(planes, nc):
    """planes: (nc_in, rows, n), exact in binary64 -> codes (nc, rows, 64 G), scales (nc, G, rows, 4)."""
    v = planes[-1].astype(np.float64)
    with np.errstate(invalid="ignore"):
        for p in planes[-2::-1]:
            v = v + p.astype(np.float64)
    rows, n = v.shape
    G = groups(n)
    r = np.zeros((rows, G * 128))
    r[:, :n] = v
    r = r.reshape(rows, G * 4, 32)
    bad = ~np.isfinite(r).all(-1)
    r[bad] = 0.0
    codes = np.zeros((nc, rows, 64 * G), np.uint8)
    scales = np.zeros((nc, G, rows, 4), np.uint8)
    for c in range(nc):
        peak = np.abs(r).max(-1)
        X = np.where(peak > 0, np.frexp(peak)[1] - 3, -127)
        X = np.clip(X, -127, 127)
        y = np.ldexp(r, -X[..., None])
        idx = round_e2m1(y)
        code = idx + 8 * np.signbit(y)
        code[bad] = 0
        byte = np.where(bad, 255, X + 127)
        pairs = code.reshape(rows, G * 64, 2)
        codes[c] = pairs[..., 0] + 16 * pairs[..., 1]
        scales[c] = byte.reshape(rows, G, 4).transpose(1, 0, 2)
        q = np.ldexp(MAGNITUDES[idx] * np.where(np.signbit(y), -1.0, 1.0), X[..., None])
        r = np.where(bad[..., None], 0.0, r - q)
    return codes, scales


def dequantize(codes, scales, n):
    """(rows, n) in binary64: the components' numbers, (nc, rows, n)."""
    nc, rows, _ = codes.shape
    nib = np.stack((codes & 15, codes >> 4), -1).reshape(nc, rows, -1, 32)
    s = scales.transpose(0, 2, 1, 3).reshape(nc, rows, -1, 1).astype(np.int64)
    v = np.ldexp(MAGNITUDES[nib & 7] * np.where(nib & 8, -1.0, 1.0), s - 127)
    v = np.where(s == 255, np.nan, v)
    return v.reshape(nc, rows, -1)[:, :, :n]


def distill(z, ids, t, g, T):
    """(loss, dz, p, logp, logq at the entries) in binary64; z (rows, vocab)."""
    rows, V = z.shape
    loss = np.zeros(rows)
    dz = np.zeros((rows, V))
    for r in range(rows):
        use = [i for i in range(ids.shape[1]) if 0 <= ids[r, i] < V]
        tt = t[r, use].astype(np.float64) / T
        if not use or np.all(tt == -np.inf):
            continue
        with np.errstate(divide="ignore", invalid="ignore"):
            e = np.exp(tt - tt.max())
            p = e / e.sum()
            logp = tt - tt.max() - np.log(e.sum())
            zz = z[r].astype(np.float64) / T
            m = zz.max()
            if m == -np.inf:
                q, log_s = np.zeros(V), None
            else:
                w = np.exp(zz - m)
                q, log_s = w / w.sum(), np.log(w.sum())
        grad = q.copy()
        for pi, lp, j in zip(p, logp, ids[r, use]):
            if pi > 0:
                lq = -np.inf if z[r, j] == -np.inf else (zz[j] - m) - log_s
                loss[r] += pi * (lp - lq)
                grad[j] -= pi
            elif np.isnan(pi):
                loss[r] = np.nan
                grad[:] = np.nan
        loss[r] *= T * T
        dz[r] = g[r] * T * grad
    return loss, dz
