"""Plain definitions, in 64 bits, of the 4-bit cache, of the attention over it and of
the target's probabilities (CPU, numpy / torch double)."""
import math

import numpy as np
import torch

import serving_ref as R

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
SCALES = np.array([m * 2.0 ** -17 if e == 0 else (8 + m) * 2.0 ** (e - 18) for e in range(32) for m in range(8)])[:0xe3]


def nearest(x, grid):
    """Index of the nearest value of an ascending grid, ties to the even index."""
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo = hi - 1
    below, above = x - grid[lo], grid[hi] - x
    return np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)


def quantise(x):
    """x [..., D] bf16 -> (codes [..., D/2], scales [..., D/16]) uint8 tensors."""
    x = x.double().numpy()
    x = x.reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    bad = ~np.isfinite(x).all(-1)
    y = np.where(bad[..., None], 0.0, x)
    s = nearest(np.abs(y).max(-1) / 6, SCALES)
    value = SCALES[s][..., None]
    q = np.divide(np.abs(y), value, out=np.zeros_like(y), where=value > 0)
    code = nearest(q, MAGNITUDES)
    code = (code + 8 * ((y < 0) & (code > 0))).astype(np.uint8).reshape(*x.shape[:-2], -1)
    return (torch.from_numpy(code[..., 0::2] | (code[..., 1::2] << 4)),
            torch.from_numpy(np.where(bad, 255, s).astype(np.uint8)))


def values(codes, scales):
    """The values [..., D] held, float64; NaN for scale code 255 (and an f16's infinity and NaN above 247)."""
    c = codes.numpy()
    c = np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], -1)
    mag = np.where(c >= 8, -1.0, 1.0) * MAGNITUDES[c & 7]
    every = np.concatenate([[m * 2.0 ** -17 if e == 0 else (8 + m) * 2.0 ** (e - 18) for e in range(31) for m in range(8)],
                            [math.inf], [math.nan] * 7])
    s = np.repeat(every[scales.numpy()], 16, -1)
    with np.errstate(invalid="ignore"):
        return torch.from_numpy(mag * s)


def attn(q, k, v, lens, rows, scale=None):
    """q [B, n, Hq, D]; k, v [B, Hkv, L, D] float64 values; rows: (b, i) in packed order.
    Returns dict of float64 arrays o, lse and, for the error bounds, absv = sum w |v|,
    sumv = sum |v| over what a row sees, and big, the largest scale * sum |q k|."""
    B, n, Hq, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    scale = scale or 1.0 / math.sqrt(D)
    N = len(rows)
    o, absv, sumv = (torch.zeros(N, Hq, D, dtype=torch.float64) for _ in range(3))
    lse = torch.full((Hq, N), -math.inf, dtype=torch.float64)
    big = 0.0
    for r, (b, i) in enumerate(rows):
        vis = R.own_visible(lens[b], n, i)
        for h in range(Hkv if vis else 0):
            hs = slice(h * G, (h + 1) * G)
            kk, vv, qq = k[b, h, :vis], v[b, h, :vis], q[b, i, hs].double()
            x = scale * (qq @ kk.T)
            big = max(big, float((qq.abs() @ kk.abs().T).max()) * scale)
            lse[hs, r] = torch.logsumexp(x, 1)
            w = torch.softmax(x, 1)
            o[r, hs], absv[r, hs], sumv[r, hs] = w @ vv, w @ vv.abs(), vv.abs().sum(0)
    return dict(o=o.numpy(), lse=lse.numpy(), absv=absv.numpy(), sumv=sumv.numpy(), big=big)


def adjusted(logits, penalty=None, history=(), n_prompt=0, draft=(), bias=(), allowed=None, most=16384, real=np.float64):
    """One row's x after penalties, biases and the mask (bool [V] or None).  draft: the
    drafts before the row; bias: (token, value) pairs.  real float32: one rounding an
    operation, as the definition has it."""
    V = len(logits)
    x = np.asarray(logits, dtype=real).copy()
    if penalty is not None:
        rep, freq, pres = (real(t) for t in penalty)
        old = [t for t in [*history, *draft] if 0 <= t < V]
        made = [t for t in [*list(history)[max(n_prompt, len(history) - most):], *draft] if 0 <= t < V]
        for t in set(old):
            x[t] = x[t] / rep if x[t] > 0 else x[t] * rep
        for t in set(made):
            x[t] = x[t] - (real(made.count(t)) * freq + pres)
    total = {}
    for t, val in bias:
        if 0 <= t < V:
            total[t] = real(total.get(t, real(0)) + real(val))
    for t, val in total.items():
        x[t] = x[t] + val
    if allowed is not None:
        x = np.where(allowed, x, real(-np.inf))
    return x


def probs(x, T, allowed=None):
    """The row's probabilities from its adjusted x, float64."""
    V = len(x)
    out = np.zeros(V)
    ok = np.ones(V, bool) if allowed is None else allowed
    with np.errstate(invalid="ignore", over="ignore"):
        y = x.astype(np.float64) / T if T != 0 else x
    if np.isnan(y[ok]).any():
        out[ok] = np.nan
    elif not (y[ok] > -np.inf).any():
        pass
    elif T == 0:
        out[int(np.argmax(np.where(ok, y, -np.inf)))] = 1
    elif (y[ok] == np.inf).any():
        out[ok] = np.nan
    else:
        e = np.where(ok, np.exp(y - y[ok].max()), 0)
        out = e / e.sum()
    return out
