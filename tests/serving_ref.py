"""Plain definitions, in 64 bits, of the serving operators (CPU, numpy / torch
double): attention over a shared prefix and own caches, eviction by
accumulated weight, verification of drafts."""
import math

import numpy as np
import torch


def own_visible(length, n_new, i):
    return min(length, max(0, length - n_new + i + 1))


def prefix_attn(q, kp, vp, kc, vc, lens, rows, mass_in=None, scale=None):
    """rows: list of (b, i) in packed order.  Returns dict of float64 arrays:
    o [N, Hq, D], lse [Hq, N], mass (or None), and, for the error bounds,
    absv [N, Hq, D] = sum w |v| and eps_x, the largest scale * sum |q k|."""
    B, n_new, Hq, D = q.shape
    Hkv = kc.shape[2]
    G = Hq // Hkv
    scale = scale or 1.0 / math.sqrt(D)
    N = len(rows)
    o = torch.zeros(N, Hq, D, dtype=torch.float64)
    absv = torch.zeros(N, Hq, D, dtype=torch.float64)
    lse = torch.full((Hq, N), -math.inf, dtype=torch.float64)
    big = 0.0
    mass = add = None
    if mass_in is not None:
        mass = mass_in.double().clone()
        add = torch.zeros_like(mass)
        for b in range(B):
            mass[b, :, max(0, lens[b] - n_new):lens[b]] = 0
    for r, (b, i) in enumerate(rows):
        vis = own_visible(lens[b], n_new, i)
        for h in range(Hkv):
            k = torch.cat([kp[:, h], kc[b, :vis, h]]).double()
            v = torch.cat([vp[:, h], vc[b, :vis, h]]).double()
            if k.shape[0] == 0:
                continue
            hs = slice(h * G, (h + 1) * G)
            qq = q[b, i, hs].double()
            x = scale * (qq @ k.T)
            big = max(big, float((qq.abs() @ k.abs().T).max()) * scale)
            lse[hs, r] = torch.logsumexp(x, 1)
            w = torch.softmax(x, 1)
            o[r, hs] = w @ v
            absv[r, hs] = w @ v.abs()
            if add is not None:
                add[b, h, :vis] += w[:, kp.shape[0]:].sum(0)
    if mass is not None:
        mass += add
    return dict(o=o.numpy(), lse=lse.numpy(), mass=None if mass is None else mass.numpy(), absv=absv.numpy(),
                add=None if add is None else add.numpy(), big=big)


def evict(mass, slot_pos, length, n_seen, budget, recent):
    """One (sequence, KV head).  Returns (src, end): row s < end holds what row
    src[s] held."""
    end = min(length, budget)
    if length <= budget:
        return list(range(end)), end

    def worth(s):
        if slot_pos[s] >= n_seen - recent:
            return (0, 0.0, s)
        m = float(mass[s])
        return (2, 0.0, s) if math.isnan(m) else (1, -m, s)

    kept = sorted(sorted(range(length), key=worth)[:budget])
    low = set(s for s in kept if s < end)
    late = iter([s for s in kept if s >= end])
    return [s if s in low else next(late) for s in range(end)], end


def verify(draft, q, p, u, noise, draft_len):
    """float32 numpy inputs.  Returns tokens [B, m+1], n_accept [B]."""
    B, m1, V = p.shape
    m = m1 - 1
    tokens = np.full((B, m1), -1, dtype=np.int32)
    n_accept = np.zeros(B, dtype=np.int32)
    for b in range(B):
        k = max(0, min(m, int(draft_len[b])))
        a = 0
        while a < k:
            d = int(draft[b, a])
            if not 0 <= d < V or not (p[b, a, d] > 0 and u[b, a] * q[b, a, d] <= p[b, a, d]):
                break
            a += 1
        r = p[b, a] - q[b, a] if a < k else p[b, a]
        if not (r > 0).any():
            r = p[b, a]
        ok = r > 0
        score = np.where(ok, np.divide(r, noise[b], out=np.zeros_like(r), where=ok), np.float32(-1))
        tokens[b, :a] = draft[b, :a]
        tokens[b, a] = int(score.argmax()) if ok.any() else 0
        n_accept[b] = a
    return tokens, n_accept
