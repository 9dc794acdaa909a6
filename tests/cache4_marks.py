"""Caches in which every 32 rows show in the output: in each stretch of 32 rows of a
sequence and KV head one row has a V, in one channel, and logits are nearly even.  So a
step of a warp that is lost, or counted twice, changes a channel by a good part and not by
a hundredth of its rounding, as among thousands of random rows.

Bounds, from the arithmetic: the output is rounded to bf16 (2^-8) and weights to fp16
(2^-11); a logit is a sum of D exact products in fp32, scaled once (D + 8 times 2^-24 of
scale * sum |q k|), its exponential adds 2^-20.  A sum passes through the additions of a
group's stretch of 128-row units, in each two matrix steps of up to 17 terms and four
single ones, through the joins of its four warps and of the run's stretches, and a few
rescalings: `chain` counts them.  Each costs at most one ulp (2^-23) of the sum of
magnitudes, and all V are positive.
"""
import numpy as np
import torch

import cache4_ref as R

STEP = 32


def caches(B, n, Hq, Hkv, D, L, lens, seed):
    """q, codes and scales of K and V (rows past the lengths hold NaN), as entry points take them."""
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn((B, n, Hq, D), generator=g) * 0.05).to(torch.bfloat16)
    k = torch.randn((B, Hkv, L, D), generator=g)
    v = torch.zeros((B, Hkv, L, D))
    for b in range(B):
        for h in range(Hkv):
            first = torch.arange(0, lens[b], STEP)
            at = first + (torch.rand(len(first), generator=g) * torch.clamp(lens[b] - first, max=STEP)).long()
            v[b, h, at, (torch.arange(len(first)) + h) % D] = 2 + 2 * torch.rand(len(first), generator=g)
    (kc, ks), (vc, vs) = (R.quantise(x.to(torch.bfloat16)) for x in (k, v))
    for b in range(B):
        ks[b, :, lens[b]:] = vs[b, :, lens[b]:] = 255
    return q, kc, vc, ks, vs


def chain(lens, counts, G, Hkv, n, sms):
    """How many additions a sum passes through at most.  counts: selected tokens a sequence."""
    tiles = min(4, (n * G + 7) // 8)
    groups = 3 if tiles == 1 else 2  # of warps an SM, at least
    units = [max(1, (m + 127) // 128) for m in lens]
    line = sum((u + 2) * ((c * G + 8 * tiles - 1) // (8 * tiles)) * Hkv for u, c in zip(units, counts) if c)
    stretch = line // (sms * groups) + 2
    parts = min(max(units), 4 * sms)
    return 38 * stretch + parts + 32


def check(o, lse, ref, D, additions):
    x = (D + 8) * 2.0 ** -24 * ref["big"] + 2.0 ** -20
    sums = additions * 2.0 ** -23
    assert (np.abs(lse - ref["lse"]) <= x + sums + 2.0 ** -23 * np.abs(ref["lse"])).all()
    # (as V is positive the sum of magnitudes is o; weights far below a row's largest: none)
    bound = ref["o"] * (2.0 ** -8 + 2.0 ** -11 + 2 * x + 2 * sums)
    err = np.abs(o - ref["o"])
    assert (err <= 1.01 * bound).all(), float((err / np.maximum(bound, 1e-30)).max())


# D, L, B, n, G, Hkv
SIZES = [(128, 9001, 2, 1, 4, 2), (64, 20011, 1, 2, 2, 1), (128, 4097, 1, 5, 8, 1), (64, 2048, 3, 8, 8, 2),
         (128, 70001, 1, 1, 2, 1), (64, 30013, 2, 4, 16, 1), (128, 16389, 2, 5, 4, 2), (64, 8269, 3, 3, 4, 1),
         (128, 40000, 1, 3, 5, 1), (128, 3001, 40, 1, 4, 1)]


def lengths(L, B):
    return [L, L // 2 + 3, L - 31, *(max(200, L - 71 * b) for b in range(3, B))][:B]
