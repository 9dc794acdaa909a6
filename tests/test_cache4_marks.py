"""That the check of marked caches sees what it is for (CPU): mistakes planted in the
definition's sums, 32 rows left out or counted twice, are found wherever they are."""
import numpy as np
import pytest
import torch

import cache4_marks as M
import cache4_ref as R


def _sums(q, k, v, keys):
    """Weights' sums, and of weights times V, over a choice of keys."""
    w = torch.exp(q @ k[keys].T)
    return w.sum(1), w @ v[keys]


@pytest.mark.parametrize("D,L,B,n,G,Hkv", M.SIZES)
def test_planted_mistakes_are_found(D, L, B, n, G, Hkv):
    lens = M.lengths(L, B)
    q, kc, vc, ks, vs = M.caches(B, n, G * Hkv, Hkv, D, L, lens, 5)
    steps = M.chain(lens, [n] * B, G, Hkv, n, 148)
    b, i, h = B - 1, n - 1, Hkv - 1
    k, v = (R.values(c[b:b + 1, h:h + 1], s[b:b + 1, h:h + 1])[0, 0, :lens[b]] for c, s in ((kc, ks), (vc, vs)))
    qq = q[b, i, h * G:(h + 1) * G].double() / D ** 0.5
    l, o = _sums(qq, k, v, slice(0, lens[b]))
    one = dict(o=(o / l[:, None]).numpy(), lse=torch.log(l).numpy(), big=float((qq.abs() @ k.abs().T).max()))

    def passes(l, o):
        try:
            M.check((o / l[:, None]).to(torch.bfloat16).double().numpy(), torch.log(l).float().double().numpy(), one, D, steps)
        except AssertionError:
            return False
        return True

    assert passes(l, o)
    last = (lens[b] - 1) // M.STEP
    for j in sorted({0, 1, last // 3, last // 2, last - 1, *np.random.default_rng(L).integers(0, last, 20).tolist()}):
        dl, do = _sums(qq, k, v, slice(j * M.STEP, (j + 1) * M.STEP))
        assert not passes(l - dl, o - do) and not passes(l + dl, o + do)  # a step lost, or twice
        assert not passes(l, o - do) and not passes(l - dl, o)            # its V, or its weights, alone
