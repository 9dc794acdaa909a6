"""logo_decode_cache4_attn over caches of which every 32 rows show in the output."""
import pytest
import torch

import cache4_marks as M
import cache4_ref as R
from test_gpu_cache4_attn import _call, _logo, _pack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("share", [1.0, 0.4])
@pytest.mark.parametrize("D,L,B,n,G,Hkv", M.SIZES)
def test_every_step_counts_once(D, L, B, n, G, Hkv, share):
    lens = M.lengths(L, B)
    x = M.caches(B, n, G * Hkv, Hkv, D, L, lens, 5)
    z = torch.rand((B, n), generator=torch.Generator().manual_seed(n)) < share
    z[0, n - 1] = True
    pos, cu, ns, rows = _pack(z)
    ref = R.attn(x[0], R.values(x[1], x[3]), R.values(x[2], x[4]), lens, rows)
    o, lse = _call(*x, lens, pos, cu, ns)
    M.check(o, lse, ref, D, M.chain(lens, z.sum(1).tolist(), G, Hkv, n, _logo().lib().logo_num_sms()))
