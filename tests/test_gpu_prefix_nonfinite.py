"""logo_decode_prefix_attn with infinities and NaN: in what a row sees, or in its
query, they show in its output.  """
import pytest
import torch

import test_gpu_prefix_attn as T

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def _call(q, kp, vp, kc, vc, lens, pos, cu, ns, mass):
    from paper_2608_29539_gb300 import logo as Lg
    d = lambda t: t.cuda()  # noqa: E731
    P, m = kp.shape[0], None if mass is None else d(mass)
    out = Lg.logo_decode_prefix_attn(d(q), d(kp) if P else None, d(vp) if P else None, d(kc), d(vc),
                                     torch.tensor(lens, dtype=torch.int32, device="cuda"), d(pos), d(cu), d(ns),
                                     mass_in=m, mass_out=None if m is None else torch.zeros_like(m))
    torch.cuda.synchronize()
    assert Lg.logo_get_device_status() == 0
    return out


@pytest.mark.parametrize("P,wide", [(0, False), (300, False), (None, True)])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_a_query_that_is_not_a_number_shows(P, wide, bad):
    """The row of a NaN query has a NaN output and lse; other rows are as they were."""
    import test_gpu_prefix_wide as W
    B, n, Hkv, G, D, L = 9, 2, 1, 32, 128, 40
    if wide:
        P = W._prefix_for(B * n * G, Hkv, 9)
    q, kp, vp, kc, vc = T._inputs(B, n, G * Hkv, Hkv, D, P, L, 6)
    lens = [n + 3 * b for b in range(B)]
    pos, cu, ns, rows = T._pack(torch.ones(B, n, dtype=torch.bool))
    clean = _call(q, kp, vp, kc, vc, lens, pos, cu, ns, None)
    q[3, 1, 5, ::3] = bad  # (infinities of both signs: the logits are NaN)
    q[3, 1, 5, 1::3] = -bad
    o, lse, _ = _call(q, kp, vp, kc, vc, lens, pos, cu, ns, None)
    hit = torch.zeros(B * n, G * Hkv, dtype=torch.bool)
    hit[rows.index((3, 1)), 5] = True
    assert bool(torch.isnan(o.cpu()[hit]).all()) and bool(torch.isnan(lse.cpu().T[hit]).all())
    assert torch.equal(o.cpu()[~hit], clean[0].cpu()[~hit]) and torch.equal(lse.cpu().T[~hit], clean[1].cpu().T[~hit])


def test_a_key_that_is_not_a_number_reaches_every_weight_of_its_rows():
    """Rows over a finite prefix and one NaN key of their own: their softmax is not a
    number anywhere, so neither are the weights."""
    B, n, Hq, Hkv, D, P, L = 2, 1, 4, 2, 64, 10, 8
    q, kp, vp, kc, vc = T._inputs(B, n, Hq, Hkv, D, P, L, 9)
    kc[0, 0] = NAN
    lens = [1, 5]
    pos, cu, ns, rows = T._pack(torch.ones(B, n, dtype=torch.bool))
    o, lse, m = _call(q, kp, vp, kc, vc, lens, pos, cu, ns, torch.zeros(B, Hkv, L))
    assert bool(torch.isnan(o[0]).all()) and bool(torch.isnan(lse[:, 0]).all()) and bool(torch.isnan(m[0, :, :1]).all())
    assert bool(torch.isfinite(o[1]).all()) and bool(torch.isfinite(m[1, :, :5]).all())
