"""logo_decode_prefix_attn with infinities and NaN: in the keys and values of
drafts that a row does not see they change nothing; in what a row sees, or in its
query, they show in its output.  Bounds as in test_gpu_prefix_attn."""
import numpy as np
import pytest
import torch

import serving_ref as R
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


@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("D,G,n,P", [(128, 4, 3, 0), (128, 2, 8, 70), (64, 1, 5, 0), (64, 16, 2, 200), (128, 9, 7, 0)])
def test_unseen_drafts_change_nothing(D, G, n, P, where):
    """Sequence b's draft c[b] and all after it hold infinities and NaN; the rows
    before it are compared, of up to 63 (row, head) pairs a KV head."""
    Hkv, L = 2, 300
    lens = [n, 31 + n, 128, 129, 160, 257, 300]
    B = len(lens)
    q, kp, vp, kc, vc = T._inputs(B, n, G * Hkv, Hkv, D, P, L, 40 + n)
    mass = torch.rand((B, Hkv, L), generator=torch.Generator().manual_seed(1))
    pos, cu, ns, rows = T._pack(torch.ones(B, n, dtype=torch.bool))
    first = [1 + b % (n - 1) for b in range(B)]
    ref = R.prefix_attn(q, kp, vp, kc, vc, lens, rows, mass)
    bad = kc if where == "k" else vc
    for b in range(B):
        for j in range(first[b], n):
            row = bad[b, lens[b] - n + j]
            if (b + j) % 3 == 0:
                row[:] = NAN
            elif (b + j) % 3 == 1:
                row[:, ::5] = INF
                row[:, 1::7] = -INF
            else:
                row[:, (11 * b + j) % D] = -INF
    o, lse, m = _call(q, kp, vp, kc, vc, lens, pos, cu, ns, mass)
    keep = [r for r, (b, i) in enumerate(rows) if i < first[b]]
    T._check(o[keep], lse[:, keep], None, {k: ref[k][:, keep] if k == "lse" else ref[k][keep] for k in ("o", "lse", "absv")}
             | {"big": ref["big"]}, keep, D, lens)
    for r, (b, i) in enumerate(rows):
        for h in range(G * Hkv):
            got = o[r, h].float().cpu()
            if where == "v":  # a seen row's infinity or NaN is in its column, and only there
                seen = torch.stack([vc[b, lens[b] - n + j, h // G] for j in range(i + 1)]).float()
                assert torch.equal(~torch.isfinite(got), ~torch.isfinite(seen).all(0)), (r, h)
    if where == "v":  # weights do not depend on V
        for b, length in enumerate(lens):
            want, add = ref["mass"][b, :, :length], ref["add"][b, :, :length]
            err = np.abs(m[b, :, :length].cpu().numpy().astype(np.float64) - want)
            assert (err <= (2 * 2.0 ** -24 * D * ref["big"] + 2.0 ** -18) * add + 2.0 ** -22 * want).all()


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
