"""logo_decode_prefix_attn against the 64-bit definition.  Cache rows past a
sequence's length hold NaN; output rows past the selected count hold
sentinels.

Error bounds, from the formats alone (bf16 has 8 significant bits: rounding x
moves it by at most 2^-8 |x|; A = sum w |v|; E = 2^-24 D max scale sum |q k|,
the fp32 accumulation error of a logit):
  o    2^-8 |o| (its rounding to bf16) + 2^-8 A (weights rounded to bf16)
       + (2 E + 2^-16) A (logits, fp32 sums)
  lse  E + 2^-20 + 2^-22 |lse|
  mass (2 E + 2^-18) of what was added + 2^-22 of the whole
"""
import math

import numpy as np
import pytest
import torch

import serving_ref as R

pytestmark = pytest.mark.gpu


def _inputs(B, n, Hq, Hkv, D, P, L, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    t = lambda *s: (torch.randn(s, generator=g) * std).to(torch.bfloat16)  # noqa: E731
    return t(B, n, Hq, D), t(P, Hkv, D), t(P, Hkv, D), t(B, L, Hkv, D), t(B, L, Hkv, D)


def _pack(z):
    """z [B, n] bool -> pos, cu_q, n_sel as logo_select leaves them, rows."""
    B, n = z.shape
    rows = [(b, i) for b in range(B) for i in range(n) if z[b, i]]
    pos = torch.full((B * n,), -1, dtype=torch.int32)
    pos[:len(rows)] = torch.tensor([i for _, i in rows], dtype=torch.int32)
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = z.sum(1).cumsum(0)
    return pos, cu, cu[-1:].clone(), rows


def _check(got_o, got_lse, got_mass, ref, rows, D, lens):
    N = len(rows)
    E = 2.0 ** -24 * D * ref["big"]
    o = got_o[:N].float().cpu().numpy().astype(np.float64)
    bound = 2.0 ** -8 * (np.abs(ref["o"]) + ref["absv"]) + (2 * E + 2.0 ** -16) * ref["absv"]
    assert np.isfinite(o).all()
    assert (np.abs(o - ref["o"]) <= bound).all(), float((np.abs(o - ref["o"]) - bound).max())
    lse = got_lse[:, :N].cpu().numpy().astype(np.float64)
    seen = np.isfinite(ref["lse"])
    assert (lse[~seen] == -math.inf).all()
    tol = E + 2.0 ** -20 + 2.0 ** -22 * np.abs(ref["lse"][seen])
    assert (np.abs(lse[seen] - ref["lse"][seen]) <= tol).all(), float(np.abs(lse[seen] - ref["lse"][seen]).max())
    if got_mass is not None:
        m = got_mass.cpu().numpy().astype(np.float64)
        for b, n in enumerate(lens):
            err = np.abs(m[b, :, :n] - ref["mass"][b, :, :n])
            tol = (2 * E + 2.0 ** -18) * ref["add"][b, :, :n] + 2.0 ** -22 * np.abs(ref["mass"][b, :, :n])
            assert (err <= tol).all(), (b, float((err - tol).max()))


def _run(B, n, Hq, Hkv, D, P, L, lens, z, seed=0, mass=True, scale=0.0, std=1.0):
    from paper_2608_29539_gb300 import logo as Lg
    q, kp, vp, kc, vc = _inputs(B, n, Hq, Hkv, D, P, L, seed, std)
    pos, cu, ns, rows = _pack(z)
    N = len(rows)
    for b, m in enumerate(lens):
        kc[b, m:] = float("nan")
        vc[b, m:] = float("nan")
    mass_in = torch.rand((B, Hkv, L), generator=torch.Generator().manual_seed(seed + 1)) if mass else None
    ref = R.prefix_attn(q, kp, vp, kc, vc, lens, rows, mass_in, scale or None)
    d = lambda t: t.cuda()  # noqa: E731
    o = torch.full((B * n, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((Hq, B * n), 7.0, device="cuda")
    m_out = torch.full((B, Hkv, L), 7.0, device="cuda") if mass else None
    args = (d(q), d(kp) if P else None, d(vp) if P else None, d(kc), d(vc),
            torch.tensor(lens, dtype=torch.int32, device="cuda"), d(pos), d(cu), d(ns))
    Lg.logo_decode_prefix_attn(*args, scale=scale, mass_in=d(mass_in) if mass else None, mass_out=m_out, o_c=o,
                               lse_c=lse)
    torch.cuda.synchronize()
    assert Lg.logo_get_device_status() == 0
    _check(o, lse, m_out, ref, rows, D, lens)
    assert bool((o[N:] == 7.0).all()) and bool((lse[:, N:] == 7.0).all())
    if mass:
        for b, m in enumerate(lens):
            assert bool((m_out[b, :, m:] == 7.0).all())
    # the same call again, in place, gives the same bits
    o2, lse2 = torch.full_like(o, 7.0), torch.full_like(lse, 7.0)
    m2 = d(mass_in) if mass else None
    Lg.logo_decode_prefix_attn(*args, scale=scale, mass_in=m2, o_c=o2, lse_c=lse2)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    if mass:
        for b, m in enumerate(lens):
            assert torch.equal(m_out[b, :, :m], m2[b, :, :m])
    return o, lse, m_out


def _z(B, n, share, seed):
    z = torch.rand((B, n), generator=torch.Generator().manual_seed(seed + 77)) < share
    z[-1, -1] = True
    return z


@pytest.mark.parametrize("P", [0, 1, 127, 128, 129, 500])
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (64, 4, 4)])
def test_one_new_token_prefix_lengths(P, D, Hq, Hkv):
    lens = [1, 127, 128, 129, 300, 64]
    _run(6, 1, Hq, Hkv, D, P, 301, lens, _z(6, 1, 0.7, P), seed=P + D)


@pytest.mark.parametrize("G,Hkv", [(1, 3), (3, 2), (5, 1), (8, 2), (16, 1), (40, 1)])
@pytest.mark.parametrize("n", [1, 2, 5])
def test_head_groups_and_drafts(G, Hkv, n):
    lens = [n, 130, 257, n + 1, 200]
    _run(5, n, G * Hkv, Hkv, 128, 150, 260, lens, _z(5, n, 0.8, G), seed=G * 10 + n)


@pytest.mark.parametrize("D", [64, 128])
def test_rows_without_a_key_and_short_caches(D):
    """No prefix: a sequence of length 0, and drafts that precede the cache's
    first row, see nothing; their output is 0 and their lse -inf."""
    lens = [0, 1, 2, 3, 7]
    z = torch.ones(5, 4, dtype=torch.bool)
    o, lse, _ = _run(5, 4, 4, 2, D, 0, 8, lens, z, seed=5)
    assert bool((o[:4] == 0).all()) and bool((lse[:, :4] == -math.inf).all())
    _run(5, 4, 4, 2, D, 3, 8, lens, z, seed=6)


@pytest.mark.parametrize("D,Hq,Hkv,n", [(128, 16, 4, 4), (64, 8, 1, 3), (128, 4, 4, 1)])
def test_many_rows_share_the_prefix(D, Hq, Hkv, n):
    """More rows of a KV head than one tile of 128 holds."""
    B = 45
    lens = [(37 * b) % 140 + n for b in range(B)]
    _run(B, n, Hq, Hkv, D, 700, 145, lens, _z(B, n, 0.9, D), seed=9)


@pytest.mark.parametrize("share", [0.9, 0.2])
@pytest.mark.parametrize("D,Hq,Hkv,n,P", [(128, 16, 4, 4, 2500), (64, 8, 1, 3, 6701)])
def test_many_rows_share_a_long_prefix(D, Hq, Hkv, n, P, share):
    """Enough rows and keys for 128-row tiles, and too few rows selected for them."""
    B = 45
    lens = [(37 * b) % 140 + n for b in range(B)]
    _run(B, n, Hq, Hkv, D, P, 145, lens, _z(B, n, share, D), seed=11)


@pytest.mark.parametrize("n,G", [(1, 4), (4, 8)])
def test_caches_that_end_inside_a_tile(n, G):
    """Every remainder of the cache's length modulo a copy's 32 rows and around them."""
    lens = [n, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 129, 159, 161, 191, 193, 223, 225]
    _run(len(lens), n, 2 * G, 2, 128, 40, 230, lens, _z(len(lens), n, 1.0, G), seed=n)


@pytest.mark.parametrize("P", [3, 130, 4000])
def test_many_sequences(P):
    """More than a CTA has threads; most of them not selected."""
    B, n = 400, 2
    lens = [(11 * b) % 19 + 1 for b in range(B)]
    _run(B, n, 4, 2, 64, P, 21, lens, _z(B, n, 0.3, P), seed=P)


@pytest.mark.parametrize("n,G,L", [(8, 40, 131), (33, 8, 200)])
def test_many_rows_of_a_sequence(n, G, L):
    """More rows than the join and the weights take in one launch."""
    lens = [L, n, 130, 1]
    _run(4, n, 2 * G, 2, 64, 70, L, lens, _z(4, n, 0.9, n), seed=n)


@pytest.mark.parametrize("D,Hq,Hkv,n", [(128, 4, 1, 1), (64, 16, 2, 2), (128, 32, 1, 5)])
def test_few_rows_long_prefix_and_caches(D, Hq, Hkv, n):
    _run(2, n, Hq, Hkv, D, 9001, 5000, [5000, 1700], torch.ones(2, n, dtype=torch.bool), seed=21)


def test_nothing_selected():
    """No output row is written; every weight is carried over."""
    from paper_2608_29539_gb300 import logo as Lg
    B, n, L = 3, 2, 50
    q, kp, vp, kc, vc = (t.cuda() for t in _inputs(B, n, 4, 2, 128, 40, L, 3))
    pos, cu, ns, _ = _pack(torch.zeros(B, n, dtype=torch.bool))
    lens = torch.tensor([50, 1, 30], dtype=torch.int32, device="cuda")
    o = torch.full((B * n, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((4, B * n), 3.0, device="cuda")
    m = torch.rand(B, 2, L, device="cuda")
    out = torch.full_like(m, -1.0)
    Lg.logo_decode_prefix_attn(q, kp, vp, kc, vc, lens, pos.cuda(), cu.cuda(), ns.cuda(), mass_in=m, mass_out=out,
                               o_c=o, lse_c=lse)
    torch.cuda.synchronize()
    assert bool((o == 3.0).all()) and bool((lse == 3.0).all())
    for b, k in enumerate([50, 1, 30]):
        old = max(0, k - n)
        assert torch.equal(out[b, :, :old], m[b, :, :old])
        assert bool((out[b, :, old:k] == 0).all()) and bool((out[b, :, k:] == -1).all())


def test_large_logits_and_scale():
    """Logits of a few hundred: one key takes all the weight of a row."""
    _run(4, 2, 4, 2, 128, 200, 150, [150, 2, 77, 128], torch.ones(4, 2, dtype=torch.bool), seed=33, scale=0.6, std=2.0)


def test_matches_the_decode_call_when_there_is_no_prefix():
    """The same caches through logo_decode_global_sparse_attn (bf16 outputs of
    the same sums: one rounding of weights and output each)."""
    from paper_2608_29539_gb300 import logo as Lg
    B, L, Hq, Hkv, D = 5, 900, 8, 2, 128
    q, _, _, kc, vc = (t.cuda() for t in _inputs(B, 1, Hq, Hkv, D, 0, L, 12))
    gate = torch.tensor([[0.9], [0.1], [0.8], [0.7], [0.2]], device="cuda")
    z, pos, cu, row_of, ns = Lg.logo_select(gate, Lg.LOGO_SELECT_THRESHOLD, b_th=0.5)
    lens = torch.tensor([900, 3, 128, 555, 1], dtype=torch.int32, device="cuda")
    a = Lg.logo_decode_global_sparse_attn(q.view(B, Hq, D), kc, vc, lens, cu, ns)
    b, lse, mass = Lg.logo_decode_prefix_attn(q, None, None, kc, vc, lens, pos, cu, ns)
    torch.cuda.synchronize()
    assert Lg.logo_get_device_status() == 0
    assert mass is None
    n = int(ns)
    assert n == 3
    err = (a[:n].double() - b[:n].double()).abs()
    absv = vc.double().abs().amax()
    assert float((err - 2.0 ** -7 * absv).max()) <= 0


def test_cache_offsets_beyond_32_bits():
    """K and V of 2^31 + elements each: the last sequence's last KV head."""
    from paper_2608_29539_gb300 import logo as Lg
    B, L, Hkv, D = 2, 131200, 64, 128
    assert B * L * Hkv * D > 2 ** 31
    kc = torch.zeros((B, L, Hkv, D), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    g = torch.Generator().manual_seed(4)
    tail_k = torch.randn((300, D), generator=g).to(torch.bfloat16)
    tail_v = torch.randn((300, D), generator=g).to(torch.bfloat16)
    kc[1, L - 300:, 63] = tail_k.cuda()
    vc[1, L - 300:, 63] = tail_v.cuda()
    q = torch.randn((B, 1, Hkv, D), generator=g).to(torch.bfloat16)
    q[:, :, 63] *= 4
    pos, cu, ns, rows = _pack(torch.ones(B, 1, dtype=torch.bool))
    lens = torch.tensor([5, L], dtype=torch.int32, device="cuda")
    m = torch.zeros(B, Hkv, L, device="cuda")
    o, lse, m = Lg.logo_decode_prefix_attn(q.cuda(), None, None, kc, vc, lens, pos.cuda(), cu.cuda(), ns.cuda(),
                                           mass_in=m)
    torch.cuda.synchronize()
    assert Lg.logo_get_device_status() == 0
    x = (q[1, 0, 63].double() @ tail_k.double().T) / math.sqrt(D)
    total = x.exp().sum() + (L - 300)
    E = 2.0 ** -24 * D * float((q[1, 0, 63].double().abs() @ tail_k.double().abs().T).max()) / math.sqrt(D)
    assert abs(float(lse[63, 1]) - math.log(total)) <= E + 2.0 ** -20 + 2.0 ** -22 * math.log(total)
    w = x.exp() / total
    ref = w @ tail_v.double()
    absv = w @ tail_v.double().abs()
    got = o[1, 63].double().cpu()
    assert ((got - ref).abs() <= 2.0 ** -8 * (ref.abs() + absv) + (2 * E + 2.0 ** -16) * absv).all()
    assert ((m[1, 63, L - 300:].double().cpu() - w).abs() <= (2 * E + 2.0 ** -18) * w).all()
    assert bool((o[0] == 0).all()) and float((m[0, :, :5] - 0.2).abs().max()) <= 2.0 ** -18


def test_captures_in_a_graph_and_runs_on_another_stream():
    from paper_2608_29539_gb300 import logo as Lg
    B, n, L = 4, 2, 300
    q, kp, vp, kc, vc = (t.cuda() for t in _inputs(B, n, 8, 2, 128, 333, L, 8))
    pos, cu, ns, _ = _pack(torch.ones(B, n, dtype=torch.bool))
    pos, cu, ns = pos.cuda(), cu.cuda(), ns.cuda()
    lens = torch.tensor([300, 2, 128, 200], dtype=torch.int32, device="cuda")
    m = torch.rand(B, 2, L, device="cuda")
    args = (q, kp, vp, kc, vc, lens, pos, cu, ns)
    ws = Lg.logo_decode_prefix_workspace(q, kp, kc, True)
    ref = [t.clone() for t in Lg.logo_decode_prefix_attn(*args, mass_in=m, mass_out=torch.zeros_like(m), workspace=ws)]
    o, lse, mo = torch.zeros_like(ref[0]), torch.zeros_like(ref[1]), torch.zeros_like(m)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Lg.logo_decode_prefix_attn(*args, mass_in=m, mass_out=mo, o_c=o, lse_c=lse, workspace=ws)
    torch.cuda.synchronize()
    for a, b in zip(ref, (o, lse, mo)):
        assert torch.equal(a, b)
    for t in (o, lse, mo):
        t.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Lg.logo_decode_prefix_attn(*args, mass_in=m, mass_out=mo, o_c=o, lse_c=lse, workspace=ws)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(ref, (o, lse, mo)):
        assert torch.equal(a, b)


def test_refusals():
    from paper_2608_29539_gb300 import logo as Lg
    B, n, L = 2, 1, 16
    q, kp, vp, kc, vc = (t.cuda() for t in _inputs(B, n, 4, 2, 64, 8, L, 1))
    pos, cu, ns, _ = _pack(torch.ones(B, n, dtype=torch.bool))
    pos, cu, ns = pos.cuda(), cu.cuda(), ns.cuda()
    lens = torch.tensor([4, 5], dtype=torch.int32, device="cuda")
    call = Lg.logo_decode_prefix_attn
    m = torch.zeros(B, 2, L, device="cuda")
    with pytest.raises(ValueError):
        call(q.float(), kp, vp, kc, vc, lens, pos, cu, ns)
    with pytest.raises(ValueError):
        call(q, kp, None, kc, vc, lens, pos, cu, ns)
    with pytest.raises(ValueError):
        call(q, kp, vp[:4], kc, vc, lens, pos, cu, ns)
    with pytest.raises(ValueError):
        call(q, kp, vp, kc.transpose(1, 2), vc, lens, pos, cu, ns)
    with pytest.raises(ValueError):
        call(q, kp, vp, kc, vc, lens.long(), pos, cu, ns)
    with pytest.raises(ValueError):
        call(q, kp, vp, kc, vc, lens, pos, cu[:2], ns)
    with pytest.raises(ValueError):
        call(q, kp, vp, kc, vc, lens, pos, cu, ns, mass_out=m)
    with pytest.raises(ValueError):
        call(q, kp, vp, kc, vc, lens, pos, cu, ns, mass_in=m[:, :, :8])
    with pytest.raises(ValueError):
        call(q, kp, vp, kc, vc, lens, pos, cu, ns, o_c=torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(Lg.LogoError) as e:
        call(q, kp, vp, kc, vc, lens, pos, cu, ns, scale=-1.0)
    assert e.value.code == Lg.LOGO_ERR_INVALID_ARG
    with pytest.raises(Lg.LogoError) as e:
        call(q, kp, vp, kc, vc, lens, pos, cu, ns, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == Lg.LOGO_ERR_WORKSPACE
    with pytest.raises(Lg.LogoError) as e:
        call(q[:, :, :3].contiguous(), kp, vp, kc, vc, lens, pos, cu, ns)
    assert e.value.code == Lg.LOGO_ERR_UNSUPPORTED
