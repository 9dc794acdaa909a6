"""logo_decode_cache4_attn against attention in 64 bits over the values that the
cache holds.

Bounds, from the arithmetic: a logit is a sum of D exact products in fp32, scaled
once: off by (D + 8) 2^-24 of scale * sum |q k| at most, and its exponential by that
plus 2^-20 (the approximate exp2 and its argument's rounding up to |x| = 16).  A
weight is rounded to fp16 for the product (2^-11 of it, or 2^-25 of the row's largest
weight), sums over len keys in fp32 add len 2^-24.  The output is rounded to bf16 once
(2^-8)."""
import numpy as np
import pytest
import torch

import cache4_ref as R

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def _logo():
    from paper_2608_29539_gb300 import logo
    return logo


def _inputs(B, n, Hq, Hkv, D, L, lens, seed):
    """Queries, and caches whose rows past each length hold anything, NaN scales too."""
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((B, n, Hq, D), generator=g).to(torch.bfloat16)
    parts = []
    for _ in range(2):
        c, s = R.quantise(torch.randn((B, Hkv, L, D), generator=g).to(torch.bfloat16))
        for b in range(B):
            m = max(0, lens[b])
            c[b, :, m:] = torch.randint(0, 256, c[b, :, m:].shape, generator=g, dtype=torch.uint8)
            s[b, :, m:] = torch.randint(200, 256, s[b, :, m:].shape, generator=g, dtype=torch.uint8)
        parts.append((c, s))
    (kc, ks), (vc, vs) = parts
    return q, kc, vc, ks, vs


def _pack(z):
    """z [B, n] bool -> pos, cu_q, n_sel, rows."""
    B, n = z.shape
    rows = [(b, i) for b in range(B) for i in range(n) if z[b, i]]
    pos = torch.full((B * n,), -7, dtype=torch.int32)
    pos[:len(rows)] = torch.tensor([i for _, i in rows], dtype=torch.int32)
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = z.sum(1).cumsum(0)
    return pos, cu, cu[-1:].clone(), rows


def _call(q, kc, vc, ks, vs, lens, pos, cu, ns, scale=0.0):
    logo = _logo()
    d = lambda t: t.cuda().contiguous()  # noqa: E731
    q = d(q)
    cache = logo.Cache4(d(kc), d(vc), d(ks), d(vs))
    ws = logo.logo_decode_cache4_workspace(q, cache)
    ws.fill_(255)
    B, n, Hq, D = q.shape
    o = torch.full((B * n, Hq, D), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((Hq, B * n), 5.0, device="cuda")
    logo.logo_decode_cache4_attn(q, cache, torch.tensor(lens, dtype=torch.int32, device="cuda"), d(pos), d(cu), d(ns),
                                 scale, o, lse, ws)
    torch.cuda.synchronize()
    assert logo.logo_get_device_status() == 0
    N = int(ns)
    assert (o[N:] == 3).all() and (lse[:, N:] == 5).all()
    return o[:N].double().cpu().numpy(), lse[:, :N].double().cpu().numpy()


def _check(o, lse, ref, D, most):
    seen = np.isfinite(ref["lse"])
    assert np.array_equal(seen, np.isfinite(lse)) and (lse[~seen] == -np.inf).all()
    x = (D + 8) * 2.0 ** -24 * ref["big"] + 2.0 ** -20
    sums = most * 2.0 ** -24
    assert (np.abs(lse[seen] - ref["lse"][seen]) <= x + sums + 2.0 ** -23 * np.abs(ref["lse"][seen])).all()
    bound = 2.0 ** -8 * np.abs(ref["o"]) + ref["absv"] * (2.0 ** -11 + 2 * x + 2 * sums) + 2.0 ** -25 * ref["sumv"]
    err = np.abs(o - ref["o"])
    assert (err <= 1.01 * bound).all(), float((err / np.maximum(bound, 1e-30)).max())


def _some(B, n, seed, share):
    z = torch.rand((B, n), generator=torch.Generator().manual_seed(seed)) < share
    if B > 2:
        z[1] = False  # a sequence without a selected token
    z[0, n - 1] = True
    return z


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,Hkv,n", [(1, 1, 1), (4, 2, 1), (8, 1, 1), (3, 2, 3), (4, 2, 4), (5, 1, 5), (16, 1, 2),
                                     (8, 1, 8), (1, 3, 7), (13, 1, 1), (16, 1, 9)])
def test_heads_and_drafts(D, G, Hkv, n):
    L = 300
    lens = [n, 57, 32, 33, 31, L, max(1, n - 1), 129, 64]
    B = len(lens)
    x = _inputs(B, n, G * Hkv, Hkv, D, L, lens, G + n)
    pos, cu, ns, rows = _pack(_some(B, n, n, 0.7))
    ref = R.attn(x[0], R.values(x[1], x[3]), R.values(x[2], x[4]), lens, rows)
    _check(*_call(*x, lens, pos, cu, ns), ref, D, L)


@pytest.mark.parametrize("D,L,B,n,G,Hkv", [(128, 9001, 2, 1, 4, 2), (64, 20011, 1, 2, 2, 1), (128, 4097, 1, 5, 8, 1),
                                           (64, 2048, 3, 8, 8, 2), (128, 70001, 1, 1, 2, 1)])
def test_long(D, L, B, n, G, Hkv):
    lens = [L, L // 2 + 3, L - 31][:B]
    x = _inputs(B, n, G * Hkv, Hkv, D, L, lens, 5)
    pos, cu, ns, rows = _pack(torch.ones((B, n), dtype=torch.bool))
    ref = R.attn(x[0], R.values(x[1], x[3]), R.values(x[2], x[4]), lens, rows)
    _check(*_call(*x, lens, pos, cu, ns), ref, D, L)


@pytest.mark.parametrize("B,L,n,G,Hkv,D", [(400, 70, 1, 4, 2, 64), (1100, 9, 2, 1, 1, 128), (130, 200, 3, 3, 3, 128)])
def test_many_sequences(B, L, n, G, Hkv, D):
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, L + 1, (B,), generator=g).tolist()
    x = _inputs(B, n, G * Hkv, Hkv, D, L, lens, 6)
    z = torch.rand((B, n), generator=g) < 0.5
    z[0, 0] = True
    pos, cu, ns, rows = _pack(z)
    ref = R.attn(x[0], R.values(x[1], x[3]), R.values(x[2], x[4]), lens, rows)
    _check(*_call(*x, lens, pos, cu, ns), ref, D, L)


def test_empty():
    """Empty caches, lengths out of range, drafts that come before any key, no selected
    row at all."""
    B, n, L, D = 5, 3, 40, 64
    lens = [0, 1, 2, -5, 99]
    x = _inputs(B, n, 4, 2, D, L, [min(max(m, 0), L) for m in lens], 7)
    pos, cu, ns, rows = _pack(torch.ones((B, n), dtype=torch.bool))
    cut = [min(max(m, 0), L) for m in lens]
    ref = R.attn(x[0], R.values(x[1], x[3]), R.values(x[2], x[4]), cut, rows)
    o, lse = _call(*x, lens, pos, cu, ns)
    _check(o, lse, ref, D, L)
    assert (o[:3] == 0).all() and (lse[:, :3] == -np.inf).all() and (lse[:, 12:] > -np.inf).all()
    pos, cu, ns, rows = _pack(torch.zeros((B, n), dtype=torch.bool))
    _call(*x, lens, pos, cu, ns)


@pytest.mark.parametrize("size", [1e-30, 1e-6, 300.0, 1e6])
def test_sizes_of_queries(size):
    """Tiny and huge queries: the fp16 product sees them scaled by a power of two."""
    B, n, L, D = 2, 2, 100, 128
    lens = [100, 37]
    q, *x = _inputs(B, n, 4, 1, D, L, lens, 8)
    q = (q.float() * size).to(torch.bfloat16)
    pos, cu, ns, rows = _pack(torch.ones((B, n), dtype=torch.bool))
    scale = 1.0 / (D ** 0.5 * max(size, 1e-6))
    ref = R.attn(q, R.values(x[0], x[2]), R.values(x[1], x[3]), lens, rows, scale)
    _check(*_call(q, *x, lens, pos, cu, ns, scale), ref, D, L)


def test_peaked_and_rising():
    """Logits that rise along the cache by far more than a rescaling takes, and ones
    that one key dominates."""
    B, n, L, D = 1, 1, 500, 64
    q = torch.ones((B, n, 2, D), dtype=torch.bfloat16)
    rise = torch.linspace(-6, 6, L)[None, None, :, None].expand(B, 1, L, D)
    g = torch.Generator().manual_seed(2)
    kc, ks = R.quantise(rise.to(torch.bfloat16))
    vc, vs = R.quantise(torch.randn((B, 1, L, D), generator=g).to(torch.bfloat16))
    pos, cu, ns, rows = _pack(torch.ones((B, n), dtype=torch.bool))
    for scale in (0.05, 1.0, 8.0):
        for c, s in ((kc, ks), (kc.flip(2), ks.flip(2))):
            ref = R.attn(q, R.values(c, s), R.values(vc, vs), [L], rows, scale)
            _check(*_call(q, c, vc, s, vs, [L], pos, cu, ns, scale), ref, D, L)


@pytest.mark.parametrize("D,G,n", [(128, 2, 4), (64, 8, 3), (128, 9, 5), (64, 1, 8)])
def test_nan_of_unseen_drafts(D, G, n):
    """A draft whose values (or keys) hold a NaN: it shows in the rows that see it, in
    the channels of its group, and in no other row."""
    Hkv, L = 2, 90
    lens = [n, 31 + n, 64, 90]
    B = len(lens)
    q, kc, vc, ks, vs = _inputs(B, n, G * Hkv, Hkv, D, L, lens, 9)
    pos, cu, ns, rows = _pack(torch.ones((B, n), dtype=torch.bool))
    clean = R.attn(q, R.values(kc, ks), R.values(vc, vs), lens, rows)
    first = [1 + b % (n - 1) for b in range(B)]
    group = [b % (D // 16) for b in range(B)]
    for where in ("v", "k"):
        sc = (vs if where == "v" else ks).clone()
        for b in range(B):
            for j in range(first[b], n):
                sc[b, :, lens[b] - n + j, group[b]] = 255
        o, lse = _call(q, kc, vc, ks if where == "v" else sc, sc if where == "v" else vs, lens, pos, cu, ns)
        for r, (b, i) in enumerate(rows):
            if i < first[b]:
                one = {k: clean[k][:, r:r + 1] if k == "lse" else clean[k][r:r + 1] for k in ("o", "lse", "absv", "sumv")}
                _check(o[r:r + 1], lse[:, r:r + 1], one | {"big": clean["big"]}, D, L)
            elif where == "k":
                assert np.isnan(o[r]).all() and np.isnan(lse[:, r]).all()
            else:
                bad = np.zeros(D, bool)
                bad[16 * group[b]:16 * group[b] + 16] = True
                assert np.isnan(o[r][:, bad]).all() and np.isfinite(o[r][:, ~bad]).all() and np.isfinite(lse[:, r]).all()


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_queries_that_are_not_finite(bad):
    B, n, L, D = 2, 2, 50, 128
    lens = [50, 20]
    q, *x = _inputs(B, n, 4, 2, D, L, lens, 10)
    pos, cu, ns, rows = _pack(torch.ones((B, n), dtype=torch.bool))
    ref = R.attn(q, R.values(x[0], x[2]), R.values(x[1], x[3]), lens, rows)
    q[1, 0, 3, 17] = bad
    o, lse = _call(q, *x, lens, pos, cu, ns)
    assert np.isnan(o[2, 3]).all() and np.isnan(lse[3, 2])
    o[2, 3], lse[3, 2] = ref["o"][2, 3], ref["lse"][3, 2]
    _check(o, lse, ref, D, L)


def test_same_bits_in_a_graph_and_on_other_streams():
    """Two captured calls that share nothing but the inputs, replayed with new queries and
    lengths, and calls on two streams with a workspace each, give the eager call's bits."""
    logo = _logo()
    B, n, Hq, Hkv, D, L = 3, 2, 8, 2, 128, 3000
    lens = [3000, 1234, 7]
    q, kc, vc, ks, vs = _inputs(B, n, Hq, Hkv, D, L, lens, 11)
    cache = logo.Cache4(*(t.cuda() for t in (kc, vc, ks, vs)))
    pos, cu, ns, _ = (t.cuda() if torch.is_tensor(t) else t for t in _pack(torch.ones((B, n), dtype=torch.bool)))
    dq, seq = q.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    eager = lambda: [t.clone() for t in logo.logo_decode_cache4_attn(dq, cache, seq, pos, cu, ns)]  # noqa: E731
    eager()
    side = torch.cuda.Stream()
    outs, graphs = [], []
    for _ in range(2):
        ws = logo.logo_decode_cache4_workspace(dq, cache)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(logo.logo_decode_cache4_attn(dq, cache, seq, pos, cu, ns, workspace=ws))
        graphs.append((graph, ws))
    for step in range(3):
        dq.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(step)))
        seq.copy_(torch.tensor([2999 - step, 40 * step + 2, 3000], dtype=torch.int32))
        want = eager()
        side.wait_stream(torch.cuda.current_stream())
        graphs[0][0].replay()
        with torch.cuda.stream(side):
            graphs[1][0].replay()
            again = logo.logo_decode_cache4_attn(dq, cache, seq, pos, cu, ns)
        torch.cuda.current_stream().wait_stream(side)
        for got in (*outs, again):
            # (as bits: the lengths reach rows that hold anything, NaN too)
            assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(got, want))


@pytest.mark.parametrize("n,G", [(1, 4), (3, 4)])
def test_offsets_past_32_bits(n, G):
    """Rows written, read and attended past 2^32 bytes of codes.  All other rows hold zeros:
    a logit of 0 each and nothing added to the sums."""
    logo = _logo()
    B, Hkv, D, L = 2, 8, 128, 2 ** 22 + 2 ** 18 + 77
    assert B * Hkv * L * (D // 2) > 2 ** 32 > (B * Hkv - 1) * L * (D // 2)
    g = torch.Generator().manual_seed(n)
    bf = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)  # noqa: E731
    q, k, v = bf(B, n, G * Hkv, D), bf(B, 5, Hkv, D) * 4, bf(B, 5, Hkv, D)
    cache = logo.logo_cache4_empty(B, L, Hkv, D)
    lens = [700, L]
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    logo.logo_cache4_append(cache, k.cuda(), v.cuda(), seq)
    k, v = (R.values(*R.quantise(x)) for x in (k, v))
    rows = (seq[:, None] - 5 + torch.arange(5, device="cuda")).int()
    for got, want in zip(logo.logo_cache4_read(cache, seq, rows=rows), (k, v)):
        assert torch.equal(got.double().cpu(), want)
    pos, cu, ns, packed = (t.cuda() if torch.is_tensor(t) else t for t in _pack(torch.ones((B, n), dtype=torch.bool)))
    o, lse = logo.logo_decode_cache4_attn(q.cuda(), cache, seq, pos, cu, ns)
    for r in range(B * n):
        b, i = divmod(r, n)
        m = 5 - n + i + 1  # of the rows that are not zeros it sees these
        for h in range(G * Hkv):
            kk, vv, qq = k[b, :m, h // G], v[b, :m, h // G], q[b, i, h].double()
            w = torch.exp(kk @ qq / D ** 0.5)
            total = w.sum() + lens[b] - n + i + 1 - m
            want, absv = w @ vv / total, w @ vv.abs() / total
            x = (D + 8) * 2.0 ** -24 * float((kk.abs() @ qq.abs()).max()) / D ** 0.5 + 2.0 ** -20
            # no thread adds more than 4 weights for each of 1/456 of the 8 heads' units of 128 rows
            sums = 3000 * 2.0 ** -24
            tol = 2.0 ** -8 * want.abs() + absv * (2.0 ** -11 + 2 * x + 2 * sums) + 2.0 ** -25 * w.max() / total * vv.abs().sum(0)
            assert ((o[r, h].double().cpu() - want).abs() <= 1.01 * tol).all()
            assert abs(float(lse[h, r]) - float(torch.log(total))) <= x + sums + 2.0 ** -23 * abs(float(torch.log(total)))


def test_refusals():
    logo = _logo()
    cache = logo.logo_cache4_empty(2, 16, 2, 64)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    good = dict(q=bf(2, 1, 4, 64), cache=cache, seq_len=i32(2), pos=i32(2), cu_q=i32(3), n_sel_total=i32(1))
    logo.logo_decode_cache4_attn(**good)
    for kw in (dict(q=bf(2, 4, 64)), dict(q=bf(3, 1, 4, 64)), dict(q=bf(2, 1, 4, 128)), dict(pos=i32(3)),
               dict(cu_q=i32(2)), dict(seq_len=i32(2).long()), dict(n_sel_total=i32(2)), dict(o_c=bf(2, 4, 32)),
               dict(lse_c=torch.zeros(2, 4, device="cuda")), dict(workspace=torch.zeros(1 << 20, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            logo.logo_decode_cache4_attn(**(good | kw))
    with pytest.raises(logo.LogoError, match="UNSUPPORTED"):
        logo.logo_decode_cache4_attn(**(good | dict(q=bf(2, 1, 5, 64))))
    with pytest.raises(logo.LogoError, match="WORKSPACE"):
        logo.logo_decode_cache4_attn(**good, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("D,G,n", [(128, 4, 1), (64, 2, 3), (128, 4, 5), (64, 8, 4)])
@pytest.mark.parametrize("far", [15.0, 17.0, 18.0, 20.0])
def test_the_tail_beside_one_key_that_takes_nearly_all_weight(D, G, n, far):
    """One key with V = 0, `far` above all others, whose V is what comes out.  As many
    sequences as there are groups of warps, so that each has a run of its own.  Weights go
    through fp16 relative to 2^-10 of the largest: off by 2^-11 of themselves or by 2^-25 2^-10
    of the largest weight, at most.  Each group adds its 16 units of 128 keys in
    steps of 16 and joins a few sums: fewer than 100 additions, an ulp each."""
    L, B, Hkv = 2048, 640, 1
    g = torch.Generator().manual_seed(int(far))
    kc, ks = R.quantise(torch.cat([torch.full((1, 1, 1, D), 6.0), torch.zeros(1, 1, L - 1, D)], 2).to(torch.bfloat16))
    v = torch.rand((1, 1, L, D), generator=g) + 0.5
    v[:, :, 0] = 0
    vc, vs = R.quantise(v.to(torch.bfloat16))
    q = torch.ones((1, n, G * Hkv, D), dtype=torch.bfloat16)
    scale = far / (6 * D)
    ref = R.attn(q, R.values(kc, ks), R.values(vc, vs), [L], [(0, i) for i in range(n)], scale)
    pos, cu, ns, _ = _pack(torch.ones((B, n), dtype=torch.bool))
    many = lambda t: t.expand(B, *t.shape[1:])  # noqa: E731
    o, lse = _call(*(many(t) for t in (q, kc, vc, ks, vs)), [L] * B, pos, cu, ns, scale)
    x = (D + 8) * 2.0 ** -24 * ref["big"] + 2.0 ** -20
    rel = 2.0 ** -11 + 2 * x + 100 * 2.0 ** -23
    want = np.tile(ref["o"], (B, 1, 1))
    bound = 2.0 ** -8 * want + np.tile(ref["absv"] * rel + ref["sumv"] * 2.0 ** -35, (B, 1, 1))
    err = np.abs(o - want)
    assert (err <= 1.01 * bound).all(), float((err / want).max())
    assert (np.abs(lse - np.tile(ref["lse"], (1, B))) <= x + 100 * 2.0 ** -23 + 2.0 ** -23 * far).all()


@pytest.mark.parametrize("D,G,n", [(128, 4, 1), (64, 8, 4)])
@pytest.mark.parametrize("size", [1e3, 1e6, 3e7])
def test_large_logits(D, G, n, size):
    """Logits up to `size`, in no order: whatever their rounding, weights stay finite and what
    comes out is a mean of V, all of which is between 0.5 and 1.5."""
    L, B = 1024, 640
    g = torch.Generator().manual_seed(D)
    kc, ks = R.quantise(torch.randn((1, 1, L, D), generator=g).to(torch.bfloat16))
    vc, vs = R.quantise((torch.rand((1, 1, L, D), generator=g) + 0.5).to(torch.bfloat16))
    low, high = float(R.values(vc, vs).min()), float(R.values(vc, vs).max())
    q = torch.randn((1, n, G, D), generator=g).to(torch.bfloat16)
    pos, cu, ns, _ = _pack(torch.ones((B, n), dtype=torch.bool))
    many = lambda t: t.expand(B, *t.shape[1:])  # noqa: E731
    raw = torch.einsum("nhd,ld->nhl", q[0].double(), R.values(kc, ks)[0, 0])
    scale = size / float(raw.abs().max())
    o, lse = _call(*(many(t) for t in (q, kc, vc, ks, vs)), [L] * B, pos, cu, ns, scale)
    slack = 1 + 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -16  # o's rounding, a weight's, the sums'
    assert (o >= low / slack).all() and (o <= high * slack).all()
    for i in range(n):
        want = torch.logsumexp(scale * raw[i, :, :L - n + i + 1], 1).numpy()
        x = (D + 8) * 2.0 ** -24 * scale * float(torch.einsum("hd,ld->hl", q[0, i].double().abs(), R.values(kc, ks)[0, 0].abs()).max())
        assert (np.abs(lse[:, i::n] - want[:, None]) <= x + 2.0 ** -16 + 2.0 ** -23 * np.abs(want[:, None])).all()
