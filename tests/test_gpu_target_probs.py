"""logo_target_probs against its definition in 64 bits.

Bounds, from the arithmetic: up to seven float32 operations make x / T out of the
logit, each off by 2^-24 of a value no larger than the largest that occurs; the
difference to the row's largest adds one more, exp and the division a few 2^-23, the
sum of V positive terms (in at most V / 256 + 64 steps a chain) as many 2^-24.  Below
2^-126 a float32 keeps no digits."""
import numpy as np
import pytest
import torch

import cache4_ref as R

pytestmark = pytest.mark.gpu


def _logo():
    from paper_2608_29539_gb300 import logo
    return logo


def _words(ok):
    """bool [..., V] -> int32 [..., ceil(V / 32)]; the bits past V are set."""
    V = ok.shape[-1]
    pad = torch.ones(*ok.shape[:-1], -V % 32, dtype=torch.bool)
    bits = torch.cat([ok, pad], -1).unflatten(-1, (-1, 32)).long()
    w = (bits << torch.arange(32)).sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).int()


def _random(B, m1, V, H, K, seed, mask=True, half=False, T=None):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, m1, V), generator=g) * 3
    s = dict(logits=x.to(torch.bfloat16) if half else x)
    s["temperature"] = torch.rand(B, generator=g) + 0.4 if T is None else torch.tensor(T)
    ids = lambda *n: (torch.rand(n, generator=g) ** 3 * (V + 2)).int() - 1  # noqa: E731  (-1, V and repetitions too)
    if H or m1 > 1:
        s["penalty"] = torch.stack([torch.rand(B, generator=g) + 0.7, torch.randn(B, generator=g) * 0.3,
                                    torch.randn(B, generator=g) * 0.5], 1)
        s["penalty"][0, 0] = 1.7
    if H:
        s["history"] = ids(B, H)
        s["hist_len"] = torch.randint(0, H + 1, (B,), generator=g).int()
        s["hist_len"][0] = H
        s["n_prompt"] = (s["hist_len"] * torch.rand(B, generator=g)).int()
    if m1 > 1:
        s["draft"] = ids(B, m1 - 1)
        s["draft"][0] = 0
    if K:
        s["bias_tok"], s["bias_val"] = ids(B, K), torch.randn((B, K), generator=g) * 2
    ok = None
    if mask:
        ok = torch.rand((B, m1, V), generator=g) < torch.rand((B, m1, 1), generator=g)
        ok[-1, -1] = False  # a row that allows nothing
        s["allowed"] = _words(ok)
    return s, ok


def _row(s, ok, b, i, real=np.float64):
    hist = s["history"][b, :max(0, min(int(s["hist_len"][b]), s["history"].shape[1]))].tolist() if "history" in s else []
    n_prompt = int(s["n_prompt"][b]) if "n_prompt" in s else 0
    return R.adjusted(s["logits"][b, i].float().numpy(), s["penalty"][b].numpy() if "penalty" in s else None, hist, n_prompt,
                      s["draft"][b, :i].tolist() if "draft" in s else [],
                      list(zip(s["bias_tok"][b].tolist(), s["bias_val"][b].numpy())) if "bias_tok" in s else [],
                      None if ok is None else ok[b, i].numpy(), real=real)


def _run(s, **kw):
    return _logo().logo_target_probs(**{k: v.cuda().contiguous() for k, v in s.items()}, **kw)


def _check(s, ok, p):
    B, m1, V = s["logits"].shape
    p = p.double().cpu().numpy()
    for b in range(B):
        T = float(s["temperature"][b]) if "temperature" in s else 1.0
        for i in range(m1):
            if T == 0:
                want = R.probs(_row(s, ok, b, i, np.float32), 0.0, None if ok is None else ok[b, i].numpy())
                assert np.array_equal(p[b, i], want)
                continue
            x = _row(s, ok, b, i)
            want = R.probs(x, T, None if ok is None else ok[b, i].numpy())
            size = max(np.abs(x[np.isfinite(x)]).max(initial=0.0), float(s["logits"][b, i].float().abs().max())) / min(T, 1.0)
            rel = 2.0 ** -24 * (9 * size * 2 + V / 256 + 96)
            err = np.abs(p[b, i] - want)
            assert (err <= rel * want + 2.0 ** -126).all(), (b, i, float((err / np.maximum(want, 1e-30)).max()), rel)


@pytest.mark.parametrize("B,m1,V,H,K,half", [
    (1, 1, 1, 3, 1, False), (2, 1, 31, 0, 0, False), (1, 2, 33, 5, 3, True), (3, 4, 1000, 40, 7, True),
    (2, 3, 4099, 700, 30, False), (1, 1, 32000, 300, 0, False), (5, 2, 50021, 2000, 200, True), (1, 8, 131072, 64, 5, True),
    (1, 1, 262143, 100, 300, False), (1, 1, 278528, 10, 2, True), (40, 1, 2053, 9, 1, False), (2, 300, 257, 50, 3, True),
    (3, 3, 16377, 90, 9, False), (3, 3, 16379, 90, 9, True)])
def test_against_the_definition(B, m1, V, H, K, half):
    s, ok = _random(B, m1, V, H, K, V + H, half=half)
    _check(s, ok, _run(s))


@pytest.mark.parametrize("drop", [("allowed",), ("temperature",), ("n_prompt",), ("history", "hist_len", "n_prompt"),
                                  ("draft",), ("penalty", "history", "hist_len", "n_prompt", "draft"),
                                  ("bias_tok", "bias_val")])
def test_parts_left_out(drop):
    s, ok = _random(3, 3, 5000, 60, 9, 4)
    for name in drop:
        del s[name]
    _check(s, None if "allowed" in drop else ok, _run(s))


@pytest.mark.parametrize("B,m1,V,H,K,half", [(1, 2, 30011, 12000, 3, False), (2, 1, 9001, 9500, 0, True),
                                             (1, 1, 278528, 4000, 4096, True), (1, 3, 262147, 4000, 4096, False)])
def test_long_lists(B, m1, V, H, K, half):
    """More listed tokens than are counted in shared memory, and as many as are; in place where
    that can be."""
    s, ok = _random(B, m1, V, H, K, V + H, half=half)
    _check(s, ok, _run(s))
    if not half:
        d = {k: v.cuda() for k, v in s.items()}
        _check(s, ok, _logo().logo_target_probs(**d, p=d["logits"]))


def test_offsets_past_32_bits():
    """The last rows of 2^32 tokens and more; those ahead of them are uniform."""
    B, m1, V = 15421, 1, 278528
    s, ok = _random(2, m1, V, 40, 3, 12, mask=False, half=True)
    grow = lambda t, x=0: torch.cat([t.new_full((B - 2, *t.shape[1:]), x).cuda(), t.cuda()])  # noqa: E731
    d = {k: grow(v, 1 if k in ("temperature", "penalty") else 0) for k, v in s.items()}
    d["bias_tok"][:-2] = -1
    p = _logo().logo_target_probs(**d)
    assert (B - 2) * V < 2 ** 32 < B * V
    _check(s, None, p[-2:])
    for b in (0, B // 2, B - 3):
        assert ((p[b] * V - 1).abs() < 1e-4).all()


@pytest.mark.parametrize("V", [40013, 5003])
def test_in_place(V):
    s, ok = _random(2, 3, V, 60, 9, 5)
    x = s["logits"].cuda()
    others = {k: v.cuda() for k, v in s.items() if k != "logits"}
    out = _logo().logo_target_probs(x, **others, p=x)
    assert out is x
    _check(s, ok, x)


@pytest.mark.parametrize("V", [37, 16379, 70001])
def test_greedy(V):
    """Ties go to the lowest token, also where a penalty or a bias makes them."""
    s, ok = _random(4, 3, V, 30, 5, 6, half=True, T=[0.0, 0.7, 0.0, 0.0])
    s["logits"][0] = 2.0
    s["logits"][2, 1, V // 2:] = 50.0
    ok[0, 0] = True
    s["allowed"] = _words(ok)
    _check(s, ok, _run(s))


def test_counts_and_sums():
    """One token all along a long history, the latest of which count, and one listed
    often among the biases: the sum is in the list's order."""
    V, H, K = 100, 20000, 4096
    g = torch.Generator().manual_seed(3)
    s = dict(logits=torch.zeros(2, 2, V), penalty=torch.tensor([[1.5, 2.0 ** -10, 0.25], [1.0, 2.0 ** -8, 0.0]]),
             history=torch.full((2, H), 3, dtype=torch.int32), hist_len=torch.tensor([H, 17000], dtype=torch.int32),
             n_prompt=torch.tensor([5, 12000], dtype=torch.int32), draft=torch.full((2, 1), 3, dtype=torch.int32),
             bias_tok=torch.full((2, K), 7, dtype=torch.int32), bias_val=torch.randn((2, K), generator=g) * 0.05)
    s["logits"][:, :, 3] = 4.0
    p = _run(s)
    _check_sum = np.float32(0)
    for v in s["bias_val"][0].numpy():
        _check_sum = np.float32(_check_sum + v)
    got = torch.log(p[0, 0].double() / p[0, 0, 0].double()).cpu()
    assert abs(float(got[7]) - float(_check_sum)) < 1e-5
    # 16384 generated ones count in row 0, the draft too in row 1; 5000 and 5001 in sequence 1
    want = [[4 / 1.5 - 16384 / 1024 - 0.25, 4 / 1.5 - 16385 / 1024 - 0.25], [4 - 5000 / 256, 4 - 5001 / 256]]
    for b in range(2):
        for i in range(2):
            q = torch.log(p[b, i].double() / p[b, i, 0].double()).cpu()
            assert abs(float(q[3]) - want[b][i]) < 1e-5


@pytest.mark.parametrize("V", [3000, 20011])
def test_values_that_are_not_finite(V):
    x = torch.randn((8, 1, V), generator=torch.Generator().manual_seed(1))
    ok = torch.rand((8, 1, V), generator=torch.Generator().manual_seed(2)) < 0.5
    ok[:, :, :20] = True
    nan, inf = float("nan"), float("inf")
    x[0, 0, 5] = nan                      # an allowed NaN
    x[1, 0, ~ok[1, 0]] = nan              # NaN in masked places
    x[2, 0, ~ok[2, 0]] = inf
    x[3, 0, 7] = inf
    x[4] = -inf                           # nothing left
    x[5, 0, 3:] = -inf
    x[6, 0, 9] = inf                      # greedy: the infinity is the largest
    x[7, 0] = torch.finfo(torch.float32).min
    T = torch.ones(8)
    T[6] = 0
    s = dict(logits=x, temperature=T, allowed=_words(ok))
    p = _run(s).double().cpu().numpy()
    for b in range(8):
        with np.errstate(invalid="ignore"):
            want = R.probs(np.where(ok[b, 0].numpy(), x[b, 0].double().numpy(), -np.inf), float(T[b]), ok[b, 0].numpy())
        assert np.array_equal(np.isnan(p[b, 0]), np.isnan(want)), b
        assert np.allclose(np.nan_to_num(p[b, 0]), np.nan_to_num(want), rtol=1e-5, atol=1e-30), b


@pytest.mark.parametrize("V", [9001, 33001])
def test_the_same_in_a_graph(V):
    s, ok = _random(3, 4, V, 100, 10, 8, half=True)
    d = {k: v.cuda() for k, v in s.items()}
    logo = _logo()
    logo.logo_target_probs(**d)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p = logo.logo_target_probs(**d)
    for step in range(3):
        d["logits"].copy_(torch.randn(s["logits"].shape, generator=torch.Generator().manual_seed(step)))
        d["hist_len"].fill_(30 * step)
        graph.replay()
        assert torch.equal(p, logo.logo_target_probs(**d))


def test_makes_what_verification_takes():
    """Greedy rows: verification accepts the drafts that are the largest logits."""
    logo = _logo()
    B, m, V = 4, 3, 5000
    g = torch.Generator().manual_seed(9)
    logits = torch.randn((B, m + 1, V), generator=g).cuda()
    draft = logits[:, :m].argmax(-1).int()
    draft[1, 1] = (draft[1, 1] + 1) % V
    p = logo.logo_target_probs(logits, temperature=torch.zeros(B, device="cuda"))
    q = torch.nn.functional.one_hot(draft.long(), V).float()
    tokens, n = logo.logo_verify_draft(draft, q, p, torch.rand((B, m), device="cuda"),
                                       torch.empty((B, V), device="cuda").exponential_())
    assert n.tolist() == [m, 1, m, m]
    best = logits.argmax(-1).int()
    assert tokens[1].tolist() == [int(draft[1, 0]), int(best[1, 1]), -1, -1] and torch.equal(tokens[0], best[0])


def test_refusals():
    logo = _logo()
    x = torch.zeros(2, 3, 64, device="cuda")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    pen = f(2, 3)
    for kw in (dict(logits=x.half()), dict(logits=x[0]), dict(logits=x[:, :, ::2]), dict(logits=x.cpu()),
               dict(temperature=f(3)), dict(penalty=f(2, 2)), dict(history=i32(2, 5)), dict(history=i32(2, 5), penalty=pen),
               dict(hist_len=i32(2)), dict(n_prompt=i32(2), penalty=pen), dict(draft=i32(2, 2)),
               dict(draft=i32(2, 3), penalty=pen), dict(bias_tok=i32(2, 4)), dict(bias_val=f(2, 4)),
               dict(bias_tok=i32(2, 4), bias_val=f(2, 3)), dict(allowed=i32(2, 3, 3)), dict(p=f(2, 3, 32)),
               dict(history=i32(5), hist_len=i32(2), penalty=pen)):
        with pytest.raises(ValueError):
            logo.logo_target_probs(**(dict(logits=x) | kw))
    # empty lists are none
    want = logo.logo_target_probs(x)
    assert torch.equal(want, logo.logo_target_probs(x, penalty=pen + 1, history=i32(2, 0), hist_len=i32(2),
                                                    bias_tok=i32(2, 0), bias_val=f(2, 0)))


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", [3000, 20011])
def test_lists_with_values_that_are_not_finite(V, half):
    """NaN and infinities at tokens that a history or a bias names, allowed and masked, for one
    CTA a row and for two passes; and ones that the penalties and biases make."""
    B, H, K = 14, 40, 6
    nan, inf = float("nan"), float("inf")
    g = torch.Generator().manual_seed(V)
    x = torch.randn((B, 1, V), generator=g) * 2
    hist = torch.randint(0, V, (B, H), generator=g).int()
    hist[:, :8] = torch.arange(8) * (V // 8)
    tok = torch.full((B, K), -1, dtype=torch.int32)
    tok[:, 0] = 11
    val = torch.randn((B, K), generator=g)
    penalty = torch.tensor([1.3, 0.25, 0.5]).repeat(B, 1)
    ok = torch.rand((B, 1, V), generator=g) < 0.5
    ok.scatter_(2, hist.long()[:, None], True)
    ok[:, :, 11:13] = True
    T = torch.ones(B)
    h3 = V // 8 * 3                            # a listed token
    x[0, 0, h3] = nan                          # allowed: shows
    x[1, 0, h3], ok[1, 0, h3] = nan, False     # masked: does not
    x[2, 0, h3], ok[2, 0, h3] = inf, False
    x[3, 0, h3] = inf
    x[4] = -inf                                # nothing left, listed tokens among it
    x[5] = -inf
    x[5, 0, hist[5].long()] = 0.5              # listed ones alone are left
    T[6], x[6, 0, h3] = 0.0, inf               # greedy: the largest
    T[7], x[7, 0, h3] = 0.0, nan
    val[8, 0] = inf
    val[9, 0] = -inf
    tok[10, :2], val[10, 0], val[10, 1] = 12, inf, -inf
    penalty[11, 1] = 3e38                      # taken twice it is infinite
    hist[11, 8:10] = hist[11, 0]
    T[12], x[12] = 0.0, -inf
    T[13], x[13, 0, h3], ok[13, 0, h3] = 0.0, nan, False
    s = dict(logits=x.to(torch.bfloat16) if half else x, temperature=T, penalty=penalty, history=hist,
             hist_len=torch.full((B,), H, dtype=torch.int32), n_prompt=torch.zeros(B, dtype=torch.int32), bias_tok=tok,
             bias_val=val, allowed=_words(ok))
    p = _run(s).double().cpu().numpy()
    for b in range(B):
        with np.errstate(invalid="ignore", over="ignore"):
            row = _row(s, ok, b, 0, np.float32)
            want = R.probs(row, float(T[b]), ok[b, 0].numpy())
        assert np.array_equal(np.isnan(p[b, 0]), np.isnan(want)), b
        assert np.isnan(want).any() == (b in (0, 3, 7, 8, 10)) and (want == 0).all() == (b in (4, 12)), b
        if T[b] == 0:
            assert np.array_equal(p[b, 0], want, equal_nan=True), b
            continue
        # x is rounded as the definition has it; a probability's error is that of its own x and of the
        # largest, so of tokens that have one (an x of -3e38 has none: its bound is the 2^-126)
        rel = 2.0 ** -24 * (3 * 2 * np.abs(row[want > 0]).max(initial=0.0) + V / 256 + 96)
        there = ~np.isnan(want)
        assert (np.abs(p[b, 0] - want)[there] <= rel * want[there] + 2.0 ** -126).all(), b


@pytest.mark.parametrize("lists", [False, True])
@pytest.mark.parametrize("V", [3000, 20011])
def test_temperatures_that_are_none(V, lists):
    """Below 0 or NaN: NaN for all allowed tokens, whatever the logits, 0 for the others."""
    s, ok = _random(4, 2, V, 30 if lists else 0, 5 if lists else 0, 3, T=[-1.0, float("nan"), -float("inf"), 0.7])
    s["logits"][0, 1] = -float("inf")
    ok[1, 0] = False
    s["allowed"] = _words(ok)
    p = _run(s).cpu()
    assert torch.equal(torch.isnan(p[:3]), ok[:3]) and (p[:3][~ok[:3]] == 0).all()
    only = {k: v[3:] for k, v in s.items()}
    _check(only, ok[3:], p[3:])
