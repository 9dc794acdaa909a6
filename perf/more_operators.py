"""Cases of the 4-bit cache and of the target's probabilities: new tokens quantised into the cache and read back,
listed rows read back, attention of new tokens over the cache, and logits made into the probabilities that draft
verification takes (penalties for repeated tokens, biases, grammar masks, temperature).

`own` false: plain torch in float32.  `own` true: the framework's entry points.

A cache row's channels go in groups of 16 with a scale each: an unsigned float of 5 exponent (bias 15) and 3 mantissa
bits, the group's largest magnitude over 6 rounded to nearest even (at most 10240).  A channel is held as a 4-bit
float (sign, 2 exponent bits, 1 mantissa bit; magnitudes 0 0.5 1 1.5 2 3 4 6), the quotient by the scale rounded to
nearest even; a byte holds an even channel in its low half and the next one in its high half.
"""
import math

import torch

own = False

DEV = "cuda"
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MAX_SCALE = 10240.0


# --------------------------------------------------------------------- cases
def listed():
    return [
        # one token of one chat joins a short cache: latency
        dict(name="cache token", op="cache", B=1, n=1, Hkv=4, D=64, L=128),
        # a chunk of long prompts joins, and the context so far is read back for the chunk's dense attention
        dict(name="cache chunk", op="cache", B=4, n=2048, Hkv=8, D=128, L=16384),
        # ragged prompts of a batch, written and read back whole; odd capacity
        dict(name="cache prompt", op="cache", B=8, n=8187, Hkv=8, D=128, L=8187),
        # a few rows of two chats
        dict(name="rows few", op="rows", B=2, m=37, Hkv=4, D=64, L=2048),
        # the rows that a selection kept of a served batch, by their numbers
        dict(name="rows batch", op="rows", B=32, m=2048, Hkv=8, D=128, L=16384),
        # a short chat, one new token: latency
        dict(name="attn small", op="attn", B=1, n=1, Hq=8, Hkv=2, D=64, L=512, sel=1.0),
        # ordinary decode step of a served batch, every second token gated to the global branch
        dict(name="attn serve", op="attn", B=32, n=1, Hq=32, Hkv=8, D=128, L=16384, sel=0.5),
        # one long document, odd length
        dict(name="attn long", op="attn", B=1, n=1, Hq=32, Hkv=8, D=128, L=262139, sel=1.0),
        # four drafts and the last accepted token of a large batch
        dict(name="attn drafts", op="attn", B=64, n=5, Hq=32, Hkv=8, D=128, L=8192, sel=1.0),
        # one KV head for all 16 query heads, half-size heads, drafts
        dict(name="attn mqa", op="attn", B=16, n=4, Hq=16, Hkv=1, D=64, L=32768, sel=0.5),
        # one chat, a small vocabulary: latency
        dict(name="probs one", op="probs", B=1, m1=1, V=32000, H=200, K=0, mask=False, half=False),
        # a served batch with drafts, long histories, biases and a grammar
        dict(name="probs batch", op="probs", B=48, m1=5, V=131072, H=4000, K=48, mask=True, half=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("cache", "rows", "attn", "attn", "probs"))
    if op == "probs":
        c = dict(op="probs", B=_log_int(rng, 1, 64), m1=rng.randint(1, 8), V=_log_int(rng, 1000, 262144),
                 H=_log_int(rng, 1, 8192), K=rng.choice((0, 1)) * _log_int(rng, 1, 300), mask=rng.random() < 0.6,
                 half=rng.random() < 0.5)
        while c["B"] * c["m1"] * c["V"] > 48 * 5 * 131072:
            c["B"] = max(1, c["B"] // 2)
        return c
    Hkv, D = rng.choice((1, 2, 4, 8, 16)), rng.choice((64, 128))
    if op == "attn":
        G = rng.choice((1, 2, 3, 4, 5, 8, 16))
        while Hkv * G > 64:
            G //= 2
        c = dict(op="attn", B=_log_int(rng, 1, 128), n=rng.randint(1, 8), Hq=Hkv * G, Hkv=Hkv, D=D,
                 L=_log_int(rng, 16, 262144), sel=round(rng.uniform(0.1, 1.0), 2))
        most = max(work(k)["flops"] for k in listed() if k["op"] == "attn")
        while work(c)["flops"] > most or c["B"] * c["L"] * c["Hkv"] * c["D"] > 2 ** 29:
            c["B"] = max(1, c["B"] // 2)
            c["L"] = max(16, c["L"] // 2)
        return c
    B, L = _log_int(rng, 1, 32), _log_int(rng, 16, 65536)
    if op == "cache":
        c = dict(op="cache", B=B, n=min(L, _log_int(rng, 1, 16384)), Hkv=Hkv, D=D, L=L)
        while c["B"] * c["L"] * c["Hkv"] * c["D"] > 2 ** 26:
            c["B"] = max(1, c["B"] // 2)
            c["Hkv"] = max(1, c["Hkv"] // 2)
        return c
    c = dict(op="rows", B=B, m=_log_int(rng, 1, 8192), Hkv=Hkv, D=D, L=L)
    while c["B"] * max(8 * c["m"], c["L"]) * c["Hkv"] * c["D"] > 2 ** 29:
        c["B"] = max(1, c["B"] // 2)
        c["Hkv"] = max(1, c["Hkv"] // 2)
    return c


# -------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _quantise(x):
    """[..., D] -> codes [..., D/2] uint8 and scales [..., D/16] uint8."""
    D = x.shape[-1]
    x = x.float().unflatten(-1, (D // 16, 16))
    s = x.abs().amax(-1) / 6
    step = torch.exp2(torch.frexp(s).exponent.clamp(min=-13).float() - 4)
    s = (torch.round(s / step) * step).clamp(max=MAX_SCALE)
    y = torch.where(s[..., None] > 0, x.abs() / s[..., None], 0.0)
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5))
    code = (code + 8 * (x < 0).to(torch.uint8)).flatten(-2)
    scale = (s.half().view(torch.int16) >> 7).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def _values(codes, scales):
    """The float32 values [..., D] that a cache's codes and scales stand for."""
    table = torch.tensor([*MAGNITUDES, *(-m for m in MAGNITUDES)], device=codes.device)
    pair = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    s = (scales.to(torch.int16) << 7).view(torch.float16).float()
    return (table[pair.int()].unflatten(-1, (scales.shape[-1], 16)) * s[..., None]).flatten(-2)


def _tokens(g, B, n, Hkv, D):
    """Keys with channels of different spread, as rotated keys have them, and values."""
    spread = torch.randn(Hkv, D, generator=g, device=DEV).mul_(0.5).exp_()
    k = torch.randn(B, n, Hkv, D, generator=g, device=DEV).mul_(spread)
    return k.to(torch.bfloat16), torch.randn(B, n, Hkv, D, generator=g, device=DEV, dtype=torch.bfloat16)


def _cache(g, B, L, Hkv, D):
    """A cache of L random rows a sequence: (k, v codes [B, Hkv, L, D/2], k, v scales [B, Hkv, L, D/16])."""
    out = [torch.empty(B, Hkv, L, w, dtype=torch.uint8, device=DEV) for w in (D // 2, D // 2, D // 16, D // 16)]
    some = max(1, 2 ** 24 // (L * Hkv * D))
    for b in range(0, B, some):
        for i, t in enumerate(_tokens(g, min(some, B - b), L, Hkv, D)):
            codes, scales = _quantise(t)
            out[i][b:b + some], out[2 + i][b:b + some] = codes.transpose(1, 2), scales.transpose(1, 2)
    return tuple(out)


def _prepare_cache(c, g):
    B, n, Hkv, D, L = (c[k] for k in ("B", "n", "Hkv", "D", "L"))
    s = dict(cache=_cache(g, B, L, Hkv, D))
    s["k"], s["v"] = _tokens(g, B, n, Hkv, D)
    # ragged: every sequence brings up to n tokens and then holds between that many and L
    s["n_valid"] = torch.randint(max(1, n // 2), n + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    s["n_valid"][0] = n
    s["seq_len"] = torch.maximum(s["n_valid"], torch.randint(max(1, 3 * L // 4), L + 1, (B,), generator=g, device=DEV, dtype=torch.int32))
    s["k_out"] = torch.zeros(B, L, Hkv, D, dtype=torch.bfloat16, device=DEV)
    s["v_out"] = torch.zeros_like(s["k_out"])
    return s


def _prepare_rows(c, g):
    B, m, Hkv, D, L = (c[k] for k in ("B", "m", "Hkv", "D", "L"))
    s = dict(cache=_cache(g, B, L, Hkv, D))
    s["seq_len"] = torch.randint(max(1, L // 2), L + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    # ascending rows, as a selection lists them, and a list that ends early for one sequence
    at = torch.rand(B, m, generator=g, device=DEV).sort(-1).values
    s["rows"] = (at * s["seq_len"][:, None]).int().clamp(max=L - 1)
    s["rows"][0, (m + 1) // 2:] = -1
    s["k_out"] = torch.zeros(B, m, Hkv, D, dtype=torch.bfloat16, device=DEV)
    s["v_out"] = torch.zeros_like(s["k_out"])
    return s


def _prepare_attn(c, g):
    B, n, Hq, Hkv, D, L = (c[k] for k in ("B", "n", "Hq", "Hkv", "D", "L"))
    s = dict(cache=_cache(g, B, L, Hkv, D))
    s["q"] = torch.randn(B, n, Hq, D, generator=g, device=DEV, dtype=torch.bfloat16)
    # ragged caches, one of them (of several) with the new tokens alone
    lens = torch.randint(max(min(n, L), L // 4), L + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    lens[0] = min(n, L) if B > 1 else L
    s["seq_len"] = lens
    # the gate's selection: a fixed number of the (B, n) tokens, packed in order
    N = _n_sel(c)
    z = torch.zeros(B * n, dtype=torch.bool, device=DEV)
    z[torch.randperm(B * n, generator=g, device=DEV)[:N]] = True
    z = z.view(B, n)
    count = z.sum(1)
    s["cu_q"] = torch.cat([count.new_zeros(1), count.cumsum(0)]).int()
    s["row_of"] = torch.where(z.view(-1), z.view(-1).cumsum(0) - 1, -1).view(B, n).int()
    s["pos"] = torch.zeros(B * n, dtype=torch.int32, device=DEV)
    s["pos"][:N] = z.nonzero()[:, 1].int()
    s["n_sel"] = s["cu_q"][-1:].clone()
    s["o_c"] = torch.zeros(B * n, Hq, D, dtype=torch.bfloat16, device=DEV)
    s["lse_c"] = torch.zeros(Hq, B * n, dtype=torch.float32, device=DEV)
    return s


def _prepare_probs(c, g):
    B, m1, V, H, K = (c[k] for k in ("B", "m1", "V", "H", "K"))
    ids = lambda *s: (torch.rand(s, generator=g, device=DEV).pow_(3) * V).int().clamp_(max=V - 1)  # noqa: E731
    s = dict(logits=torch.randn(B, m1, V, generator=g, device=DEV).mul_(2.5).add_(-3.0))
    if c["half"]:
        s["logits"] = s["logits"].to(torch.bfloat16)
    # frequent tokens come again and again; ragged histories, a prompt ahead of the generated tokens
    s["history"] = ids(B, H)
    s["hist_len"] = torch.randint((H + 1) // 2, H + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    s["n_prompt"] = s["hist_len"] // 3
    s["draft"] = ids(B, m1 - 1) if m1 > 1 else None
    # (repetition, frequency, presence) as users set them
    s["penalty"] = torch.tensor([1.1, 0.2, 0.4], device=DEV).repeat(B, 1)
    s["penalty"][0] = torch.tensor([1.0, 0.0, 0.0], device=DEV)
    s["temperature"] = torch.rand(B, generator=g, device=DEV) + 0.5
    if B > 2:  # one greedy sequence
        s["temperature"][1] = 0.0
    s["bias_tok"] = s["bias_val"] = s["allowed"] = None
    if K:
        s["bias_tok"] = ids(B, K)
        s["bias_tok"][0, K // 2:] = -1
        s["bias_val"] = torch.randn(B, K, generator=g, device=DEV).mul_(3.0)
    if c["mask"]:
        # rows that a grammar leaves a share of the vocabulary, and rows it leaves alone
        share = torch.rand(B, m1, 1, generator=g, device=DEV)
        share = torch.where(share < 0.5, 1.0, share - 0.4)
        words = (V + 31) // 32
        word = torch.zeros(B, m1, words, dtype=torch.int32, device=DEV)
        for bit in range(32):
            word |= (torch.rand(B, m1, words, generator=g, device=DEV) < share).int() << bit
        s["allowed"] = word
    s["p"] = torch.zeros(B, m1, V, device=DEV)
    return s


def prepare(case, seed):
    prep = dict(cache=_prepare_cache, rows=_prepare_rows, attn=_prepare_attn, probs=_prepare_probs)
    s = prep[case["op"]](case, _gen(seed))
    s["case"] = case
    s["ws"] = {}
    return s


# --------------------------------------------------------------- plain forms
def _plain_read(s, at):
    """Rows `at` [B, m] of the cache as bf16 [B, m, Hkv, D]; rows that hold no token as zeros."""
    held = (at >= 0) & (at < s["seq_len"][:, None])
    where = torch.where(held, at, 0).long()[:, None, :, None]
    kc, vc, ks, vs = s["cache"]
    for codes, scales, out in ((kc, ks, s["k_out"]), (vc, vs, s["v_out"])):
        codes = codes.gather(2, where.expand(-1, codes.shape[1], -1, codes.shape[3]))
        scales = scales.gather(2, where.expand(-1, scales.shape[1], -1, scales.shape[3]))
        x = torch.where(held[:, None, :, None], _values(codes, scales), 0.0)
        out.copy_(x.transpose(1, 2))
    return dict(k=s["k_out"], v=s["v_out"])


def _plain_cache(s):
    c = s["case"]
    B, n, L = c["B"], c["n"], c["L"]
    i = torch.arange(n, device=DEV)
    row = s["seq_len"][:, None].long() - s["n_valid"][:, None] + i
    new = (i < s["n_valid"][:, None]) & (row >= 0) & (row < L)
    b, i = new.nonzero(as_tuple=True)
    row = row[b, i]
    kc, vc, ks, vs = s["cache"]
    for x, codes, scales in ((s["k"], kc, ks), (s["v"], vc, vs)):
        codes[b, :, row], scales[b, :, row] = _quantise(x[b, i])
    return _plain_read(s, torch.arange(L, device=DEV).expand(B, L))


def _plain_rows(s):
    return _plain_read(s, s["rows"])


def _plain_attn(s):
    c = s["case"]
    B, n, Hq, Hkv, D, L = (c[k] for k in ("B", "n", "Hq", "Hkv", "D", "L"))
    G = Hq // Hkv
    kc, vc, ks, vs = s["cache"]
    q = s["q"].float().view(B, n, Hkv, G, D).transpose(1, 2).reshape(B, Hkv, n * G, D)
    slot = torch.arange(L, device=DEV)
    lens = s["seq_len"].long()
    x = (q @ _values(kc, ks).transpose(2, 3)).mul_(1.0 / math.sqrt(D)).view(B, Hkv, n, G, L)
    vis = torch.minimum(lens[:, None], (lens[:, None] - n + 1 + torch.arange(n, device=DEV)).clamp(min=0))
    x = torch.where((slot < vis[:, :, None])[:, None, :, None], x, -math.inf).view(B, Hkv, n * G, L)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = x.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    v = torch.where((slot < lens[:, None])[:, None, :, None], _values(vc, vs), 0.0)
    o = (e @ v) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log()).squeeze(-1)
    o = o.view(B, Hkv, n, G, D).transpose(1, 2).reshape(B * n, Hq, D).to(torch.bfloat16)
    lse = lse.view(B, Hkv, n, G).permute(1, 3, 0, 2).reshape(Hq, B * n)
    # packed rows: token t of the batch goes to row row_of[t]
    row = s["row_of"].view(-1).long()
    N = _n_sel(c)
    token = torch.zeros(B * n + 1, dtype=torch.long, device=DEV)
    token[torch.where(row >= 0, row, B * n)] = torch.arange(B * n, device=DEV)
    token = token[:N]
    s["o_c"][:N] = o[token]
    s["lse_c"][:, :N] = lse[:, token]
    return dict(o=s["o_c"], lse=s["lse_c"])


def _counts(s, real):
    """seen [B, m1, V] (in the history or among the drafts before row i) and how often a token was generated."""
    c = s["case"]
    B, m1, V, H = c["B"], c["m1"], c["V"], c["H"]
    ids, draft = s["history"], s["draft"]
    at = torch.arange(H + m1 - 1, device=DEV)
    if draft is not None:
        ids = torch.cat([ids, draft], 1)
    row = torch.arange(m1, device=DEV)[:, None]
    old = (at < H) & (at < s["hist_len"][:, None])
    drafted = (at >= H) & (at - H < row)  # [m1, H + m]
    there = old[:, None] | drafted
    made = (old & (at >= s["n_prompt"][:, None]))[:, None] | drafted
    ids = ids.long()[:, None].expand(-1, m1, -1)
    zero = torch.zeros(B, m1, V, dtype=real, device=DEV)
    return zero.scatter_add(2, ids, there.to(real)) > 0, zero.scatter_add(2, ids, made.to(real))


def _plain_probs(s):
    c = s["case"]
    B, m1, V = c["B"], c["m1"], c["V"]
    x = s["logits"].float()
    seen, count = _counts(s, torch.float32)
    rep, freq, pres = (s["penalty"][:, i].view(B, 1, 1) for i in range(3))
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = torch.where(count > 0, x - (count * freq + pres), x)
    if s["bias_tok"] is not None:
        ok = s["bias_tok"] >= 0
        bias = torch.zeros(B, V, device=DEV)
        bias.scatter_add_(1, s["bias_tok"].clamp(min=0).long(), torch.where(ok, s["bias_val"], 0.0))
        x = x + bias[:, None]
    if s["allowed"] is not None:
        v = torch.arange(V, device=DEV)
        bit = (s["allowed"][..., v // 32] >> (v % 32).int()) & 1
        x = torch.where(bit > 0, x, -math.inf)
    t = s["temperature"].view(B, 1, 1)
    x = torch.where(t > 0, x / torch.where(t > 0, t, 1.0), x)
    top = x.amax(-1, keepdim=True)
    none = top == -math.inf
    first = torch.zeros_like(x).scatter_(2, x.argmax(-1, keepdim=True), 1.0)
    e = (x - torch.where(none, 0.0, top)).exp_()
    p = torch.where(t > 0, e / torch.where(none, 1.0, e.sum(-1, keepdim=True)), first)
    s["p"].copy_(torch.where(none, 0.0, p))
    return dict(p=s["p"])


# ----------------------------------------------------------- framework calls
def _own_cache(s):
    from paper_2608_29539_gb300 import logo as L
    cache = L.Cache4(*s["cache"])
    L.logo_cache4_append(cache, s["k"], s["v"], s["seq_len"], n_valid=s["n_valid"])
    k, v = L.logo_cache4_read(cache, s["seq_len"], k=s["k_out"], v=s["v_out"])
    return dict(k=k, v=v)


def _own_rows(s):
    from paper_2608_29539_gb300 import logo as L
    k, v = L.logo_cache4_read(L.Cache4(*s["cache"]), s["seq_len"], rows=s["rows"], k=s["k_out"], v=s["v_out"])
    return dict(k=k, v=v)


def _own_attn(s):
    from paper_2608_29539_gb300 import logo as L
    cache = L.Cache4(*s["cache"])
    if "attn" not in s["ws"]:
        s["ws"]["attn"] = L.logo_decode_cache4_workspace(s["q"], cache)
    o, lse = L.logo_decode_cache4_attn(s["q"], cache, s["seq_len"], s["pos"], s["cu_q"], s["n_sel"], o_c=s["o_c"],
                                       lse_c=s["lse_c"], workspace=s["ws"]["attn"])
    return dict(o=o, lse=lse)


def _own_probs(s):
    from paper_2608_29539_gb300 import logo as L
    p = L.logo_target_probs(s["logits"], temperature=s["temperature"], penalty=s["penalty"], history=s["history"],
                            hist_len=s["hist_len"], n_prompt=s["n_prompt"], draft=s["draft"], bias_tok=s["bias_tok"],
                            bias_val=s["bias_val"], allowed=s["allowed"], p=s["p"])
    return dict(p=p)


def run(state):
    op = state["case"]["op"]
    if own:
        return dict(cache=_own_cache, rows=_own_rows, attn=_own_attn, probs=_own_probs)[op](state)
    return dict(cache=_plain_cache, rows=_plain_rows, attn=_plain_attn, probs=_plain_probs)[op](state)


# ---------------------------------------------------------------------- work
def _n_sel(c):
    return max(1, int(c["sel"] * c["B"] * c["n"]))


def work(case):
    c = case
    if c["op"] == "probs":
        B, m1, V = c["B"], c["m1"], c["V"]
        data = B * m1 * V * ((2 if c["half"] else 4) + 4 + (1 / 8 if c["mask"] else 0))
        return dict(bytes=data + B * (4 * 0.75 * c["H"] + 8 * c["K"]), flops=4 * B * m1 * V)
    B, Hkv, D, L = (c[k] for k in ("B", "Hkv", "D", "L"))
    packed = 2 * Hkv * (D // 2 + D // 16)  # bytes of a cache row, K and V
    if c["op"] == "cache":
        new = (c["n"] + (B - 1) * 0.75 * c["n"])
        length = B * max(0.875 * L, c["n"])
        return dict(bytes=new * (4 * Hkv * D + packed) + length * packed + B * L * 4 * Hkv * D, flops=0)
    if c["op"] == "rows":
        held = c["m"] * (B - 0.5)
        return dict(bytes=held * packed + B * c["m"] * (4 * Hkv * D + 4), flops=0)
    n, Hq, N = c["n"], c["Hq"], _n_sel(c)
    # tokens of a cache on average, all but one of them (of several) ragged
    length = L if B == 1 else ((B - 1) * (max(min(n, L), L // 4) + L) / 2 + min(n, L)) / B
    reached = B * (1 - (1 - N / (B * n)) ** n)  # sequences with a selected token, on average
    data = 4 * N * Hq * D + 4 * N * Hq + reached * length * packed
    return dict(bytes=data, flops=4 * D * Hq * N * max(1.0, length - (n - 1) / 2))


# --------------------------------------------------------------- definitions
def _exact_value(x):
    """What a cache holds for x [..., D], in 64 bits from the definition: the nearest of the representable scales
    and of the representable quotients, ties to the even one of the two."""
    D = x.shape[-1]
    x = x.double().unflatten(-1, (D // 16, 16))
    grid = [m * 2.0 ** -17 for m in range(8)] + [(8 + m) * 2.0 ** (e - 18) for e in range(1, 30) for m in range(8)]
    s = _nearest((x.abs().amax(-1) / 6), torch.tensor([v for v in grid if v <= MAX_SCALE], dtype=torch.float64, device=DEV))
    y = torch.where(s[..., None] > 0, x.abs() / s[..., None], torch.zeros_like(x))
    y = _nearest(y, torch.tensor(MAGNITUDES, dtype=torch.float64, device=DEV))
    return (torch.copysign(y, x) * s[..., None]).flatten(-2)


def _nearest(x, grid):
    hi = torch.bucketize(x, grid).clamp(1, len(grid) - 1)
    lo = hi - 1
    below, above = x - grid[lo], grid[hi] - x
    return grid[torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)]


def _held(s, b, h, rows):
    """The values of rows of one sequence and KV head in 64 bits: (k, v)."""
    kc, vc, ks, vs = s["cache"]
    out = []
    for codes, scales in ((kc, ks), (vc, vs)):
        byte, sc = codes[b, h, rows].long(), scales[b, h, rows].long()
        nibble = torch.stack([byte % 16, byte // 16], -1).flatten(-2)
        e, m = (nibble // 2) % 4, (nibble % 2).double()
        mag = torch.where(e == 0, 0.5 * m, torch.ldexp(1 + 0.5 * m, (e - 1).double()))
        mag = torch.where(nibble >= 8, -mag, mag)
        e, m = sc // 8, (sc % 8).double()
        scale = torch.where(e == 0, m * 2.0 ** -17, torch.ldexp(8 + m, (e - 18).double()))
        out.append(mag * scale.repeat_interleave(16, -1))
    return out


def _exact_attn(c, s):
    B, n, Hq, Hkv, D, L = (c[k] for k in ("B", "n", "Hq", "Hkv", "D", "L"))
    G = Hq // Hkv
    o = torch.zeros(B * n, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(Hq, B * n, dtype=torch.float64, device=DEV)
    lens, cu, pos = s["seq_len"].tolist(), s["cu_q"].tolist(), s["pos"].tolist()
    for b in range(B):
        for h in range(Hkv if cu[b] < cu[b + 1] else 0):
            k, v = _held(s, b, h, slice(0, lens[b]))
            for r in range(cu[b], cu[b + 1]):
                seen = max(0, lens[b] - n + pos[r] + 1)
                heads = slice(h * G, (h + 1) * G)
                x = s["q"][b, pos[r], heads].double() @ k[:seen].T / math.sqrt(D)
                lse[heads, r] = torch.logsumexp(x, 1) if seen else -math.inf
                o[r, heads] = torch.softmax(x, 1) @ v[:seen]
    return dict(o=o, lse=lse)


def _exact_probs(c, s):
    B, m1, V, H = (c[k] for k in ("B", "m1", "V", "H"))
    p = torch.zeros(B, m1, V, dtype=torch.float64, device=DEV)
    hist, length, prompt = s["history"].long(), s["hist_len"].tolist(), s["n_prompt"].tolist()
    for b in range(B):
        rep, freq, pres = s["penalty"][b].double()
        for i in range(m1):
            x = s["logits"][b, i].double()
            new = s["draft"][b, :i].long() if i else hist[b, :0]
            past = torch.cat([hist[b, :length[b]], new])
            count = torch.bincount(torch.cat([hist[b, prompt[b]:length[b]], new]), minlength=V).double()
            x[past] = torch.where(x > 0, x / rep, x * rep)[past]
            x = torch.where(count > 0, x - freq * count - pres, x)
            if s["bias_tok"] is not None:
                ok = s["bias_tok"][b] >= 0
                x.index_put_((s["bias_tok"][b][ok].long(),), s["bias_val"][b][ok].double(), accumulate=True)
            if s["allowed"] is not None:
                bits = (s["allowed"][b, i].long()[:, None] >> torch.arange(32, device=DEV)) & 1
                x[bits.flatten()[:V] == 0] = -math.inf
            if float(x.max()) == -math.inf:
                continue
            t = float(s["temperature"][b])
            if t > 0:
                p[b, i] = torch.softmax(x / t, 0)
            else:
                p[b, i, int((x == x.max()).nonzero()[0])] = 1.0
    return dict(p=p)


def _exact_read(s, rows):
    """rows: per sequence the list of rows, negative for none."""
    k, v = (torch.zeros(s["k_out"].shape, dtype=torch.float64, device=DEV) for _ in range(2))
    for b, at in enumerate(rows):
        at = torch.tensor(at, device=DEV)
        there = (at >= 0) & (at < int(s["seq_len"][b]))
        for h in range(k.shape[2]):
            k[b, there, h], v[b, there, h] = _held(s, b, h, at[there])
    return dict(k=k, v=v)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rows":
        return _exact_read(s, s["rows"].tolist())
    if case["op"] == "cache":
        out = _exact_read(s, [range(case["L"])] * case["B"])
        for b, (length, n) in enumerate(zip(s["seq_len"].tolist(), s["n_valid"].tolist())):
            for name in ("k", "v"):
                out[name][b, length - n:length] = _exact_value(s[name][b, :n])
        return out
    if case["op"] == "probs":
        return _exact_probs(case, s) if case["B"] * case["m1"] <= 512 else None
    if 4 * case["D"] * case["Hq"] * _n_sel(case) * case["L"] > 1e12 or _n_sel(case) * case["Hkv"] > 8192:
        return None
    return _exact_attn(case, s)
