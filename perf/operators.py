"""Cases of the serving operators: attention of drafted tokens over a shared prefix and each sequence's own
cache (with the accumulated attention weights), eviction from the caches by those weights, and verification of
drafted tokens against the target's probabilities.

`own` false: plain torch in float32.  `own` true: the framework's entry points.
"""
import math

import torch

own = False

DEV = "cuda"


# --------------------------------------------------------------------- cases
def listed():
    return [
        # a short system prompt shared by two chats, one new token each: latency
        dict(name="attn small", op="attn", B=2, n=1, Hq=4, Hkv=4, D=64, P=512, L=64, sel=1.0, mass=False),
        # ordinary decode step of a served batch, every second token gated to the global branch, weights kept
        dict(name="attn serve", op="attn", B=32, n=1, Hq=32, Hkv=8, D=128, P=16384, L=2048, sel=0.5, mass=True),
        # drafted tokens verified in one call: four drafts and the last accepted token, odd prefix
        dict(name="attn drafts", op="attn", B=32, n=5, Hq=32, Hkv=8, D=128, P=32749, L=1024, sel=0.5, mass=True),
        # large batch of drafts over a long shared document: bound by the tensor cores
        dict(name="attn large", op="attn", B=128, n=4, Hq=32, Hkv=8, D=128, P=65536, L=1024, sel=1.0, mass=False),
        # one KV head per query head, long own caches behind a short odd prefix: bound by HBM
        dict(name="attn own", op="attn", B=8, n=1, Hq=16, Hkv=16, D=128, P=1000, L=16384, sel=1.0, mass=True),
        # one KV head for all 16 query heads, half-size heads, eight new tokens
        dict(name="attn mqa", op="attn", B=16, n=8, Hq=16, Hkv=1, D=64, P=32768, L=4096, sel=0.5, mass=True),
        # small cache of one sequence halved: latency
        dict(name="evict small", op="evict", B=1, Hkv=4, D=64, L=512, budget=256, recent=32, fresh=False),
        # every step of a served batch: as many slots leave as drafted tokens came
        dict(name="evict step", op="evict", B=32, Hkv=8, D=128, L=2056, budget=2048, recent=256, fresh=False),
        # once after a long prompt: an eighth of the cache stays
        dict(name="evict prompt", op="evict", B=8, Hkv=8, D=128, L=16384, budget=2048, recent=512, fresh=True),
        # one sequence, a small vocabulary: latency
        dict(name="verify one", op="verify", B=1, m=4, V=32000, good=0.8),
        # a served batch
        dict(name="verify serve", op="verify", B=32, m=4, V=131072, good=0.8),
        # many sequences, more drafts, odd vocabulary
        dict(name="verify large", op="verify", B=256, m=7, V=50021, good=0.6),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attn", "attn", "evict", "verify"))
    if op == "attn":
        Hkv = rng.choice((1, 2, 4, 8, 16))
        G = rng.choice((1, 2, 3, 4, 8, 16))
        while Hkv * G > 64:
            G //= 2
        n = rng.randint(1, 8)
        c = dict(op="attn", B=_log_int(rng, 1, 128), n=n, Hq=Hkv * G, Hkv=Hkv, D=rng.choice((64, 128)),
                 P=rng.choice((0, 1, 1, 1)) * _log_int(rng, 1, 65536), L=_log_int(rng, 16, 16384),
                 sel=round(rng.uniform(0.1, 1.0), 2), mass=rng.random() < 0.6)
        big = listed()[3]
        while work(c)["flops"] > work(big)["flops"] or c["B"] * c["L"] * c["Hkv"] * c["D"] > 2 ** 29:
            c["B"] = max(1, c["B"] // 2)
            c["P"] //= 2
            c["L"] = max(16, c["L"] // 2)
        return c
    if op == "evict":
        L = _log_int(rng, 32, 16384)
        budget = rng.randint(max(1, L // 16), L)
        c = dict(op="evict", B=_log_int(rng, 1, 64), Hkv=rng.choice((1, 2, 4, 8, 16)), D=rng.choice((64, 128)), L=L,
                 budget=budget, recent=rng.randint(0, min(budget, 512)), fresh=rng.random() < 0.5)
        while c["B"] * c["L"] * c["Hkv"] * c["D"] > 2 ** 27:
            c["B"] = max(1, c["B"] // 2)
            c["Hkv"] = max(1, c["Hkv"] // 2)
        return c
    c = dict(op="verify", B=_log_int(rng, 1, 256), m=rng.randint(1, 8), V=_log_int(rng, 1000, 131072),
             good=round(rng.uniform(0.1, 1.0), 2))
    while c["B"] * c["m"] * c["V"] > 2 ** 26:
        c["B"] = max(1, c["B"] // 2)
    return c


# -------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _prepare_attn(c, g):
    B, n, Hq, Hkv, D, P, L = (c[k] for k in ("B", "n", "Hq", "Hkv", "D", "P", "L"))
    bf = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=torch.bfloat16)  # noqa: E731
    s = dict(q=bf(B, n, Hq, D), kp=bf(P, Hkv, D), vp=bf(P, Hkv, D), kc=bf(B, L, Hkv, D), vc=bf(B, L, Hkv, D))
    # ragged caches, the first one with the new tokens alone
    lens = torch.randint(min(n, L), L + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    lens[0] = min(n, L)
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
    s["mass_in"] = s["mass_out"] = None
    if c["mass"]:
        # what about ten earlier steps have left: an even share of each row's weight a step
        share = 10 * (Hq // Hkv) * N / B / (P + L / 2 + 1)
        s["mass_in"] = torch.empty(B, Hkv, L, device=DEV).exponential_(1.0, generator=g).mul_(share)
        s["mass_out"] = torch.zeros(B, Hkv, L, device=DEV)
    return s


def _prepare_evict(c, g):
    B, Hkv, D, L = (c[k] for k in ("B", "Hkv", "D", "L"))
    bf = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=torch.bfloat16)  # noqa: E731
    s = dict(kc=bf(B, L, Hkv, D), vc=bf(B, L, Hkv, D))
    # heavy-tailed weights; a few slots share the value 0 (tokens that nothing has attended yet)
    mass = torch.randn(B, Hkv, L, generator=g, device=DEV).mul_(1.5).exp_()
    mass[torch.rand(B, Hkv, L, generator=g, device=DEV) < 0.02] = 0.0
    s["mass"] = mass
    lens = torch.full((B,), L, dtype=torch.int32, device=DEV)
    if B > 1:  # one sequence still below its budget
        lens[0] = min(L, max(1, c["budget"] - 1))
    s["seq_len"] = lens
    if c["fresh"]:  # straight after the prompt: slot s holds position s
        s["slot_pos"] = torch.arange(L, device=DEV, dtype=torch.int32).expand(B, Hkv, L).contiguous()
        s["n_seen"] = lens.clone()
    else:  # in the steady state: L distinct positions out of 2 L, in any order, the latest ones among them
        order = torch.rand(B, Hkv, L, generator=g, device=DEV).argsort(-1)
        s["slot_pos"] = (2 * order + 1).int()
        s["n_seen"] = torch.full((B,), 2 * L, dtype=torch.int32, device=DEV)
    s["mass_out"] = torch.zeros_like(mass)
    s["slot_pos_out"] = torch.zeros_like(s["slot_pos"])
    s["new_len"] = torch.zeros_like(lens)
    return s


def _prepare_verify(c, g):
    B, m, V = c["B"], c["m"], c["V"]
    # the target's probabilities are peaked; the draft's are near them for a share `good` of the drafts
    z = torch.randn(B, m + 1, V, generator=g, device=DEV).mul_(2.0)
    p = torch.softmax(z, -1)
    far = torch.rand(B, m, 1, generator=g, device=DEV) >= c["good"]
    zq = z[:, :m] + torch.where(far, 2.0, 0.1) * torch.randn(B, m, V, generator=g, device=DEV)
    q = torch.softmax(zq, -1)
    draft = torch.multinomial(q.view(B * m, V), 1, generator=g).view(B, m).int()
    u = torch.rand(B, m, generator=g, device=DEV)
    e = torch.empty(B, V, device=DEV).exponential_(1.0, generator=g)
    draft_len = torch.full((B,), m, dtype=torch.int32, device=DEV)
    if B > 1:  # one sequence for which fewer tokens were drafted
        draft_len[0] = m // 2
    return dict(draft=draft, q=q, p=p, u=u, e=e, draft_len=draft_len,
                tokens=torch.zeros(B, m + 1, dtype=torch.int32, device=DEV),
                n_accept=torch.zeros(B, dtype=torch.int32, device=DEV))


def prepare(case, seed):
    g = _gen(seed)
    s = {"attn": _prepare_attn, "evict": _prepare_evict, "verify": _prepare_verify}[case["op"]](case, g)
    s["case"] = case
    s["ws"] = {}
    return s


# --------------------------------------------------------------- plain forms
def _plain_attn(s):
    c = s["case"]
    B, n, Hq, Hkv, D, P, L = (c[k] for k in ("B", "n", "Hq", "Hkv", "D", "P", "L"))
    G = Hq // Hkv
    q = s["q"].float().view(B, n, Hkv, G, D).permute(2, 0, 1, 3, 4)  # [Hkv, B, n, G, D]
    kp = s["kp"].float().permute(1, 2, 0)  # [Hkv, D, P]
    vp = s["vp"].float().permute(1, 0, 2)
    kc = s["kc"].float().permute(2, 0, 3, 1)  # [Hkv, B, D, L]
    slot = torch.arange(L, device=DEV)
    lens = s["seq_len"].long()
    inside = slot < lens[:, None]  # [B, L]
    vc = torch.where(inside[:, :, None, None], s["vc"].float(), 0.0).permute(2, 0, 1, 3)
    scale = 1.0 / math.sqrt(D)
    xp = (q.reshape(Hkv, B * n * G, D) @ kp).mul_(scale).view(Hkv, B, n * G, P)
    xc = (q.reshape(Hkv, B, n * G, D) @ kc).mul_(scale).view(Hkv, B, n, G, L)
    vis = (lens[:, None] - n + 1 + torch.arange(n, device=DEV)).clamp(min=0)  # [B, n]
    seen = inside[:, None] & (slot < vis[:, :, None])  # [B, n, L]
    xc = torch.where(seen[None, :, :, None], xc, -math.inf).view(Hkv, B, n * G, L)
    top = xc.amax(-1, keepdim=True)
    if P:
        top = torch.maximum(top, xp.amax(-1, keepdim=True))
    top = torch.where(top == -math.inf, 0.0, top)
    ep, ec = xp.sub_(top).exp_(), (xc - top).exp_()
    total = ep.sum(-1, keepdim=True) + ec.sum(-1, keepdim=True)
    o = (ep.view(Hkv, B * n * G, P) @ vp).view(Hkv, B, n * G, D) + ec @ vc
    o = o / torch.where(total > 0, total, 1.0)
    lse = top + total.log()
    o = o.view(Hkv, B * n, G, D).permute(1, 0, 2, 3).reshape(B * n, Hq, D).to(torch.bfloat16)
    lse = lse.view(Hkv, B * n, G).permute(0, 2, 1).reshape(Hq, B * n)
    # packed rows: token t of the batch goes to row row_of[t]
    row = s["row_of"].view(-1).long()
    chosen = row >= 0
    N = _n_sel(c)
    token = torch.zeros(B * n + 1, dtype=torch.long, device=DEV)
    token[torch.where(chosen, row, B * n)] = torch.arange(B * n, device=DEV)
    token = token[:N]
    s["o_c"][:N] = o[token]
    s["lse_c"][:, :N] = lse[:, token]
    out = dict(o=s["o_c"], lse=s["lse_c"])
    if s["mass_in"] is not None:
        w = ec / torch.where(total > 0, total, 1.0) * chosen.view(1, B, n, 1).expand(Hkv, B, n, G).reshape(Hkv, B, n * G, 1)
        add = w.sum(2).permute(1, 0, 2)  # [B, Hkv, L]
        old = torch.where((slot < lens[:, None] - n)[:, None], s["mass_in"], 0.0)
        s["mass_out"].copy_(torch.where(inside[:, None], old + add, s["mass_out"]))
        out["mass"] = s["mass_out"]
    return out


def _plain_evict(s):
    c = s["case"]
    L, n = c["L"], c["budget"]
    slot = torch.arange(L, device=DEV)
    lens = s["seq_len"].long()[:, None, None]
    new_len = lens.clamp(max=n)
    kept_first = s["slot_pos"] >= s["n_seen"][:, None, None] - c["recent"]
    key = torch.where(kept_first, math.inf, s["mass"])
    key = torch.where(slot < lens, key, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, slot.expand_as(order).contiguous())
    keep = rank < new_len
    hole = ~keep & (slot < new_len)
    late = keep & (slot >= new_len)
    # i-th kept slot at or above new_len, for every i
    late_of = torch.zeros(*keep.shape[:2], L + 1, dtype=torch.long, device=DEV)
    late_of.scatter_(-1, torch.where(late, late.cumsum(-1) - 1, L), slot.expand_as(order).contiguous())
    src = torch.where(hole, late_of.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), slot)
    rows = src.permute(0, 2, 1)[..., None].expand_as(s["kc"])
    s["kc"].copy_(s["kc"].gather(1, rows))
    s["vc"].copy_(s["vc"].gather(1, rows))
    inside = slot < new_len
    s["mass_out"].copy_(torch.where(inside, s["mass"].gather(-1, src), s["mass_out"]))
    s["slot_pos_out"].copy_(torch.where(inside, s["slot_pos"].gather(-1, src), s["slot_pos_out"]))
    s["new_len"].copy_(new_len.view(-1))
    return dict(k=s["kc"], v=s["vc"], mass=s["mass_out"], slot_pos=s["slot_pos_out"], new_len=s["new_len"])


def _plain_verify(s):
    c = s["case"]
    B, m = c["B"], c["m"]
    d = s["draft"].long()[..., None]
    pd, qd = s["p"][:, :m].gather(-1, d)[..., 0], s["q"].gather(-1, d)[..., 0]
    step = torch.arange(m, device=DEV)
    ok = (pd > 0) & (s["u"] * qd <= pd) & (step < s["draft_len"][:, None])
    a = ok.long().cumprod(1).sum(1)  # accepted
    batch = torch.arange(B, device=DEV)
    p = s["p"][batch, a]
    q = s["q"][batch, a.clamp(max=m - 1)]
    rejected = (a < s["draft_len"])[:, None]
    r = torch.where(rejected, (p - q).clamp(min=0), p)
    r = torch.where((r > 0).any(1, keepdim=True), r, p)
    token = torch.where(r > 0, r / s["e"], 0.0).argmax(1)
    at = torch.arange(m + 1, device=DEV)
    tokens = torch.where(at < a[:, None], torch.cat([s["draft"], s["draft"][:, :1]], 1), -1)
    tokens[batch, a] = token.int()
    s["tokens"].copy_(tokens)
    s["n_accept"].copy_(a)
    return dict(tokens=s["tokens"], n_accept=s["n_accept"])


# ----------------------------------------------------------- framework calls
def _own_attn(s):
    from paper_2608_29539_gb300 import logo as L
    if "attn" not in s["ws"]:
        s["ws"]["attn"] = L.logo_decode_prefix_workspace(s["q"], s["kp"], s["kc"], s["mass_in"] is not None)
    o, lse, mass = L.logo_decode_prefix_attn(s["q"], s["kp"], s["vp"], s["kc"], s["vc"], s["seq_len"], s["pos"],
                                             s["cu_q"], s["n_sel"], mass_in=s["mass_in"], mass_out=s["mass_out"],
                                             o_c=s["o_c"], lse_c=s["lse_c"], workspace=s["ws"]["attn"])
    return dict(o=o, lse=lse) if mass is None else dict(o=o, lse=lse, mass=mass)


def _own_evict(s):
    from paper_2608_29539_gb300 import logo as L
    c = s["case"]
    if "evict" not in s["ws"]:
        s["ws"]["evict"] = L.logo_cache_evict_workspace(s["kc"])
    mass, slot_pos, new_len = L.logo_cache_evict(s["kc"], s["vc"], s["mass"], s["slot_pos"], s["seq_len"], s["n_seen"],
                                                 c["budget"], c["recent"], mass_out=s["mass_out"],
                                                 slot_pos_out=s["slot_pos_out"], new_len=s["new_len"],
                                                 workspace=s["ws"]["evict"])
    return dict(k=s["kc"], v=s["vc"], mass=mass, slot_pos=slot_pos, new_len=new_len)


def _own_verify(s):
    from paper_2608_29539_gb300 import logo as L
    if "verify" not in s["ws"]:
        s["ws"]["verify"] = L.logo_verify_draft_workspace(s["p"])
    tokens, n_accept = L.logo_verify_draft(s["draft"], s["q"], s["p"], s["u"], s["e"], draft_len=s["draft_len"],
                                           tokens=s["tokens"], n_accept=s["n_accept"], workspace=s["ws"]["verify"])
    return dict(tokens=tokens, n_accept=n_accept)


def run(state):
    op = state["case"]["op"]
    if own:
        return {"attn": _own_attn, "evict": _own_evict, "verify": _own_verify}[op](state)
    return {"attn": _plain_attn, "evict": _plain_evict, "verify": _plain_verify}[op](state)


# ---------------------------------------------------------------------- work
def _n_sel(c):
    return max(1, int(c["sel"] * c["B"] * c["n"]))


def work(case):
    c = case
    if c["op"] == "attn":
        B, n, Hq, Hkv, D, P, L = (c[k] for k in ("B", "n", "Hq", "Hkv", "D", "P", "L"))
        N = _n_sel(c)
        length = (min(n, L) + L) / 2  # tokens of a cache, on average
        reached = B * (1 - (1 - N / (B * n)) ** n)  # sequences with a selected token, on average
        data = 4 * N * Hq * D + 4 * N * Hq + 4 * P * Hkv * D + 4 * reached * length * Hkv * D
        if c["mass"]:
            data += 8 * B * Hkv * length
        return dict(bytes=data, flops=4 * D * Hq * N * (P + max(1.0, length - (n - 1) / 2)))
    if c["op"] == "evict":
        B, Hkv, D, L, n, w = (c[k] for k in ("B", "Hkv", "D", "L", "budget", "recent"))
        over = L - n  # slots at or above the budget
        full = B if B == 1 else B - 1  # sequences that are over it
        if c["fresh"]:  # the latest ones all lie at the end
            moved = over if w >= over else w + (n - w) / max(1, L - w) * (over - w)
        else:
            moved = over * n / L
        if over <= 0:
            moved = 0
        return dict(bytes=B * Hkv * (8 * L + 8 * n) + full * Hkv * moved * 8 * D, flops=0)
    B, V = c["B"], c["V"]
    return dict(bytes=4 * B * V * 3, flops=2 * B * V)


# --------------------------------------------------------------- definitions
def _exact_attn(c, s):
    B, n, Hq, Hkv, D, P, L = (c[k] for k in ("B", "n", "Hq", "Hkv", "D", "P", "L"))
    G = Hq // Hkv
    o = torch.zeros(B * n, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(Hq, B * n, dtype=torch.float64, device=DEV)
    mass = torch.zeros(B, Hkv, L, dtype=torch.float64, device=DEV) if c["mass"] else None
    lens, cu, pos = s["seq_len"].tolist(), s["cu_q"].tolist(), s["pos"].tolist()
    for h in range(Hkv):
        kp, vp = s["kp"][:, h].double(), s["vp"][:, h].double()
        for b in range(B):
            m = lens[b]
            k = torch.cat([kp, s["kc"][b, :m, h].double()])
            v = torch.cat([vp, s["vc"][b, :m, h].double()])
            if mass is not None:
                mass[b, h, :max(0, m - n)] = s["mass_in"][b, h, :max(0, m - n)].double()
            for r in range(cu[b], cu[b + 1]):
                seen = P + min(m, max(0, m - n + pos[r] + 1))
                x = s["q"][b, pos[r], h * G:(h + 1) * G].double() @ k[:seen].T / math.sqrt(D)
                lse[h * G:(h + 1) * G, r] = torch.logsumexp(x, 1) if seen else -math.inf
                w = torch.softmax(x, 1)
                o[r, h * G:(h + 1) * G] = w @ v[:seen]
                if mass is not None:
                    mass[b, h, :seen - P] += w[:, P:].sum(0)
    return dict(o=o, lse=lse) if mass is None else dict(o=o, lse=lse, mass=mass)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attn":
        # one pass over the keys in 64 bits for every row and KV head
        if 4 * case["D"] * case["Hq"] * _n_sel(case) * (case["P"] + case["L"]) > 1e12 or _n_sel(case) * case["Hkv"] > 8192:
            return None
        return _exact_attn(case, s)
    if case["op"] == "evict":
        B, Hkv, n, w = (case[k] for k in ("B", "Hkv", "budget", "recent"))
        if B * Hkv * case["L"] > 2 ** 20:
            return None
        mass = s["mass"].double().cpu()
        out = s["mass_out"].double().cpu()
        lens, pos, seen = s["seq_len"].tolist(), s["slot_pos"].cpu().tolist(), s["n_seen"].tolist()
        for b in range(B):
            for h in range(Hkv):
                m = mass[b, h].tolist()
                by_worth = sorted(range(lens[b]), key=lambda i: (pos[b][h][i] < seen[b] - w, -m[i] if pos[b][h][i] < seen[b] - w else 0, i))
                kept = sorted(by_worth[:n])
                end = len(kept)
                late = (i for i in kept if i >= end)
                low = {i for i in kept if i < end}
                if end:
                    out[b, h, :end] = torch.tensor([m[i if i in low else next(late)] for i in range(end)]).double()
        return dict(k=None, v=None, mass=out, slot_pos=None, new_len=None)
    return None
