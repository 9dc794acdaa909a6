"""ServeBatch4: prompts in chunks, steps of drafted tokens, verification from logits with
penalties and grammars, against plain bookkeeping and the definitions in 64 bits; and the
same steps as a captured graph."""
import numpy as np
import pytest
import torch

import cache4_ref as C
import serving_ref as R

pytestmark = pytest.mark.gpu


def _inputs(g, B, n_new, Hq, Hkv, D, V, H, dev="cpu"):
    bf = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)  # noqa: E731
    m = n_new - 1
    x = dict(q=bf(B, n_new, Hq, D), k=bf(B, n_new, Hkv, D), v=bf(B, n_new, Hkv, D), gate=torch.rand((B, n_new), generator=g),
             draft=torch.randint(0, V, (B, m), generator=g).int(), qd=torch.softmax(torch.randn((B, m, V), generator=g), -1),
             logits=torch.randn((B, n_new, V), generator=g) * 2, u=torch.rand((B, m), generator=g),
             e=torch.empty((B, V)).exponential_(1.0, generator=g),
             history=torch.randint(0, V, (B, H), generator=g).int(), hist_len=torch.randint(0, H + 1, (B,), generator=g).int(),
             penalty=torch.tensor([[1.2, 0.1, 0.2]]).repeat(B, 1), temperature=torch.rand(B, generator=g) + 0.5,
             allowed=torch.randint(-2 ** 31, 2 ** 31 - 1, (B, n_new, (V + 31) // 32), generator=g).int())
    return {k: v.to(dev) for k, v in x.items()}


SAMPLING = ("history", "hist_len", "penalty", "temperature", "allowed")


def _step(batch, x):
    o = batch.step(x["q"], x["k"], x["v"], x["gate"])
    return o, batch.verify(x["draft"], x["qd"], x["logits"], x["u"], x["e"], **{k: x[k] for k in SAMPLING})


@pytest.mark.parametrize("D,Hq,Hkv,n_new", [(128, 8, 2, 3), (64, 4, 4, 1), (64, 12, 1, 4)])
def test_prompts_steps_and_verification(D, Hq, Hkv, n_new):
    from paper_2608_29539_gb300 import logo as Lg
    from paper_2608_29539_gb300.serve import Serve4Config, ServeBatch4
    B, rows, V, H, steps = 3, 150, 50, 12, 8
    G = Hq // Hkv
    g = torch.Generator().manual_seed(D + n_new)
    batch = ServeBatch4(Serve4Config(B, n_new, Hq, Hkv, D, rows))
    held = [[[] for _ in range(B)] for _ in range(2)]  # per sequence the rows [Hkv, D] that K (V) holds, in 64 bits
    for n, valid in ((60, [60, 1, 33]), (17, None)):
        k, v = (torch.randn((B, n, Hkv, D), generator=g).to(torch.bfloat16) for _ in range(2))
        batch.fill(k.cuda(), v.cuda(), None if valid is None else torch.tensor(valid, dtype=torch.int32, device="cuda"))
        for x, rows_of in zip((k, v), held):
            y = C.values(*C.quantise(x))
            for b in range(B):
                rows_of[b] += list(y[b, :n if valid is None else valid[b]])
    ck, cv = batch.context(90)
    for got, rows_of in zip((ck, cv), held):
        for b in range(B):
            n = min(90, len(rows_of[b]))
            assert torch.equal(got[b, :n].double().cpu(), torch.stack(rows_of[b])[:n]) and (got[b, n:] == 0).all()
    for _ in range(steps):
        x = _inputs(g, B, n_new, Hq, Hkv, D, V, H)
        (o_c, z, row_of), (tokens, n_acc) = _step(batch, {k: v.cuda() for k, v in x.items()})
        torch.cuda.synchronize()
        assert Lg.logo_get_device_status() == 0
        want_z = x["gate"] > 0.5
        assert torch.equal(z.cpu().bool(), want_z)
        for t, rows_of in zip((x["k"], x["v"]), held):
            y = C.values(*C.quantise(t))
            for b in range(B):
                rows_of[b] += list(y[b])
        rows = [(b, i) for b in range(B) for i in range(n_new) if want_z[b, i]]
        for r, (b, i) in enumerate(rows):
            vis = len(held[0][b]) - n_new + i + 1
            k, v = (torch.stack(h[b][:vis]) for h in held)
            for h in range(Hkv):
                w = torch.softmax(x["q"][b, i, h * G:(h + 1) * G].double() @ k[:, h].T / D ** 0.5, 1)
                o, absv = w @ v[:, h], w @ v[:, h].abs()
                got = o_c[r, h * G:(h + 1) * G].double().cpu()
                # one rounding of the output to bf16, weights to fp16, fp32 sums
                assert ((got - o).abs() <= 2.0 ** -8 * o.abs() + 2.0 ** -10 * absv).all()
        # the verdict follows the definition on probabilities that differ from it by float32's rounding:
        # the same unless a draw is as near a border as that
        p = np.zeros((B, n_new, V))
        for b in range(B):
            for i in range(n_new):
                bits = (x["allowed"][b, i].long()[:, None] >> torch.arange(32)) & 1
                ok = bits.flatten()[:V].bool().numpy()
                adj = C.adjusted(x["logits"][b, i].numpy(), x["penalty"][b].numpy(), x["history"][b, :int(x["hist_len"][b])].tolist(),
                                 0, x["draft"][b, :i].tolist(), (), ok)
                p[b, i] = C.probs(adj, float(x["temperature"][b]), ok)
        if n_new > 1:
            want_t, want_n = R.verify(x["draft"].numpy(), x["qd"].numpy(), p.astype(np.float32), x["u"].numpy(), x["e"].numpy(),
                                      [n_new - 1] * B)
            assert np.array_equal(tokens.cpu().numpy(), want_t) and n_acc.tolist() == want_n.tolist()
            for b in range(B):
                drop = n_new - 1 - int(want_n[b])
                for rows_of in held:
                    if drop:
                        del rows_of[b][-drop:]
        else:
            want = [int(np.argmax(np.where(p[b, 0] > 0, p[b, 0] / x["e"][b].numpy(), -1))) for b in range(B)]
            assert tokens[:, 0].tolist() == want
        assert batch.seq_len.tolist() == [len(r) for r in held[0]]


@pytest.mark.parametrize("n_new", [1, 3])
def test_replays_of_a_captured_step(n_new):
    """Bit for bit the steps called one by one, until the caches are full and past that."""
    from paper_2608_29539_gb300.serve import Serve4Config, ServeBatch4
    B, Hq, Hkv, D, V, H, rows = 3, 8, 2, 64, 40, 9, 30
    g = torch.Generator().manual_seed(n_new)
    plain, captured = (ServeBatch4(Serve4Config(B, n_new, Hq, Hkv, D, rows)) for _ in range(2))
    x = _inputs(g, B, n_new, Hq, Hkv, D, V, H, "cuda")
    for batch in (plain, captured):  # (also a graph's warm-up)
        _step(batch, x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(captured, x)
    plain._captured = True  # (it is not to refuse either)
    for i in range(40):
        for name, t in _inputs(g, B, n_new, Hq, Hkv, D, V, H, "cuda").items():
            x[name].copy_(t)
        want = _step(plain, x)
        graph.replay()
        torch.cuda.synchronize()
        N = int(plain.n_sel)
        assert torch.equal(want[0][0][:N], got[0][0][:N]) and torch.equal(plain.seq_len, captured.seq_len), i
        for a, b in zip(want[1], got[1]):
            assert torch.equal(a, b), i
        assert int(plain.seq_len.max()) <= rows
    for a, b in zip(plain.cache, captured.cache):
        for s, n in enumerate(plain.seq_len.tolist()):
            assert torch.equal(a[s, :, :n], b[s, :, :n])


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (64, 4, 4)])
def test_a_second_chunk_attends_the_context(D, Hq, Hkv):
    """A prompt's second chunk, ragged, through the global branch's dense form on what
    `context` gives: the rows of both chunks as the cache holds them.  The output's rounding to
    bf16 is 2^-8, a weight's for the product too; logits and sums in fp32 stay below 2^-10."""
    from paper_2608_29539_gb300 import logo as Lg
    from paper_2608_29539_gb300.serve import Serve4Config, ServeBatch4
    B, rows, G = 3, 400, Hq // Hkv
    g = torch.Generator().manual_seed(D)
    batch = ServeBatch4(Serve4Config(B, 1, Hq, Hkv, D, rows))
    bf = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)  # noqa: E731
    first, second = [200, 1, 77], [150, 130, 0]
    held = [[[] for _ in range(B)] for _ in range(2)]
    for valid in (first, second):
        n = max(valid)
        k, v = bf(B, n, Hkv, D), bf(B, n, Hkv, D)
        batch.fill(k.cuda(), v.cuda(), torch.tensor(valid, dtype=torch.int32, device="cuda"))
        for x, rows_of in zip((k, v), held):
            y = C.values(*C.quantise(x))
            for b in range(B):
                rows_of[b] += list(y[b, :valid[b]])
    m = max(a + b for a, b in zip(first, second))
    k, v = batch.context(m)
    q, gate = bf(B, m, Hq, D), torch.zeros(B, m)
    for b in range(B):
        gate[b, first[b]:first[b] + second[b]] = 1.0
    _, pos, cu, row_of, n_sel = Lg.logo_select(gate.cuda(), Lg.LOGO_SELECT_THRESHOLD, 0.5)
    o, lse = Lg.logo_global_sparse_attn_fwd(q.cuda(), k, v, pos, cu, n_sel)
    torch.cuda.synchronize()
    assert Lg.logo_get_device_status() == 0 and int(n_sel) == sum(second)
    for r, (b, t) in enumerate((b, t) for b in range(B) for t in range(first[b], first[b] + second[b])):
        kk, vv = (torch.stack(h[b][:t + 1]) for h in held)
        for h in range(Hkv):
            hs = slice(h * G, (h + 1) * G)
            x = q[b, t, hs].double() @ kk[:, h].T / D ** 0.5
            w = torch.softmax(x, 1)
            want, absv = w @ vv[:, h], w @ vv[:, h].abs()
            got = o[r, hs].double().cpu()
            assert ((got - want).abs() <= 1.01 * (2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -10) * absv)).all()
            assert ((lse[hs, r].double().cpu() - torch.logsumexp(x, 1)).abs() <= 2.0 ** -10).all()


def test_filling_after_a_capture():
    """Captured steps, then a chunk for one sequence: the others keep their rows, however
    wide the chunk is, and the next replay goes on from there."""
    from paper_2608_29539_gb300.serve import Serve4Config, ServeBatch4
    B, n_new, Hq, Hkv, D, rows = 2, 1, 4, 2, 64, 100
    g = torch.Generator().manual_seed(0)
    bf = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()  # noqa: E731
    batch = ServeBatch4(Serve4Config(B, n_new, Hq, Hkv, D, rows))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    batch.fill(bf(B, 93, Hkv, D), bf(B, 93, Hkv, D), i32(93, 8))
    x = (bf(B, n_new, Hq, D), bf(B, n_new, Hkv, D), bf(B, n_new, Hkv, D), torch.ones(B, n_new, device="cuda"))
    batch.step(*x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, _, _ = batch.step(*x)
    graph.replay()
    assert batch.seq_len.tolist() == [95, 10]
    before = [t[0].clone() for t in batch.context()]
    k, v = bf(B, 40, Hkv, D), bf(B, 40, Hkv, D)
    batch.fill(k, v, i32(0, 40))
    assert batch.seq_len.tolist() == [95, 50]
    assert all(torch.equal(a, b[0]) for a, b in zip(before, batch.context()))
    want = C.values(*C.quantise(k[1].cpu()))
    assert torch.equal(batch.context()[0][1, 10:50].double().cpu(), want)
    graph.replay()
    assert batch.seq_len.tolist() == [96, 51] and bool(torch.isfinite(o).all())
