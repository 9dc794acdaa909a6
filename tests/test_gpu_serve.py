"""ServeBatch: steps of drafted tokens over a shared prefix with verification
and eviction, against plain bookkeeping in 64 bits (the definitions of
serving_ref) of the tokens that every (sequence, KV head) still holds."""
import numpy as np
import pytest
import torch

import serving_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,Hq,Hkv,P,n_new", [(128, 8, 2, 200, 3), (64, 4, 4, 0, 1), (64, 12, 2, 130, 4)])
def test_steps_verify_and_evict(D, Hq, Hkv, P, n_new):
    from paper_2608_29539_gb300 import logo as Lg
    from paper_2608_29539_gb300.serve import ServeBatch, ServeConfig
    B, budget, recent, V, steps = 3, 24, 6, 50, max(14, 40 // n_new)
    G = Hq // Hkv
    g = torch.Generator().manual_seed(D + P + n_new)
    bf = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)  # noqa: E731
    kp, vp = bf(P, Hkv, D), bf(P, Hkv, D)
    batch = ServeBatch(ServeConfig(B, n_new, Hq, Hkv, D, budget, recent, slack=2 * n_new), kp.cuda() if P else None,
                       vp.cuda() if P else None)
    # plain: per (b, h) the rows in order: k, v, mass, position
    cache = [[dict(k=[], v=[], mass=[], pos=[]) for _ in range(Hkv)] for _ in range(B)]
    seen = [P] * B
    evicted = 0
    for step in range(steps):
        q, kn, vn = bf(B, n_new, Hq, D), bf(B, n_new, Hkv, D), bf(B, n_new, Hkv, D)
        gate = torch.rand((B, n_new), generator=g)
        o_c, z, row_of = batch.step(q.cuda(), kn.cuda(), vn.cuda(), gate.cuda())
        torch.cuda.synchronize()
        assert Lg.logo_get_device_status() == 0
        want_z = gate > 0.5
        assert torch.equal(z.cpu().bool(), want_z)
        rows = [(b, i) for b in range(B) for i in range(n_new) if want_z[b, i]]
        got_mass = batch.mass.cpu().double()
        for b in range(B):
            for h in range(Hkv):
                c = cache[b][h]
                for i in range(n_new):
                    c["k"].append(kn[b, i, h].double())
                    c["v"].append(vn[b, i, h].double())
                    c["mass"].append(0.0)
                    c["pos"].append(seen[b] + i)
            seen[b] += n_new
        for r, (b, i) in enumerate(rows):
            for h in range(Hkv):
                c = cache[b][h]
                vis = len(c["k"]) - n_new + i + 1
                k = torch.stack([*kp[:, h].double(), *c["k"][:vis]])
                v = torch.stack([*vp[:, h].double(), *c["v"][:vis]])
                x = q[b, i, h * G:(h + 1) * G].double() @ k.T / D ** 0.5
                w = torch.softmax(x, 1)
                o, absv = w @ v, w @ v.abs()
                got = o_c[r, h * G:(h + 1) * G].double().cpu()
                # bf16 rounding of the output and of the weights, fp32 sums
                assert ((got - o).abs() <= 2.0 ** -8 * (o.abs() + absv) + 2.0 ** -12 * absv).all()
                for s in range(vis):
                    c["mass"][s] += float(w[:, P + s].sum())
        for b in range(B):
            for h in range(Hkv):
                m = torch.tensor(cache[b][h]["mass"], dtype=torch.float64)
                err = (got_mass[b, h, :len(m)] - m).abs()
                assert (err <= 2.0 ** -12 * m + 1e-9).all()
                cache[b][h]["mass"] = got_mass[b, h, :len(m)].tolist()  # go on from the same values
        if n_new > 1:
            m1 = n_new - 1
            p = torch.softmax(torch.randn((B, n_new, V), generator=g), -1)
            qd = torch.softmax(torch.randn((B, m1, V), generator=g), -1)
            draft = torch.randint(0, V, (B, m1), generator=g).int()
            u = torch.rand((B, m1), generator=g)
            e = torch.empty((B, V)).exponential_(1.0, generator=g)
            tokens, n_acc = batch.verify(draft.cuda(), qd.cuda(), p.cuda(), u.cuda(), e.cuda())
            want_t, want_n = R.verify(draft.numpy(), qd.numpy(), p.numpy(), u.numpy(), e.numpy(), [m1] * B)
            assert np.array_equal(tokens.cpu().numpy(), want_t) and n_acc.tolist() == want_n.tolist()
            for b in range(B):
                drop = m1 - int(want_n[b])
                seen[b] -= drop
                for h in range(Hkv):
                    for key in ("k", "v", "mass", "pos"):
                        if drop:
                            del cache[b][h][key][-drop:]
        if step % 2 == 1:
            batch.evict()
            for b in range(B):
                for h in range(Hkv):
                    c = cache[b][h]
                    src, end = R.evict(c["mass"], c["pos"], len(c["pos"]), seen[b], budget, recent)
                    evicted += len(c["pos"]) - end
                    for key in ("k", "v", "mass", "pos"):
                        c[key] = [c[key][s] for s in src]
        assert batch.seq_len.tolist() == [len(cache[b][0]["pos"]) for b in range(B)]
        assert batch.n_seen.tolist() == seen
        for b in range(B):
            for h in range(Hkv):
                n = len(cache[b][h]["pos"])
                assert batch.slot_pos[b, h, :n].tolist() == cache[b][h]["pos"]
                assert torch.equal(batch.k[b, :n, h].double().cpu(), torch.stack(cache[b][h]["k"]))
    assert evicted > 0


def test_refuses_impossible_budgets():
    from paper_2608_29539_gb300.serve import ServeBatch, ServeConfig
    for kw in (dict(budget=0, recent=0), dict(budget=4, recent=5), dict(budget=4, recent=0, slack=-1)):
        with pytest.raises(ValueError):
            ServeBatch(ServeConfig(1, 1, 4, 4, 64, **kw))
