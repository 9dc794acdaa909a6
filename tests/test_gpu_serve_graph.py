"""ServeBatch's steps as one captured CUDA graph against the same steps called one by
one: every buffer bit for bit, over enough replays for the caches to be cut often."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_new,slack", [(1, 0), (4, 0), (3, 7)])
def test_replays_of_a_captured_step(n_new, slack):
    from paper_2608_29539_gb300 import logo as Lg
    from paper_2608_29539_gb300.serve import ServeBatch, ServeConfig
    B, Hq, Hkv, D, P, V, budget = 3, 8, 2, 64, 150, 40, 12
    g = torch.Generator(device="cuda").manual_seed(n_new)
    bf = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    kp, vp = bf(P, Hkv, D), bf(P, Hkv, D)
    plain, captured = (ServeBatch(ServeConfig(B, n_new, Hq, Hkv, D, budget, 4, slack=slack), kp, vp) for _ in range(2))
    m = n_new - 1

    def inputs():
        return dict(q=bf(B, n_new, Hq, D), k=bf(B, n_new, Hkv, D), v=bf(B, n_new, Hkv, D),
                    gate=torch.rand((B, n_new), generator=g, device="cuda"),
                    draft=torch.randint(0, V, (B, m), generator=g, device="cuda").int(),
                    qd=torch.softmax(torch.randn((B, m, V), generator=g, device="cuda"), -1),
                    p=torch.softmax(torch.randn((B, n_new, V), generator=g, device="cuda"), -1),
                    u=torch.rand((B, m), generator=g, device="cuda"),
                    e=torch.empty((B, V), device="cuda").exponential_(1.0, generator=g))

    def step(batch, x):
        batch.step(x["q"], x["k"], x["v"], x["gate"])
        out = batch.verify(x["draft"], x["qd"], x["p"], x["u"], x["e"])
        batch.evict()
        return out

    x = inputs()
    for batch in (plain, captured):  # (also a graph's warm-up)
        step(batch, x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(captured, x)
    for i in range(25):
        for name, t in inputs().items():
            x[name].copy_(t)
        want = step(plain, x)
        graph.replay()
        torch.cuda.synchronize()
        assert Lg.logo_get_device_status() == 0
        for a, b in zip(want, got):
            assert torch.equal(a, b), i
        assert torch.equal(plain.seq_len, captured.seq_len) and torch.equal(plain.n_seen, captured.n_seen), i
        assert int(plain.seq_len.max()) <= budget
        for b, n in enumerate(plain.seq_len.tolist()):
            for name in ("k", "v"):
                assert torch.equal(getattr(plain, name)[b, :n], getattr(captured, name)[b, :n]), (i, name)
            for name in ("mass", "slot_pos"):
                assert torch.equal(getattr(plain, name)[b, :, :n], getattr(captured, name)[b, :, :n]), (i, name)
        N = int(plain.n_sel)
        assert torch.equal(plain.o_c[:N], captured.o_c[:N])
    assert int(plain.seq_len.max()) == budget
