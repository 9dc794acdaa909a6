"""logo_cache_evict against the definition: every output is compared bit for
bit (rows are moved, nothing is computed)."""
import numpy as np
import pytest
import torch

import serving_ref as R

pytestmark = pytest.mark.gpu


def _positions(B, H, L, lens, gen, fresh):
    if fresh:
        return torch.arange(L, dtype=torch.int32).expand(B, H, L).contiguous(), list(lens)
    pos = torch.stack([torch.randperm(2 * L, generator=gen)[:L] for _ in range(B * H)]).view(B, H, L)
    return pos.int(), [2 * L] * B


def _run(B, H, D, L, lens, budget, recent, mass, slot_pos, n_seen, seed=0, in_place=False):
    from paper_2608_29539_gb300 import logo as Lg
    g = torch.Generator().manual_seed(seed)
    k = torch.randint(-32768, 32767, (B, L, H, D), generator=g, dtype=torch.int16)  # any bit patterns, NaN included
    v = torch.randint(-32768, 32767, (B, L, H, D), generator=g, dtype=torch.int16)
    kd, vd = k.cuda().view(torch.bfloat16), v.cuda().view(torch.bfloat16)
    md, pd = mass.cuda(), slot_pos.cuda()
    ld = torch.tensor(lens, dtype=torch.int32, device="cuda")
    nd = torch.tensor(n_seen, dtype=torch.int32, device="cuda")
    mo = None if in_place else torch.full_like(md, -5.0)
    po = None if in_place else torch.full_like(pd, -5)
    got_m, got_p, new_len = Lg.logo_cache_evict(kd, vd, md, pd, ld, nd, budget, recent, mass_out=mo, slot_pos_out=po)
    torch.cuda.synchronize()
    assert Lg.logo_get_device_status() == 0
    rest_m = mass if in_place else torch.full_like(mass, -5.0)
    rest_p = slot_pos if in_place else torch.full_like(slot_pos, -5)
    want_k, want_v, want_m, want_p = k.clone(), v.clone(), rest_m.clone(), rest_p.clone()
    for b in range(B):
        for h in range(H):
            m = max(0, min(L, lens[b]))
            src, end = R.evict(mass[b, h].tolist(), slot_pos[b, h].tolist(), m, n_seen[b], budget, recent)
            src = torch.tensor(src, dtype=torch.long)
            want_k[b, :end, h] = k[b, src, h]
            want_v[b, :end, h] = v[b, src, h]
            want_m[b, h, :end] = mass[b, h, src]
            want_p[b, h, :end] = slot_pos[b, h, src]
    assert new_len.tolist() == [min(max(0, min(L, n)), budget) for n in lens]
    assert torch.equal(got_p.cpu(), want_p)
    assert np.array_equal(got_m.cpu().numpy().view(np.uint32), want_m.numpy().view(np.uint32))
    assert torch.equal(kd.view(torch.int16).cpu(), want_k)
    assert torch.equal(vd.view(torch.int16).cpu(), want_v)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("fresh", [False, True])
@pytest.mark.parametrize("B,H,D,L,budget,recent", [
    (1, 1, 64, 1, 1, 0), (2, 3, 64, 2, 1, 1), (3, 2, 128, 300, 64, 16), (2, 2, 128, 1030, 1024, 100),
    (2, 4, 64, 1025, 1, 1), (1, 2, 128, 5000, 2500, 2500), (4, 1, 64, 257, 256, 0), (2, 2, 128, 700, 700, 10)])
def test_sizes(B, H, D, L, budget, recent, fresh, in_place):
    g = torch.Generator().manual_seed(L + budget)
    lens = [L, max(0, budget - 1), min(L, budget + 1), 0][:B] if B > 1 else [L]
    slot_pos, n_seen = _positions(B, H, L, lens, g, fresh)
    mass = torch.randn((B, H, L), generator=g).exp()
    _run(B, H, D, L, lens, budget, recent, mass, slot_pos, n_seen, in_place=in_place)


@pytest.mark.parametrize("B,H,L,budget", [(1, 2, 20000, 3000), (1, 1, 70001, 40000), (2, 8, 9000, 8990)])
def test_long_caches(B, H, L, budget):
    g = torch.Generator().manual_seed(L)
    slot_pos, n_seen = _positions(B, H, L, [L] * B, g, False)
    mass = torch.randn((B, H, L), generator=g).exp()
    _run(B, H, 64, L, [L] * B, budget, 200, mass, slot_pos, n_seen)


# one CTA and clusters of three, six and eight per (sequence, KV head); the first sequences shorter than one CTA's stretch
@pytest.mark.parametrize("B,H,L,budget", [(40, 2, 1500, 700), (40, 2, 6000, 3000), (5, 2, 6000, 3000),
                                          (5, 1, 20000, 9000)])
def test_few_different_weights_in_many_ctas(B, H, L, budget):
    g = torch.Generator().manual_seed(B + L)
    lens = ([budget + 1, 0, budget + 40, L - 1] + [L] * B)[:B]
    slot_pos, n_seen = _positions(B, H, L, lens, g, False)
    mass = torch.randint(0, 5, (B, H, L), generator=g).float()
    _run(B, H, 64, L, lens, budget, 100, mass, slot_pos, n_seen)


def test_equal_weights_go_to_the_lower_row():
    B, H, L, budget = 2, 2, 3000, 1111
    g = torch.Generator().manual_seed(2)
    mass = torch.randint(0, 4, (B, H, L), generator=g).float() / 4
    mass[0, 1] = 0.5
    mass[1, 0, ::2] = -0.0
    mass[1, 0, 1::2] = 0.0
    slot_pos, n_seen = _positions(B, H, L, [L, L - 7], g, False)
    _run(B, H, 64, L, [L, L - 7], budget, 50, mass, slot_pos, n_seen)


def test_special_weights():
    """NaN goes first, then -inf; +inf stays, behind the recent window."""
    B, H, L, budget = 1, 2, 600, 100
    g = torch.Generator().manual_seed(3)
    mass = torch.randn((B, H, L), generator=g)
    mass[:, :, 5::7] = float("nan")
    mass[:, :, 3::11] = float("inf")
    mass[:, :, 2::13] = -float("inf")
    mass[0, 1, 50:] = float("nan")  # more NaN than can go
    slot_pos, n_seen = _positions(B, H, L, [L], g, False)
    _run(B, H, 128, L, [L], budget, 40, mass, slot_pos, n_seen)


def test_more_recent_rows_than_the_budget():
    """Positions that a cache cannot hold (all recent): the lowest rows stay,
    and nothing is written out of bounds."""
    B, H, L, budget = 2, 1, 400, 30
    g = torch.Generator().manual_seed(4)
    mass = torch.rand((B, H, L), generator=g)
    slot_pos = torch.full((B, H, L), 10 ** 6, dtype=torch.int32)
    _run(B, H, 64, L, [L, L], budget, 30, mass, slot_pos, [10, 10])


def test_lengths_outside_the_cache_are_clamped():
    B, H, L, budget = 2, 2, 100, 20
    g = torch.Generator().manual_seed(5)
    mass = torch.rand((B, H, L), generator=g)
    slot_pos, n_seen = _positions(B, H, L, [L, L], g, True)
    _run(B, H, 64, L, [L + 50, -3], budget, 5, mass, slot_pos, n_seen)


def test_a_second_call_changes_nothing():
    """After the cut, a sequence is at its budget."""
    from paper_2608_29539_gb300 import logo as Lg
    B, H, D, L, budget = 2, 2, 64, 500, 200
    g = torch.Generator().manual_seed(6)
    k = torch.randn((B, L, H, D), generator=g).to(torch.bfloat16).cuda()
    v = torch.randn((B, L, H, D), generator=g).to(torch.bfloat16).cuda()
    mass = torch.rand((B, H, L), generator=g).cuda()
    pos = torch.arange(L, dtype=torch.int32, device="cuda").expand(B, H, L).contiguous()
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    _, _, n1 = Lg.logo_cache_evict(k, v, mass, pos, lens, lens, budget, 20)
    once = [t.clone() for t in (k, v, mass, pos)]
    _, _, n2 = Lg.logo_cache_evict(k, v, mass, pos, n1, lens, budget, 20)
    torch.cuda.synchronize()
    assert n1.tolist() == n2.tolist() == [budget] * B
    for a, b in zip(once, (k, v, mass, pos)):
        assert torch.equal(a, b)


def test_cache_offsets_beyond_32_bits():
    from paper_2608_29539_gb300 import logo as Lg
    B, L, H, D = 2, 131200, 64, 128
    assert B * L * H * D > 2 ** 31
    k = torch.zeros((B, L, H, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[1, L - 1, 63], v[1, L - 1, 63] = 3.0, 4.0
    mass = torch.zeros((B, H, L), device="cuda")
    mass[:, :, 1:100] = 2.0
    mass[1, 63, L - 1] = 1.0
    pos = torch.arange(L, dtype=torch.int32, device="cuda").expand(B, H, L).contiguous()
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    m, p, n = Lg.logo_cache_evict(k, v, mass, pos, lens, lens, 100, 0)
    torch.cuda.synchronize()
    assert n.tolist() == [100, 100]
    assert bool((k[1, 0, 63] == 3.0).all()) and bool((v[1, 0, 63] == 4.0).all())
    assert int(p[1, 63, 0]) == L - 1 and float(m[1, 63, 0]) == 1.0
    assert int(p[1, 62, 0]) == 0 and int(p[0, 63, 0]) == 0
    assert not bool(k[0, :200].any()) and not bool(k[1, :200, :63].any())


def test_captures_in_a_graph_and_runs_on_another_stream():
    from paper_2608_29539_gb300 import logo as Lg
    g = torch.Generator().manual_seed(4)
    B, L, H, D, budget = 2, 5000, 4, 64, 2000
    k, v = (torch.randn((B, L, H, D), generator=g).bfloat16().cuda() for _ in range(2))
    mass = torch.rand((B, H, L), generator=g).cuda()
    pos = torch.arange(L, dtype=torch.int32).expand(B, H, L).contiguous().cuda()
    lens = torch.tensor([L, 3100], dtype=torch.int32, device="cuda")
    ws = Lg.logo_cache_evict_workspace(k)

    def run(x):
        return Lg.logo_cache_evict(x[0], x[1], x[2], x[3], lens, lens, budget, 100, new_len=x[4], workspace=ws)

    state = lambda: [k.clone(), v.clone(), mass.clone(), pos.clone(), torch.zeros_like(lens)]  # noqa: E731
    want, side, replayed = state(), state(), state()
    run(want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run(side)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(replayed)
    assert torch.equal(replayed[2], mass)  # captured, not run
    graph.replay()
    torch.cuda.synchronize()
    assert want[4].tolist() == [budget, budget]
    for a, b, c in zip(want, side, replayed):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_refusals():
    from paper_2608_29539_gb300 import logo as Lg
    B, H, D, L = 2, 2, 64, 32
    k = torch.zeros((B, L, H, D), dtype=torch.bfloat16, device="cuda")
    mass = torch.zeros((B, H, L), device="cuda")
    pos = torch.zeros((B, H, L), dtype=torch.int32, device="cuda")
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    call = Lg.logo_cache_evict
    for bad in ((k.float(), k, mass, pos, lens, lens), (k, k[:, :8], mass, pos, lens, lens),
                (k, k, mass.double(), pos, lens, lens), (k, k, mass, pos.long(), lens, lens),
                (k, k, mass, pos, lens[:1], lens), (k, k, mass, pos, lens, lens.float())):
        with pytest.raises(ValueError):
            call(*bad, 16, 4)
    for budget, recent in ((0, 0), (L + 1, 0), (16, -1), (16, 17)):
        with pytest.raises(Lg.LogoError) as e:
            call(k, k.clone(), mass, pos, lens, lens, budget, recent)
        assert e.value.code == Lg.LOGO_ERR_INVALID_ARG
    with pytest.raises(Lg.LogoError) as e:
        call(k, k.clone(), mass, pos, lens, lens, 16, 4, new_len=lens)
    assert e.value.code == Lg.LOGO_ERR_INVALID_ARG
    with pytest.raises(Lg.LogoError) as e:
        call(k, k.clone(), mass, pos, lens, lens, 16, 4, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.code == Lg.LOGO_ERR_WORKSPACE
