"""logo_cache4_append and logo_cache4_read against the format's definition: codes
and values have to be equal."""
import numpy as np
import pytest
import torch

import cache4_ref as R

pytestmark = pytest.mark.gpu


def _logo():
    from paper_2608_29539_gb300 import logo
    return logo


def _same_codes(got, want):
    """Equal, but for the sign of a zero."""
    norm = lambda c: torch.stack([torch.where(x == 8, 0, x) for x in (c & 15, c >> 4)])  # noqa: E731
    return torch.equal(norm(got.cpu()), norm(want))


def _tokens(shape, seed):
    g = torch.Generator().manual_seed(seed)
    spread = torch.randn(shape[:-1] + (1,), generator=g).mul_(2.0).exp_()
    return torch.randn(shape, generator=g).mul_(spread).to(torch.bfloat16)


def _filled(logo, B, L, Hkv, D, seed):
    g = torch.Generator().manual_seed(seed)
    cache = logo.logo_cache4_empty(B, L, Hkv, D)
    for t in cache:
        t.copy_(torch.randint(0, 256, t.shape, generator=g, dtype=torch.uint8))
    return cache, [t.cpu().clone() for t in cache]


@pytest.mark.parametrize("B,n,Hkv,D,L,lens,valid", [
    (1, 1, 4, 64, 7, [7], None),
    (1, 1, 1, 128, 1, [1], None),
    (3, 5, 2, 128, 33, [5, 33, 17], None),
    (4, 9, 3, 64, 40, [9, 3, 44, 30], [9, 5, 7, 0]),      # rows before the first and past the last one
    (5, 6, 1, 128, 20, [6, 10, 20, 6, 6], [-2, 3, 99, 1, 6]),
    (2, 300, 8, 128, 301, [301, 250], [300, 211]),
    (2, 131, 16, 64, 500, [400, 131], None),
    (300, 1, 2, 64, 3, [1 + b % 3 for b in range(300)], None),
])
def test_append(B, n, Hkv, D, L, lens, valid):
    logo = _logo()
    cache, (k0, v0, ks0, vs0) = _filled(logo, B, L, Hkv, D, n)
    k, v = _tokens((B, n, Hkv, D), 1), _tokens((B, n, Hkv, D), 2)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    out = logo.logo_cache4_append(cache, k.cuda(), v.cuda(), i32(lens), None if valid is None else i32(valid))
    assert out is cache
    torch.cuda.synchronize()
    for x, codes, scales in ((k, k0, ks0), (v, v0, vs0)):
        c, s = R.quantise(x)
        for b in range(B):
            nv = n if valid is None else max(0, min(n, valid[b]))
            for i in range(nv):
                row = lens[b] - nv + i
                if 0 <= row < L:
                    codes[b, :, row], scales[b, :, row] = c[b, i], s[b, i]
    assert torch.equal(cache.k_scale.cpu(), ks0) and torch.equal(cache.v_scale.cpu(), vs0)
    assert _same_codes(cache.k, k0) and _same_codes(cache.v, v0)


def test_every_magnitude():
    """Groups whose largest magnitude is each bf16 value there is, NaN and infinities
    among them, with the other channels on and beside the borders between codes."""
    logo = _logo()
    top = torch.arange(0, 1 << 15, dtype=torch.int16).view(torch.bfloat16)
    g = torch.Generator().manual_seed(0)
    border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    c, s = R.quantise(torch.cat([top[:, None], torch.zeros(len(top), 15)], 1).to(torch.bfloat16))
    scale = R.values(torch.full((len(top), 8), 0x22, dtype=torch.uint8), s)[:, :1].float().nan_to_num(1.0)
    x = (scale * border[torch.randint(0, 7, (len(top), 64), generator=g)]).to(torch.bfloat16)
    step = torch.randint(-1, 2, x.shape, generator=g, dtype=torch.int16)  # a step of bf16 to either side
    x = (x.view(torch.int16) + step).clamp(min=0).view(torch.bfloat16)
    x = torch.where(x.abs() > top[:, None].abs(), top[:, None], x)
    x[:, ::16] = top[:, None]
    x = torch.where(torch.rand(x.shape, generator=g) < 0.5, -x, x).view(1, -1, 1, 64)
    n = x.shape[1]
    cache = logo.logo_cache4_empty(1, n, 1, 64)
    logo.logo_cache4_append(cache, x.cuda(), x.flip(1).contiguous().cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"))
    for got, scales, y in ((cache.k, cache.k_scale, x), (cache.v, cache.v_scale, x.flip(1))):
        c, s = R.quantise(y)
        assert torch.equal(scales.cpu()[0, 0], s[0, :, 0])
        live = (s[0, :, 0] != 255).repeat_interleave(8, -1)
        a, b = got.cpu()[0, 0], c[0, :, 0]
        assert _same_codes(torch.where(live, a, 0), torch.where(live, b, 0))


def test_read_every_code():
    logo = _logo()
    codes = torch.arange(256, dtype=torch.uint8).view(1, 1, 256, 1).repeat(1, 1, 1, 32)
    codes = (codes + torch.arange(32, dtype=torch.uint8)).contiguous()
    scales = torch.arange(256, dtype=torch.uint8).view(1, 1, 256, 1) + torch.tensor([0, 64, 129, 200], dtype=torch.uint8)
    # codes past the largest scale's stand for nothing that append writes, but for 255
    scales = torch.where(scales > 0xe2, 255, scales).to(torch.uint8)
    cache = logo.Cache4(*(t.cuda().contiguous() for t in (codes, codes.flip(2), scales, scales.flip(2))))
    k, v = logo.logo_cache4_read(cache, torch.tensor([256], dtype=torch.int32, device="cuda"))
    for got, c, s in ((k, codes, scales), (v, codes.flip(2), scales.flip(2))):
        want = R.values(c, s)[0, 0].numpy()
        got = got[0, :, 0].double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(np.nan_to_num(got), np.nan_to_num(want))


@pytest.mark.parametrize("B,m,Hkv,D,L,lens", [
    (1, 1, 1, 64, 1, [1]), (3, 37, 4, 128, 50, [50, 0, 13]), (2, 515, 2, 64, 333, [333, -4]),
    (4, 70, 16, 128, 64, [64, 99, 1, 63]), (260, 2, 1, 128, 5, [b % 6 for b in range(260)]),
])
def test_read(B, m, Hkv, D, L, lens):
    """All rows in order (more than there are, too) and lists with repetitions and
    numbers of no row."""
    logo = _logo()
    cache, (kc, vc, ks, vs) = _filled(logo, B, L, Hkv, D, 3)
    for t in (cache.k_scale, cache.v_scale, ks, vs):
        t.clamp_(max=0xe2)
    g = torch.Generator().manual_seed(m)
    listed = torch.randint(-2, L + 3, (B, m), generator=g, dtype=torch.int32)
    listed[0, 0] = 2 ** 31 - 1
    listed[-1, -1] = -2 ** 31
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for rows in (None, listed):
        dst = [torch.full((B, m, Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        k, v = logo.logo_cache4_read(cache, seq, None if rows is None else rows.cuda(), k=dst[0], v=dst[1])
        assert k is dst[0] and v is dst[1]
        at = (torch.arange(m).expand(B, m) if rows is None else rows).long()
        held = (at >= 0) & (at < torch.tensor(lens)[:, None]) & (at < L)
        where = torch.where(held, at, 0)
        for got, c, s in ((k, kc, ks), (v, vc, vs)):
            every = R.values(c, s)  # [B, Hkv, L, D]
            want = every[torch.arange(B)[:, None], :, where] * held[:, :, None, None]
            assert torch.equal(got.double().cpu(), want)


def test_round_trip_in_a_graph_on_a_side_stream():
    """Append and read captured together: replays follow the lengths and tokens in
    their buffers."""
    logo = _logo()
    B, n, Hkv, D, L = 3, 4, 2, 128, 32
    cache = logo.logo_cache4_empty(B, L, Hkv, D)
    k, v = (torch.zeros((B, n, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    seq = torch.full((B,), n, dtype=torch.int32, device="cuda")
    ko, vo = (torch.zeros((B, L, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        logo.logo_cache4_append(cache, k, v, seq)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logo.logo_cache4_append(cache, k, v, seq)
        logo.logo_cache4_read(cache, seq, k=ko, v=vo)
        seq += n
    want = torch.zeros((B, L, Hkv, D), dtype=torch.float64)
    seq.fill_(n)
    for step in range(3):
        x, y = _tokens((B, n, Hkv, D), 10 + step), _tokens((B, n, Hkv, D), 20 + step)
        k.copy_(x)
        v.copy_(y)
        graph.replay()
        want[:, step * n:(step + 1) * n] = R.values(*R.quantise(x))
        assert torch.equal(ko.double().cpu(), want)
        assert torch.equal(vo.double().cpu()[:, step * n:(step + 1) * n], R.values(*R.quantise(y)))


def test_refusals():
    logo = _logo()
    cache = logo.logo_cache4_empty(2, 16, 2, 64)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    x = bf(2, 3, 2, 64)
    for call in (lambda: logo.logo_cache4_append(cache, x, bf(2, 4, 2, 64), i32(2)),
                 lambda: logo.logo_cache4_append(cache, x.transpose(1, 2), x, i32(2)),
                 lambda: logo.logo_cache4_append(cache, x.float(), x, i32(2)),
                 lambda: logo.logo_cache4_append(cache, x, x, i32(3)),
                 lambda: logo.logo_cache4_append(cache, x, x, i32(2).cpu()),
                 lambda: logo.logo_cache4_append(cache, x, x, i32(2), i32(1)),
                 lambda: logo.logo_cache4_append(cache._replace(v=cache.v[:, :, :8]), x, x, i32(2)),
                 lambda: logo.logo_cache4_append(cache._replace(k_scale=cache.k), x, x, i32(2)),
                 lambda: logo.logo_cache4_read(cache, i32(2), rows=i32(2, 3, 1)),
                 lambda: logo.logo_cache4_read(cache, i32(2), rows=i32(3, 3)),
                 lambda: logo.logo_cache4_read(cache, i32(2), rows=i32(2, 3), m=4),
                 lambda: logo.logo_cache4_read(cache, i32(2), k=bf(2, 3, 2, 64), v=bf(2, 4, 2, 64)),
                 lambda: logo.logo_cache4_read(cache, i32(2, 1))):
        with pytest.raises(ValueError):
            call()
    odd = logo.logo_cache4_empty(1, 4, 1, 96)
    with pytest.raises(logo.LogoError, match="UNSUPPORTED"):
        logo.logo_cache4_append(odd, bf(1, 1, 1, 96), bf(1, 1, 1, 96), i32(1))
    with pytest.raises(logo.LogoError, match="INVALID"):
        logo.logo_cache4_append(cache, bf(2, 0, 2, 64), bf(2, 0, 2, 64), i32(2))
