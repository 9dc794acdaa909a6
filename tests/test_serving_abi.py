"""Host-side refusals of the serving entry points (CPU: nothing is launched),
and the serving definitions themselves on small cases."""
import ctypes
import math

import pytest
import torch

import serving_ref as R
from paper_2608_29539_gb300 import build

null = None
fake = ctypes.c_void_p(1 << 20)  # aligned, never dereferenced: rejected before use
odd = ctypes.c_void_p((1 << 20) + 2)
f = ctypes.c_float


@pytest.fixture(scope="module")
def logo():
    build.build()
    from paper_2608_29539_gb300 import logo
    logo.lib()
    return logo


def test_prefix_attn_host_checks(logo):
    L = logo.lib()
    d = logo.Dims(4, 256, 8, 2, 128)
    ws = L.logo_decode_prefix_workspace_size(d, 2, 100, 0)
    assert 0 < ws <= L.logo_decode_prefix_workspace_size(d, 2, 100, 1)
    for bad, n, P in ((logo.Dims(4, 256, 8, 2, 96), 1, 0), (logo.Dims(4, 256, 8, 3, 128), 1, 0),
                      (logo.Dims(0, 256, 8, 2, 128), 1, 0), (d, 0, 0), (d, 1, -1),
                      (logo.Dims(1 << 14, 4, 8, 2, 128), 1 << 11, 0)):
        assert L.logo_decode_prefix_workspace_size(bad, n, P, 0) == 0

    def call(q=fake, kp=fake, kc=fake, lens=fake, pos=fake, cu=fake, n=fake, o=fake, m_in=null, m_out=null, dims=d,
             n_new=2, P=100, scale=0.0, w=fake, wb=None):
        return L.logo_decode_prefix_attn(q, kp, kp, kc, kc, lens, pos, cu, n, o, null, m_in, m_out, dims, n_new, P,
                                         f(scale), w, ws if wb is None else wb, null)

    bad = logo.LOGO_ERR_INVALID_ARG
    for kw in (dict(q=null), dict(kp=null), dict(kc=null), dict(lens=null), dict(pos=null), dict(cu=null),
               dict(n=null), dict(o=null), dict(m_out=fake), dict(n_new=0), dict(P=-1), dict(scale=-1.0),
               dict(scale=math.nan)):
        assert call(**kw) == bad, kw
    for kw in (dict(q=odd), dict(kp=odd), dict(kc=odd), dict(o=odd), dict(dims=logo.Dims(4, 256, 8, 2, 80)),
               dict(dims=logo.Dims(4, 256, 9, 2, 128))):
        assert call(**kw) == logo.LOGO_ERR_UNSUPPORTED, kw
    for kw in (dict(w=null), dict(wb=ws - 1), dict(w=odd)):
        assert call(**kw) == logo.LOGO_ERR_WORKSPACE, kw


def test_cache_evict_host_checks(logo):
    L = logo.lib()
    d = logo.Dims(4, 256, 2, 2, 128)
    ws = L.logo_cache_evict_workspace_size(d)
    assert ws > 0
    assert L.logo_cache_evict_workspace_size(logo.Dims(4, 256, 2, 2, 96)) == 0
    assert L.logo_cache_evict_workspace_size(logo.Dims(4, 0, 2, 2, 64)) == 0
    other = ctypes.c_void_p(1 << 21)

    def call(k=fake, v=fake, mass=fake, pos=fake, lens=fake, seen=fake, mo=fake, po=fake, nl=other, dims=d, budget=64,
             recent=8, w=fake, wb=None):
        return L.logo_cache_evict(k, v, mass, pos, lens, seen, mo, po, nl, dims, budget, recent, w,
                                  ws if wb is None else wb, null)

    for kw in (dict(k=null), dict(v=null), dict(mass=null), dict(pos=null), dict(lens=null), dict(seen=null),
               dict(mo=null), dict(po=null), dict(nl=null), dict(nl=fake), dict(budget=0), dict(budget=257),
               dict(recent=-1), dict(recent=65)):
        assert call(**kw) == logo.LOGO_ERR_INVALID_ARG, kw
    for kw in (dict(k=odd), dict(v=odd), dict(dims=logo.Dims(4, 256, 2, 2, 32))):
        assert call(**kw) == logo.LOGO_ERR_UNSUPPORTED, kw
    for kw in (dict(w=null), dict(wb=ws - 1), dict(w=odd)):
        assert call(**kw) == logo.LOGO_ERR_WORKSPACE, kw


def test_verify_draft_host_checks(logo):
    L = logo.lib()
    ws = L.logo_verify_draft_workspace_size(4, 3, 1000)
    assert ws > 0
    for B, m, V in ((0, 3, 10), (1, -1, 10), (1, 3, 0), (1 << 20, 31, 10)):
        assert L.logo_verify_draft_workspace_size(B, m, V) == 0

    def call(d=fake, q=fake, p=fake, u=fake, e=fake, t=fake, n=fake, B=4, m=3, V=1000, w=fake, wb=None):
        return L.logo_verify_draft(d, q, p, u, e, null, t, n, B, m, V, w, ws if wb is None else wb, null)

    for kw in (dict(d=null), dict(q=null), dict(p=null), dict(u=null), dict(e=null), dict(t=null), dict(n=null),
               dict(B=0), dict(m=-1), dict(V=0), dict(B=1 << 20, m=31)):
        assert call(**kw) == logo.LOGO_ERR_INVALID_ARG, kw
    for kw in (dict(w=null), dict(wb=ws - 1), dict(w=odd)):
        assert call(**kw) == logo.LOGO_ERR_WORKSPACE, kw


def test_definition_of_the_weights():
    """Each row's weights over prefix and own rows add up to 1."""
    g = torch.Generator().manual_seed(0)
    t = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    q, kc, vc = t(2, 3, 4, 8), t(2, 10, 2, 8), t(2, 10, 2, 8)
    rows = [(0, 0), (0, 2), (1, 1)]
    none = t(0, 2, 8)
    r = R.prefix_attn(q, none, none, kc, vc, [10, 2], rows, torch.zeros(2, 2, 10))
    assert abs(r["mass"].sum() - 3 * 4) < 1e-12
    assert r["mass"][1, :, 2:].sum() == 0 and r["mass"][0, 0, 9] > 0
    # token 1 of the three sees one row less than the last token
    assert R.own_visible(10, 3, 1) == 9 and R.own_visible(2, 3, 0) == 0 and R.own_visible(2, 3, 1) == 1


def test_definition_of_the_cut():
    src, end = R.evict([5.0, 1.0, 3.0, 2.0, 4.0, 0.0], [0, 1, 2, 3, 4, 5], 6, 6, 3, 1)
    assert (src, end) == ([0, 4, 5], 3)  # row 5 is recent; 0 and 4 weigh most
    assert R.evict([1.0, 2.0], [0, 1], 2, 2, 3, 1) == ([0, 1], 2)
