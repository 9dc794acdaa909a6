"""Host-side refusals of the 4-bit cache's and the probabilities' entry points (CPU:
nothing is launched), and their definitions on small cases."""
import ctypes
import math

import numpy as np
import pytest
import torch

import cache4_ref as R
from paper_2608_29539_gb300 import build

null = None
fake = ctypes.c_void_p(1 << 20)  # aligned, never dereferenced: rejected before use
odd = ctypes.c_void_p((1 << 20) + 2)
other = ctypes.c_void_p(1 << 21)


@pytest.fixture(scope="module")
def logo():
    build.build()
    from paper_2608_29539_gb300 import logo
    logo.lib()
    return logo


def _cache(logo, **kw):
    at = dict(k=fake, v=fake, k_scale=fake, v_scale=fake) | kw
    return logo._Cache4Ptrs(*at.values())


def _bad_caches(logo):
    for name in ("k", "v", "k_scale", "v_scale"):
        yield _cache(logo, **{name: null}), logo.LOGO_ERR_INVALID_ARG
        yield _cache(logo, **{name: odd}), logo.LOGO_ERR_UNSUPPORTED


@pytest.mark.parametrize("fn", ["append", "read"])
def test_cache4_host_checks(logo, fn):
    L = logo.lib()
    d = logo.Dims(4, 256, 2, 2, 128)

    def call(c=None, a=fake, b=fake, lens=fake, opt=null, dims=d, n=3):
        c = c or _cache(logo)
        if fn == "append":
            return L.logo_cache4_append(c, a, b, lens, opt, dims, n, null)
        return L.logo_cache4_read(c, lens, opt, a, b, dims, n, null)

    for kw in (dict(a=null), dict(b=null), dict(lens=null), dict(n=0), dict(n=-1), dict(dims=logo.Dims(0, 256, 2, 2, 128)),
               dict(dims=logo.Dims(4, 0, 2, 2, 128)), dict(dims=logo.Dims(4, 256, 2, 0, 128))):
        assert call(**kw) == logo.LOGO_ERR_INVALID_ARG, kw
    for kw in (dict(a=odd), dict(b=odd), dict(dims=logo.Dims(4, 256, 2, 2, 96)), dict(n=1 << 29),
               dict(dims=logo.Dims(4, 256, 2, (1 << 16) + 1, 64)), dict(dims=logo.Dims(1 << 20, 1 << 11, 2, 2, 64)),
               dict(dims=logo.Dims(1 << 20, 4, 2, 1 << 15, 64))):
        assert call(**kw) == logo.LOGO_ERR_UNSUPPORTED, kw
    for c, want in _bad_caches(logo):
        assert call(c=c) == want


def test_attn_host_checks(logo):
    L = logo.lib()
    d = logo.Dims(4, 256, 8, 2, 128)
    ws = L.logo_decode_cache4_workspace_size(d, 2)
    assert ws > 0
    for bad, n in ((logo.Dims(4, 256, 8, 2, 96), 1), (logo.Dims(4, 256, 8, 3, 128), 1), (logo.Dims(0, 256, 8, 2, 128), 1),
                   (d, 0), (logo.Dims(1 << 14, 4, 8, 2, 128), 1 << 11), (d, 4096)):
        assert L.logo_decode_cache4_workspace_size(bad, n) == 0

    def call(q=fake, c=None, lens=fake, pos=fake, cu=fake, n=fake, o=fake, dims=d, n_new=2, scale=0.0, w=fake, wb=None):
        return L.logo_decode_cache4_attn(q, c or _cache(logo), lens, pos, cu, n, o, null, dims, n_new,
                                         ctypes.c_float(scale), w, ws if wb is None else wb, null)

    for kw in (dict(q=null), dict(lens=null), dict(pos=null), dict(cu=null), dict(n=null), dict(o=null), dict(n_new=0),
               dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf)):
        assert call(**kw) == logo.LOGO_ERR_INVALID_ARG, kw
    for kw in (dict(q=odd), dict(o=odd), dict(dims=logo.Dims(4, 256, 8, 2, 80)), dict(dims=logo.Dims(4, 256, 9, 2, 128)),
               dict(n_new=4096), dict(dims=logo.Dims(1, 1 << 30, 512, 512, 64), n_new=1),
               dict(dims=logo.Dims(1 << 20, 1 << 10, 1 << 12, 1 << 8, 64), n_new=16)):
        assert call(**kw) == logo.LOGO_ERR_UNSUPPORTED, kw
    for c, want in _bad_caches(logo):
        assert call(c=c) == want
    for kw in (dict(w=null), dict(wb=ws - 1), dict(w=odd)):
        assert call(**kw) == logo.LOGO_ERR_WORKSPACE, kw


def test_probs_host_checks(logo):
    L = logo.lib()

    def call(x=fake, half=0, T=null, pen=fake, hist=fake, hl=fake, npr=null, draft=null, bt=null, bv=null, ok=null,
             p=other, B=2, m1=3, V=1000, H=10, K=0, w=fake, wb=1 << 30):
        return L.logo_target_probs(x, half, T, pen, hist, hl, npr, draft, bt, bv, ok, p, B, m1, V, H, K, w, wb, null)

    for kw in (dict(x=null), dict(p=null), dict(B=0), dict(m1=0), dict(V=0), dict(H=-1), dict(K=-1), dict(hl=null),
               dict(hist=null), dict(hist=null, hl=null, npr=fake, H=0), dict(hist=null, hl=null), dict(H=0),
               dict(pen=null), dict(draft=fake, m1=1), dict(bt=fake), dict(bt=fake, bv=fake), dict(K=4),
               dict(K=4, bt=fake), dict(K=4, bv=fake), dict(pen=null, hist=null, hl=null, H=0, draft=fake)):
        assert call(**kw) == logo.LOGO_ERR_INVALID_ARG, kw
    for kw in (dict(x=odd), dict(p=odd), dict(V=278529), dict(m1=1025), dict(K=4097, bt=fake, bv=fake),
               dict(B=1 << 20, m1=17), dict(half=1, p=fake)):
        assert call(**kw) == logo.LOGO_ERR_UNSUPPORTED, kw
    ws = L.logo_target_probs_workspace_size(2, 3, 1000, 10, 0)
    assert 0 < ws < L.logo_target_probs_workspace_size(2, 3, 1000, 10, 90)
    for bad in ((0, 3, 10, 0, 0), (2, 0, 10, 0, 0), (2, 3, 0, 0, 0), (2, 3, 278529, 0, 0), (2, 3, 10, -1, 0)):
        assert L.logo_target_probs_workspace_size(*bad) == 0
    for kw in (dict(w=null), dict(w=odd), dict(wb=ws - 1)):
        assert call(**kw) == logo.LOGO_ERR_WORKSPACE, kw


def test_definition_of_the_format():
    """Every value a bf16 group can hold comes back as the nearest representable one."""
    assert R.SCALES[0xe2] == 10240 and R.SCALES[8] == 2.0 ** -14 and R.SCALES[7] == 7 * 2.0 ** -17
    assert R.SCALES[0x78] == float(np.uint16(0x78 << 7).view(np.float16)) == 1.0
    x = torch.zeros(1, 64, dtype=torch.bfloat16)
    x[0, :16] = torch.tensor([6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -5.03125, -0.26, 0.24, 0, 1e-3, 2.51, 4.9, -6])
    x[0, 16] = 1.1 * 6 * 2.0 ** -18
    x[0, 17] = 6 * 2.0 ** -18 * 0.9
    x[0, 32] = math.inf
    x[0, 48] = -1e30
    codes, scales = R.quantise(x)
    assert scales.tolist() == [[0x78, 1, 255, 0xe2]]
    v = R.values(codes, scales)[0]
    assert v[:16].tolist() == [6, 4, 4, 2, 2, 1, 1, 0, -6, -0.5, 0, 0, 0, 3, 4, -6]
    assert v[16] == 3 * 2.0 ** -17 and torch.isnan(v[32:48]).all() and v[48] == -61440


def test_definition_of_the_probabilities():
    x = R.adjusted([1.0, -1.0, 2.0, 0.0], (2.0, 0.5, 0.25), [0, 1, 1, 9, -1], 1, [2], [(3, 1.0), (3, 0.5), (7, 9.0)])
    assert x.tolist() == [0.5, -2.0 - 1.25, 1.0 - 0.75, 1.5]
    p = R.probs(x, 0.5)
    assert abs(p.sum() - 1) < 1e-12 and p.argmax() == 3
    assert R.probs(x, 0.0).tolist() == [0, 0, 0, 1]
    none = np.zeros(4, bool)
    assert R.probs(np.full(4, -np.inf), 1.0).tolist() == [0] * 4 and R.probs(x, 0.0, none).tolist() == [0] * 4
