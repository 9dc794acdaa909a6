"""Outputs of the 4-bit cache's and the probabilities' calls that lie over what is still to
be read, or over each other (CPU: refused before anything is launched)."""
import ctypes

import pytest

from paper_2608_29539_gb300 import build

at = lambda x: ctypes.c_void_p(x)  # noqa: E731  (aligned, never dereferenced: refused before use)
far = at(1 << 30)


@pytest.fixture(scope="module")
def logo():
    build.build()
    from paper_2608_29539_gb300 import logo
    logo.lib()
    return logo


def _cache(logo):
    return logo._Cache4Ptrs(*(at((i + 8) << 26) for i in range(4)))


@pytest.mark.parametrize("shift", [0, 16, 4 * 2 * 8 * 128 * 2 - 16, -16])
def test_attention_does_not_write_over_its_queries(logo, shift):
    d = logo.Dims(4, 256, 8, 2, 128)
    ws = logo.lib().logo_decode_cache4_workspace_size(d, 2)
    q = 1 << 20
    assert logo.lib().logo_decode_cache4_attn(at(q), _cache(logo), far, far, far, far, at(q + shift), None, d, 2, 0.0,
                                              at(1 << 29), ws, None) == logo.LOGO_ERR_INVALID_ARG


@pytest.mark.parametrize("shift", [0, 16, 4 * 3 * 2 * 64 * 2 - 16, -16])
def test_rows_are_read_into_two_buffers(logo, shift):
    k = 1 << 20
    assert logo.lib().logo_cache4_read(_cache(logo), far, None, at(k), at(k + shift), logo.Dims(4, 256, 2, 2, 64), 3,
                                       None) == logo.LOGO_ERR_INVALID_ARG


@pytest.mark.parametrize("half", [0, 1])
@pytest.mark.parametrize("where", ["ahead", "behind", "middle"])
def test_probabilities_go_over_all_of_the_logits_or_none(logo, half, where):
    B, m1, V = 2, 3, 1000
    x, size = 1 << 20, B * m1 * V * 4
    p = x + {"ahead": 16 - size, "behind": size // (1 + half) - 16, "middle": 4000}[where]
    assert logo.lib().logo_target_probs(at(x), half, *[None] * 9, at(p), B, m1, V, 0, 0, at(1 << 29), 1 << 20,
                                        None) == logo.LOGO_ERR_INVALID_ARG
