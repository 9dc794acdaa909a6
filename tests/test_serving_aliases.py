"""Buffers that a serving call reads throughout and so must not write (CPU: refused
before anything is launched)."""
import ctypes

import pytest

from paper_2608_29539_gb300 import build


@pytest.mark.parametrize("alias", ["seq_len", "n_seen"])
def test_the_new_lengths_are_a_buffer_of_their_own(alias):
    build.build()
    from paper_2608_29539_gb300 import logo
    L = logo.lib()
    at = {name: ctypes.c_void_p((i + 1) << 20) for i, name in enumerate(
        ("k", "v", "mass", "slot_pos", "seq_len", "n_seen", "mass_out", "slot_pos_out"))}
    d = logo.Dims(4, 256, 2, 2, 128)
    ws = L.logo_cache_evict_workspace_size(d)
    assert L.logo_cache_evict(*at.values(), at[alias], d, 64, 8, ctypes.c_void_p(1 << 26), ws, None) == \
        logo.LOGO_ERR_INVALID_ARG
