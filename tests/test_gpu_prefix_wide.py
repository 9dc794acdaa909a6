"""logo_decode_prefix_attn where the prefix's products go to 128-row tiles: many
rows of a long prefix per KV head.  The prefix's length is taken from the rule
that the call itself goes by (its constants are read from the source), so that
other constants move the cases along; and the workspace shows which way the call
went, as the shares' row sums are its last part where no weights are wanted.

Bounds as in test_gpu_prefix_attn."""
import os
import re

import pytest
import torch

import test_gpu_prefix_attn as T

pytestmark = pytest.mark.gpu

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_29539_gb300", "csrc")


def _constants():
    text = "".join(open(os.path.join(SRC, f), encoding="utf-8").read() for f in sorted(os.listdir(SRC))
                   if f.startswith("prefix"))
    return {k: int(re.search(rf"\b{k} = (\d+)", text).group(1))
            for k in ("kPaNarrow", "kPaNarrowCap", "kRunCost", "kPaRows", "kPaTile", "kPaWideUnits")}


def _limits(rows_cap, Hkv, P):
    """(tiles kernel possible, row tiles of 32 up to which it is not used)."""
    from paper_2608_29539_gb300 import logo as Lg
    c, sms = _constants(), Lg.logo_num_sms()
    units = Hkv * (-(-P // c["kPaTile"]) + c["kRunCost"])
    rt = -(-rows_cap // c["kPaRows"])
    if rt * units <= c["kPaNarrowCap"] * sms:
        return False, rt
    return rt > max(1, c["kPaNarrow"] * sms // units), max(1, c["kPaNarrow"] * sms // units)


def _prefix_for(rows_cap, Hkv, tail):
    """The shortest prefix past the rule by a quarter, ending `tail` keys into a tile."""
    k = 1
    while not (_limits(rows_cap, Hkv, 128 * k + tail)[0] and _limits(rows_cap, Hkv, 96 * k)[0]):
        k += 1
    return 128 * k + tail


def _wide_ran(B, n, Hq, Hkv, D, P, L, lens, z, seed):
    """Does a call without weights leave row sums of 128-row tiles?"""
    from paper_2608_29539_gb300 import logo as Lg
    q, kp, vp, kc, vc = (t.cuda() for t in T._inputs(B, n, Hq, Hkv, D, P, L, seed))
    pos, cu, ns, _ = T._pack(z)
    ws = Lg.logo_decode_prefix_workspace(q, kp, kc, False)
    ws.fill_(0xff)
    Lg.logo_decode_prefix_attn(q, kp, vp, kc, vc, torch.tensor(lens, dtype=torch.int32, device="cuda"), pos.cuda(),
                               cu.cuda(), ns.cuda(), workspace=ws)
    torch.cuda.synchronize()
    units = max(_constants()["kPaWideUnits"], -(-B * n * (Hq // Hkv) // 128) * Hkv)
    assert ws.numel() > units * 128 * (D + 2) * 4
    return bool((ws[-units * 128 * 4:] != 0xff).any())


@pytest.mark.parametrize("B,n,Hkv,G,D,tail,share,mass", [
    (9, 2, 2, 37, 128, 37, 1.0, True),    # weights in the join's launch; 666 rows: a partial last tile
    (5, 8, 1, 40, 64, 1, 0.9, True),      # weights in a launch of their own
    (45, 4, 4, 4, 128, 127, 0.9, True),   # many sequences, few rows each
    (1, 5, 2, 128, 64, 64, 1.0, False),   # one sequence; whole row tiles
    (33, 1, 1, 8, 128, 5, 1.0, False),    # three row tiles, many shares
])
def test_wide_prefix(B, n, Hkv, G, D, tail, share, mass):
    P = _prefix_for(B * n * G, Hkv, tail)
    lens = [(37 * b) % 140 + n for b in range(B)]
    z = T._z(B, n, share, D)
    possible, narrow = _limits(B * n * G, Hkv, P)
    assert possible and int(z.sum()) * G > 32 * narrow
    assert _wide_ran(B, n, Hkv * G, Hkv, D, P, 150, lens, z, seed=3)
    T._run(B, n, Hkv * G, Hkv, D, P, 150, lens, z, seed=17 + D, mass=mass)


def test_one_share_of_a_wide_prefix():
    """As many (row tile, KV head) pairs as SMs: the key range is not cut."""
    from paper_2608_29539_gb300 import logo as Lg
    Hkv, G = 8, 64
    B = Lg.logo_num_sms() // Hkv * 2  # 128 rows for every two sequences
    P = max(700, _prefix_for(B * G, Hkv, 60))
    lens = [(7 * b) % 33 + 1 for b in range(B)]
    z = torch.ones(B, 1, dtype=torch.bool)
    assert _wide_ran(B, 1, Hkv * G, Hkv, 64, P, 33, lens, z, seed=4)
    T._run(B, 1, Hkv * G, Hkv, 64, P, 33, lens, z, seed=23)


def test_too_few_selected_rows_for_wide_tiles():
    """Room for the tiles, but the rows that are selected do not fill them."""
    B, n, Hkv, G, D = 45, 4, 4, 4, 128
    P = _prefix_for(B * n * G, Hkv, 20)
    possible, narrow = _limits(B * n * G, Hkv, P)
    z = torch.zeros(B, n, dtype=torch.bool)
    z.view(-1)[3::7][:8 * narrow] = True  # 32 narrow rows
    z[-1, -1] = False
    assert possible and 0 < int(z.sum()) * G <= 32 * narrow
    lens = [(37 * b) % 140 + n for b in range(B)]
    assert not _wide_ran(B, n, Hkv * G, Hkv, D, P, 150, lens, z, seed=5)
    T._run(B, n, Hkv * G, Hkv, D, P, 150, lens, z, seed=29)
