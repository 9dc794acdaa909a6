"""logo_cache_evict by a cluster of seven CTAs per (sequence, KV head): rows that
do not divide by seven, weights of few values, a sequence shorter than one CTA's
stretch."""
import pytest
import torch

import test_gpu_cache_evict as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,L,budget", [(1, 2, 20000, 850), (2, 1, 19999, 850)])
def test_cluster_of_seven(B, H, L, budget):
    g = torch.Generator().manual_seed(L)
    lens = [L, budget + 1][:B]
    slot_pos, n_seen = T._positions(B, H, L, lens, g, False)
    mass = torch.randint(0, 9, (B, H, L), generator=g).float()
    T._run(B, H, 64, L, lens, budget, 100, mass, slot_pos, n_seen)
