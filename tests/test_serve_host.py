"""ServeBatch's bookkeeping on the host (CPU: the caches are CPU tensors, and what
would run on the GPU is replaced by its definition or not reached)."""
import pytest
import torch

from paper_2608_29539_gb300 import build


@pytest.fixture(scope="module")
def serve():
    build.build()
    from paper_2608_29539_gb300 import serve
    return serve


def _new(B, n, D=64, Hkv=2):
    return torch.ones(B, n, Hkv, D, dtype=torch.bfloat16), torch.ones(B, n, Hkv, D, dtype=torch.bfloat16)


def _batch(serve, B=2, n=3, budget=8, slack=0):
    return serve.ServeBatch(serve.ServeConfig(B, n, 4, 2, 64, budget, 2, slack=slack), device="cpu")


def _evict(serve, monkeypatch):
    """logo_cache_evict's lengths alone."""
    def cut(k, v, mass, slot_pos, seq_len, n_seen, budget, recent, new_len=None, workspace=None):
        new_len.copy_(seq_len.clamp(max=budget))
    monkeypatch.setattr(serve.L, "logo_cache_evict", cut)


@pytest.mark.parametrize("slack", [0, 1, 2, 3, 6])
def test_a_step_past_the_cache_is_refused(serve, monkeypatch, slack):
    """Before anything is written, and not before: slack / n_new + 1 steps fit after an
    eviction, however full it left the caches."""
    _evict(serve, monkeypatch)
    batch = _batch(serve, n=3, budget=8, slack=slack)
    for _ in range(batch.rows // 3):
        batch.append(*_new(2, 3))
    for _ in range(3):
        before = batch.seq_len.clone(), batch.n_seen.clone()
        with pytest.raises(ValueError, match="evict"):
            batch.append(*_new(2, 3))
        assert torch.equal(batch.seq_len, before[0]) and torch.equal(batch.n_seen, before[1])
        batch.evict()
        assert batch.seq_len.tolist() == [8, 8]
        for _ in range(slack // 3 + 1):
            batch.append(*_new(2, 3))


def test_full_caches_are_not_written_past(serve):
    """What a replay meets, whose steps nobody counts: the latest rows are overwritten."""
    batch = _batch(serve, n=3, budget=8)
    batch._captured = True
    for i in range(9):
        k, v = _new(2, 3)
        batch.append(k * (i + 1), v)
    assert batch.rows == 11 and batch.seq_len.tolist() == [11, 11]
    assert batch.n_seen.tolist() == [27, 27]
    assert batch.k[0, :, 0, 0].tolist() == [1, 1, 1, 2, 2, 2, 3, 3, 9, 9, 9]
    assert batch.slot_pos[0, 0, 8:].tolist() == [24, 25, 26]


def test_an_eviction_keeps_the_lengths_where_they_are(serve, monkeypatch):
    """A graph's replays read and write the buffers of the capture."""
    _evict(serve, monkeypatch)
    batch = _batch(serve, n=3, budget=4, slack=2)
    at = batch.seq_len.data_ptr(), batch.new_len.data_ptr(), batch.n_seen.data_ptr()
    for want in ([3, 3], [4, 4], [4, 4]):
        batch.append(*_new(2, 3))
        batch.evict()
        assert batch.seq_len.tolist() == want
        assert (batch.seq_len.data_ptr(), batch.new_len.data_ptr(), batch.n_seen.data_ptr()) == at
