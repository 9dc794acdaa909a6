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


def _verify(serve, monkeypatch, accepted):
    def verdict(draft, q_draft, p_target, u, noise, draft_len=None, workspace=None):
        if draft is None:
            raise ValueError("draft must be a CUDA tensor")
        tokens = torch.zeros(draft.shape[0], draft.shape[1] + 1, dtype=torch.int32)
        return tokens, torch.tensor(accepted, dtype=torch.int32)
    monkeypatch.setattr(serve.L, "logo_verify_draft", verdict)
    args = torch.zeros(2, 2, dtype=torch.int32), None
    return lambda batch: batch.verify(*args, torch.zeros(2, batch.cfg.n_new, 5), None, None)


def test_drafts_are_verified_once_and_before_the_cut(serve, monkeypatch):
    """The rejected drafts' rows are dropped from the caches' ends, which holds until an
    eviction moves rows, and once."""
    _evict(serve, monkeypatch)
    verify = _verify(serve, monkeypatch, [0, 1])
    batch = _batch(serve, n=3, budget=4, slack=4)
    for start in ([0, 0], [1, 2]):
        batch.append(*_new(2, 3))
        assert batch.seq_len.tolist() == [a + 3 for a in start]
        with pytest.raises(ValueError, match="CUDA"):
            batch.verify(None, None, torch.zeros(2, 3, 5), None, None)  # a call that was refused has verified nothing
        verify(batch)
        assert batch.seq_len.tolist() == [start[0] + 1, start[1] + 2]
        with pytest.raises(ValueError, match="since the last step"):
            verify(batch)
        assert batch.seq_len.tolist() == [start[0] + 1, start[1] + 2]
    batch.append(*_new(2, 3))
    batch.evict()
    with pytest.raises(ValueError, match="since the last step"):
        verify(batch)
    assert batch.seq_len.tolist() == [4, 4]
    batch.append(*_new(2, 3))
    verify(batch)
    assert batch.seq_len.tolist() == [5, 6]


def test_one_new_token_has_no_drafts_to_drop(serve, monkeypatch):
    _evict(serve, monkeypatch)
    verify = _verify(serve, monkeypatch, [0, 0])
    batch = _batch(serve, n=1, budget=4, slack=4)
    batch.append(*_new(2, 1))
    batch.evict()
    verify(batch)
    assert batch.seq_len.tolist() == [1, 1]


def test_a_refused_step_leaves_the_caches_alone(serve):
    """Tensors that the calls do not take (here: on the CPU) are refused before the new
    tokens join the caches."""
    batch = _batch(serve, n=3, budget=8)
    k, v = _new(2, 3)
    for q, gate in ((torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 3)), (None, None)):
        with pytest.raises(ValueError):
            batch.step(q, k, v, gate)
        assert batch.seq_len.tolist() == [0, 0] and batch.n_seen.tolist() == [0, 0]
        assert float(batch.k.abs().sum()) == 0


@pytest.mark.parametrize("shape", [(2, 4, 5), (1, 3, 5), (3, 3, 5)])
def test_more_drafts_or_sequences_than_the_step_had_are_refused(serve, monkeypatch, shape):
    """(more accepted tokens than the step brought would lengthen the caches)"""
    _verify(serve, monkeypatch, [shape[1] - 1] * shape[0])
    batch = _batch(serve, n=3, budget=8)
    batch.append(*_new(2, 3))
    draft = torch.zeros(shape[0], shape[1] - 1, dtype=torch.int32)
    with pytest.raises(ValueError, match="p_target"):
        batch.verify(draft, None, torch.zeros(shape), None, None)
    assert batch.seq_len.tolist() == [3, 3] and batch.n_seen.tolist() == [3, 3]
