"""ServeBatch4's bookkeeping on the host (CPU: the caches are CPU tensors, and what
would run on the GPU is replaced by its definition or not reached)."""
import pytest
import torch

import cache4_ref as R
from paper_2608_29539_gb300 import build


@pytest.fixture
def serve(monkeypatch):
    build.build()
    from paper_2608_29539_gb300 import serve

    def append(cache, k, v, seq_len, n_valid=None):
        for x, codes, scales in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
            c, s = R.quantise(x)
            for b in range(k.shape[0]):
                n = k.shape[1] if n_valid is None else int(n_valid[b])
                at = slice(int(seq_len[b]) - n, int(seq_len[b]))
                codes[b, :, at], scales[b, :, at] = c[b, :n].transpose(0, 1), s[b, :n].transpose(0, 1)
        return cache

    monkeypatch.setattr(serve.L, "logo_cache4_append", append)
    monkeypatch.setattr(serve.L, "_need", lambda t, *a: t)
    monkeypatch.setattr(serve.L, "logo_select", lambda *a, **kw: None)
    monkeypatch.setattr(serve.L, "logo_decode_cache4_attn", lambda *a, **kw: None)
    return serve


def _batch(serve, n=3, rows=10):
    return serve.ServeBatch4(serve.Serve4Config(2, n, 4, 2, 64, rows), device="cpu")


def _new(n, x=1.0):
    return torch.full((2, n, 2, 64), x, dtype=torch.bfloat16), torch.ones(2, n, 2, 64, dtype=torch.bfloat16)


def _step(batch, x=1.0):
    n = batch.cfg.n_new
    return batch.step(torch.zeros(2, n, 4, 64), *_new(n, x), torch.ones(2, n))


def test_impossible_sizes(serve):
    for kw in (dict(n=0), dict(n=3, rows=2)):
        with pytest.raises(ValueError):
            _batch(serve, **kw)


def test_what_might_not_fit_is_refused_before_anything_changes(serve):
    batch = _batch(serve)
    batch.fill(*_new(4), torch.tensor([4, 1], dtype=torch.int32))
    assert batch.seq_len.tolist() == [4, 1]
    _step(batch)
    _step(batch)
    assert batch.seq_len.tolist() == [10, 7]
    before = [t.clone() for t in (*batch.cache, batch.seq_len)]
    for call in (lambda: _step(batch), lambda: batch.fill(*_new(1))):
        with pytest.raises(ValueError, match="fit"):
            call()
    assert all(torch.equal(a, b) for a, b in zip(before, (*batch.cache, batch.seq_len)))
    batch.seq_len.fill_(6)  # (drafts were rejected)
    assert batch.recount() == 6
    _step(batch)


def test_full_caches_are_not_written_past(serve):
    """What a replay meets, whose steps nobody counts: the latest rows are overwritten."""
    batch = _batch(serve)
    batch._captured = True
    for i in range(5):
        _step(batch, 2.0 ** i)
    assert batch.seq_len.tolist() == [10, 10]
    k = R.values(batch.cache.k, batch.cache.k_scale)[0, 0, :, 0]
    one = R.values(*R.quantise(_new(1)[0]))[0, 0, 0, 0]  # (what a group of ones is kept as; powers of two scale it)
    assert (k / one).tolist() == [1, 1, 1, 2, 2, 2, 4, 16, 16, 16]


def test_verification(serve, monkeypatch):
    seen = {}

    def probs(logits, **kw):
        seen.update(kw)
        return logits

    monkeypatch.setattr(serve.L, "logo_target_probs", probs)
    monkeypatch.setattr(serve.L, "logo_verify_draft", lambda draft, *a, draft_len=None: (
        torch.zeros(2, 3, dtype=torch.int32), torch.tensor([2, 0], dtype=torch.int32)))
    batch = _batch(serve)
    logits, draft = torch.zeros(2, 3, 5), torch.zeros(2, 2, dtype=torch.int32)
    args = (draft, None, logits, None, None)
    with pytest.raises(ValueError, match="verified"):
        batch.verify(*args)
    _step(batch)
    with pytest.raises(ValueError, match="shape"):
        batch.verify(draft, None, logits[:, :2], None, None)
    batch.verify(*args, penalty="p", temperature="t")
    assert seen == dict(penalty="p", temperature="t", draft=draft)
    assert batch.seq_len.tolist() == [3, 1]
    with pytest.raises(ValueError, match="verified"):
        batch.verify(*args)
    _step(batch)
    batch.fill(*_new(1))
    with pytest.raises(ValueError, match="verified"):
        batch.verify(*args)


@pytest.mark.parametrize("n_valid,want", [([0, 8], [9, 9]), ([1, 5], [10, 6]), ([4, 8], [10, 9]), (None, [10, 9])])
def test_what_a_sequence_brings_joins_where_it_fits(serve, n_valid, want):
    """Once a call was captured nothing is refused: a chunk is as wide as its longest part, and a
    sequence whose own part fits, or that brings none, keeps all its rows."""
    batch = _batch(serve)
    batch.fill(*_new(9, 1.0), torch.tensor([9, 1], dtype=torch.int32))
    batch._captured = True
    held = batch.seq_len.tolist()
    batch.fill(*_new(8, 2.0), None if n_valid is None else torch.tensor(n_valid, dtype=torch.int32))
    assert batch.seq_len.tolist() == want
    k = R.values(batch.cache.k, batch.cache.k_scale)[:, 0, :, 0] / R.values(*R.quantise(_new(1)[0]))[0, 0, 0, 0]
    for b, n in enumerate(n_valid or [8, 8]):
        kept = min(held[b], batch.cfg.rows - n)
        assert k[b, :want[b]].tolist() == [1] * kept + [2] * n


def _off_by_one(t):
    """The same values at an address that is not a multiple of 16 bytes."""
    out = torch.zeros(t.numel() + 1, dtype=t.dtype)[1:].view(t.shape)
    return out.copy_(t)


@pytest.mark.parametrize("which", ["q", "k_new", "v_new"])
def test_what_a_call_of_the_step_refuses_changes_nothing(serve, monkeypatch, which):
    """Contiguous tensors that begin between 16-byte borders, which the entry points refuse."""
    def refusing(real):
        def call(*a, **kw):
            if any(torch.is_tensor(t) and t.dtype is torch.bfloat16 and t.data_ptr() % 16 for t in a):
                raise serve.L.LogoError("a call", serve.L.LOGO_ERR_UNSUPPORTED)
            return real(*a, **kw)
        return call

    for name in ("logo_cache4_append", "logo_decode_cache4_attn"):
        monkeypatch.setattr(serve.L, name, refusing(getattr(serve.L, name)))
    batch = _batch(serve)
    _step(batch)
    before = [t.clone() for t in (*batch.cache, batch.seq_len)]
    x = dict(q=torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16), k_new=_new(3, 8.0)[0], v_new=_new(3)[1], gate_p=torch.ones(2, 3))
    x[which] = _off_by_one(x[which])
    with pytest.raises((ValueError, serve.L.LogoError)):
        batch.step(**x)
    assert all(torch.equal(a, b) for a, b in zip(before, (*batch.cache, batch.seq_len)))
    _step(batch)
    _step(batch)
    assert batch.seq_len.tolist() == [9, 9]


def test_configurations_that_no_step_takes(serve):
    """What the calls of a step would refuse each time is refused at once."""
    for kw in (dict(Hq=5), dict(D=96), dict(n_new=5000, rows=5000), dict(mode=7), dict(mode=1, ratio=1.5),
               dict(scale=-1.0), dict(scale=float("nan")), dict(scale=1e39)):
        with pytest.raises(ValueError):
            serve.ServeBatch4(serve.Serve4Config(**(dict(B=2, n_new=3, Hq=4, Hkv=2, D=64, rows=10) | kw)), device="cpu")
