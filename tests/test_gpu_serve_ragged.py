"""ServeBatch.verify where sequences have drafted different numbers of tokens: the
next token after all of a sequence's drafts were accepted comes from the target's
own probabilities, and the rows of the padding leave the caches with the rejected
drafts'."""
import numpy as np
import pytest
import torch

import serving_ref as R

pytestmark = pytest.mark.gpu


def test_sequences_with_fewer_drafts():
    from paper_2608_29539_gb300.serve import ServeBatch, ServeConfig
    B, n, V = 16, 5, 30
    m = n - 1
    g = torch.Generator().manual_seed(7)
    bf = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()  # noqa: E731
    batch = ServeBatch(ServeConfig(B, n, 4, 2, 64, 8, 2))
    batch.step(bf(B, n, 4, 64), bf(B, n, 2, 64), bf(B, n, 2, 64), torch.ones(B, n, device="cuda"))
    p = torch.softmax(torch.randn((B, n, V), generator=g), -1)
    qd = torch.softmax(p[:, :m].log() + 0.3 * torch.randn((B, m, V), generator=g), -1)
    draft = torch.multinomial(qd.view(B * m, V), 1, generator=g).view(B, m).int()
    u, e = torch.rand((B, m), generator=g), torch.empty((B, V)).exponential_(1.0, generator=g)
    lens = torch.tensor([b % (m + 1) for b in range(B)], dtype=torch.int32)
    want_t, want_n = R.verify(draft.numpy(), qd.numpy(), p.numpy(), u.numpy(), e.numpy(), lens.tolist())
    tokens, n_acc = batch.verify(draft.cuda(), qd.cuda(), p.cuda(), u.cuda(), e.cuda(), draft_len=lens.cuda())
    assert np.array_equal(tokens.cpu().numpy(), want_t) and n_acc.tolist() == want_n.tolist()
    assert any(a == k < m for a, k in zip(want_n.tolist(), lens.tolist())) and max(want_n) > 1
    assert batch.seq_len.tolist() == [1 + int(a) for a in want_n]
    assert batch.n_seen.tolist() == [1 + int(a) for a in want_n]
