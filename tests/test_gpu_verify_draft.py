"""logo_verify_draft against the definition (fp32 products, differences and
quotients are single roundings on both sides, so tokens are compared
exactly), and the law of the emitted tokens."""
import math

import numpy as np
import pytest
import torch

import serving_ref as R

pytestmark = pytest.mark.gpu


def _inputs(B, m, V, seed, near=0.3):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((B, m + 1, V), generator=g) * 2
    p = torch.softmax(z, -1)
    q = torch.softmax(z[:, :m] + near * torch.randn((B, m, V), generator=g), -1)
    draft = torch.multinomial(q.reshape(B * m, V), 1, generator=g).view(B, m).int() if m else \
        torch.zeros((B, 0), dtype=torch.int32)
    u = torch.rand((B, m), generator=g)
    e = torch.empty((B, V)).exponential_(1.0, generator=g)
    return draft, q, p, u, e


def _check(draft, q, p, u, e, draft_len=None):
    from paper_2608_29539_gb300 import logo as Lg
    B, m = draft.shape
    dl = None if draft_len is None else torch.tensor(draft_len, dtype=torch.int32, device="cuda")
    tokens, n = Lg.logo_verify_draft(draft.cuda(), q.cuda(), p.cuda(), u.cuda(), e.cuda(), draft_len=dl)
    torch.cuda.synchronize()
    assert Lg.logo_get_device_status() == 0
    want_t, want_n = R.verify(draft.numpy(), q.numpy(), p.numpy(), u.numpy(), e.numpy(),
                              [m] * B if draft_len is None else draft_len)
    assert n.tolist() == want_n.tolist()
    assert np.array_equal(tokens.cpu().numpy(), want_t)
    return tokens, n


@pytest.mark.parametrize("B,m,V", [(1, 1, 1), (1, 4, 2), (3, 2, 31), (7, 3, 1000), (5, 5, 1025), (40, 4, 4099),
                                   (2, 8, 50021), (1, 3, 131072), (300, 1, 513)])
def test_sizes(B, m, V):
    _check(*_inputs(B, m, V, B + m + V))


@pytest.mark.parametrize("B,V", [(130, 2100), (96, 4001), (70, 5002), (57, 6003), (46, 7004), (36, 7205), (9, 9000)])
def test_clusters_of_every_size(B, V):
    _check(*_inputs(B, 2, V, B))


def test_no_drafts():
    _check(*_inputs(6, 0, 777, 3))


def test_ragged_drafts_and_lengths_out_of_range():
    _check(*_inputs(8, 4, 300, 5), draft_len=[0, 1, 2, 3, 4, 9, -2, 4])


def test_all_accepted_and_none():
    draft, q, p, u, e = _inputs(10, 4, 600, 7, near=0.0)
    q = p[:, :4].clone()  # the draft is the target: accepted whatever u
    u[:] = torch.tensor(1.0 - 2.0 ** -24)
    _, n = _check(draft, q, p, u, e)
    assert n.tolist() == [4] * 10
    _, n = _check(draft, q, p, u + 5.0, e)  # no uniform is that large: all rejected, the residual empty
    assert n.tolist() == [0] * 10


def test_zero_probabilities_tokens_out_of_range_and_ties():
    draft, q, p, u, e = _inputs(6, 3, 200, 9)
    p[0, 0, draft[0, 0].long()] = 0  # accepted by u = 0 only if zero probabilities were
    u[0, 0] = 0
    draft[1, 0] = -1
    draft[2, 1] = 200
    draft[3, 0] = 2 ** 31 - 1
    p[4] = 1.0 / 256  # every clock the same, every probability the same: the lowest token
    e[4] = 1.0
    q[4] = 1.0 / 512
    p[5] = 0.0  # nothing to draw from
    tokens, n = _check(draft, q, p, u, e)
    assert n[0] == 0 and n[1] == 0 and n[3] == 0 and n[4] == 3 and n[5] == 0
    assert tokens[4, 3] == 0 and tokens[5].tolist() == [0, -1, -1, -1]


def test_not_a_number_is_rejected_and_never_drawn():
    draft, q, p, u, e = _inputs(3, 2, 100, 11)
    p[0, 0, draft[0, 0].long()] = float("nan")
    q[1, 0, draft[1, 0].long()] = float("nan")
    p[2, :, ::2] = float("nan")
    tokens, n = _check(draft, q, p, u, e)
    assert n[0] == 0 and n[1] == 0


def test_emitted_tokens_follow_the_target():
    """The first emitted token has the target's law, whatever the draft's: 2^16
    trials, each token's count within 6 standard deviations."""
    from paper_2608_29539_gb300 import logo as Lg
    B, V = 1 << 16, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    target = torch.tensor([0.3, 0.05, 0.2, 0.01, 0.1, 0.14, 0.0, 0.2], device="cuda")
    law = torch.tensor([0.05, 0.3, 0.1, 0.1, 0.1, 0.1, 0.2, 0.05], device="cuda")
    p = target.expand(B, 2, V).contiguous()
    q = law.expand(B, 1, V).contiguous()
    draft = torch.multinomial(law, B, replacement=True, generator=g).view(B, 1).int()
    u = torch.rand((B, 1), generator=g, device="cuda")
    e = torch.empty((B, V), device="cuda").exponential_(1.0, generator=g)
    tokens, n = Lg.logo_verify_draft(draft, q, p, u, e)
    count = torch.bincount(tokens[:, 0].long(), minlength=V).double().cpu()
    want = B * target.double().cpu()
    assert ((count - want).abs() <= 6 * (want * (1 - target.double().cpu())).sqrt()).all(), (count, want)
    share = float(n.double().mean())
    accept = float(torch.minimum(target, law).sum())
    assert abs(share - accept) <= 6 * math.sqrt(accept * (1 - accept) / B)


def test_offsets_beyond_32_bits():
    from paper_2608_29539_gb300 import logo as Lg
    B, m, V = 2100, 7, 131072
    p = torch.zeros((B, m + 1, V), device="cuda")
    assert p.numel() > 2 ** 31
    q = torch.zeros((B, m, V), device="cuda")
    draft = torch.full((B, m), V - 1, dtype=torch.int32, device="cuda")
    q[-1, :, V - 1] = 0.5
    p[-1, :m, V - 1] = 0.5
    p[-1, m, V - 2] = 0.25
    u = torch.full((B, m), 0.5, device="cuda")
    e = torch.ones((B, V), device="cuda")
    tokens, n = Lg.logo_verify_draft(draft, q, p, u, e)
    torch.cuda.synchronize()
    assert n[-1] == m and tokens[-1].tolist() == [V - 1] * m + [V - 2]
    assert n[0] == 0 and tokens[0, 0] == 0


def test_captures_in_a_graph_and_runs_on_another_stream():
    from paper_2608_29539_gb300 import logo as Lg
    x = [t.cuda() for t in _inputs(5, 3, 20000, 6)]
    want, n = Lg.logo_verify_draft(*x)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        side, n_side = Lg.logo_verify_draft(*x)
    torch.cuda.current_stream().wait_stream(stream)
    out, n_out = torch.full_like(want, -7), torch.full_like(n, -7)
    ws = Lg.logo_verify_draft_workspace(x[2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Lg.logo_verify_draft(*x, tokens=out, n_accept=n_out, workspace=ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(want, side) and torch.equal(n, n_side)
    assert torch.equal(want, out) and torch.equal(n, n_out)


def test_refusals():
    from paper_2608_29539_gb300 import logo as Lg
    draft, q, p, u, e = (t.cuda() for t in _inputs(2, 2, 50, 1))
    call = Lg.logo_verify_draft
    for bad in ((draft.long(), q, p, u, e), (draft, q[:, :1], p, u, e), (draft, q, p.double(), u, e),
                (draft, q, p, u[:1], e), (draft, q, p, u, e[:, :49]), (draft, q, p[:, 0], u, e),
                (draft.cpu(), q, p, u, e), (draft, q.transpose(0, 1), p, u, e)):
        with pytest.raises(ValueError):
            call(*bad)
    with pytest.raises(ValueError):
        call(draft, q, p, u, e, tokens=torch.zeros(2, 2, dtype=torch.int32, device="cuda"))
    with pytest.raises(Lg.LogoError) as err:
        call(draft, q, p, u, e, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert err.value.code == Lg.LOGO_ERR_WORKSPACE
