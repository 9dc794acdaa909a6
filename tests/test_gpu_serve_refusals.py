"""What ServeBatch.step refuses, on the GPU: nothing of the batch changes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("wrong", ["q rows", "q heads", "q type", "gate rows", "gate type", "gate tokens"])
def test_wrong_shapes_and_types(wrong):
    from paper_2608_29539_gb300.serve import ServeBatch, ServeConfig
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    batch = ServeBatch(ServeConfig(2, 3, 4, 2, 64, 8, 2))
    q, k, v, gate = z(2, 3, 4, 64), z(2, 3, 2, 64) + 1, z(2, 3, 2, 64), z(2, 3, dtype=torch.float32) + 1
    bad = {"q rows": (z(3, 3, 4, 64), gate), "q heads": (z(2, 3, 8, 64), gate), "q type": (q.half(), gate),
           "gate rows": (q, z(3, 3, dtype=torch.float32)), "gate type": (q, gate.bfloat16()),
           "gate tokens": (q, z(2, 4, dtype=torch.float32))}[wrong]
    with pytest.raises(ValueError):
        batch.step(bad[0], k, v, bad[1])
    assert batch.seq_len.tolist() == [0, 0] and batch.n_seen.tolist() == [0, 0]
    assert float(batch.k.abs().sum()) == 0 and int(batch.z.sum()) == 0
    batch.step(q, k, v, gate)
    assert batch.seq_len.tolist() == [3, 3] and int(batch.n_sel) == 6
