"""Workspaces that the library could not write are refused before a launch: it is
handed an address and a size."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _cases():
    from paper_2608_29539_gb300 import logo as L
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    f32 = lambda *s: torch.ones(s, device="cuda")  # noqa: E731
    kc = bf(2, 16, 2, 64)
    yield lambda ws: L.logo_decode_prefix_attn(bf(2, 1, 4, 64), None, None, kc, kc, i32(4, 5), i32(0, 0), i32(0, 1, 2),
                                               i32(2), workspace=ws)
    slot_pos = torch.zeros(2, 2, 16, dtype=torch.int32, device="cuda")
    yield lambda ws: L.logo_cache_evict(kc, kc.clone(), f32(2, 2, 16), slot_pos, i32(4, 5), i32(4, 5), 4, 1,
                                        workspace=ws)
    yield lambda ws: L.logo_verify_draft(i32(1, 1).view(2, 1), f32(2, 1, 8), f32(2, 2, 8), f32(2, 1), f32(2, 8),
                                         workspace=ws)
    yield lambda ws: L.logo_select(f32(2, 16), L.LOGO_SELECT_THRESHOLD, workspace=ws)
    yield lambda ws: L.logo_decode_global_sparse_attn(bf(2, 4, 64), kc, kc, i32(4, 5), i32(0, 1, 2), i32(2),
                                                      workspace=ws)


@pytest.mark.parametrize("call", range(5))
def test_refused(call):
    run = list(_cases())[call]
    big = 1 << 22
    for ws in (torch.empty(big, dtype=torch.uint8), torch.empty(2 * big, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            run(ws)
    run(torch.empty(big, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    from paper_2608_29539_gb300 import logo as L
    assert L.logo_get_device_status() == 0
