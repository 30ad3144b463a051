"""Steps without rows through the Python calls: an empty plan's append with queries, and with positions on several axes."""
import pytest
import torch

from test_gpu_paged import D, DEV, L, i32  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("axes", [0, 1, 3])
def test_no_rows(L, bits, axes):  # noqa: F811
    cache = (L.alloc_paged_cache if bits == 8 else L.alloc_paged_mx_cache)(2, 2, 4, DEV)
    st = L.alloc_paged_state(2, 4, 4, DEV)
    plan = L.paged_plan(i32([0, 3]), i32([0, 0]), st["held"], st["queue"], st["state"], st["table"], max_rows=0)
    rot = L.Rotary(L.rotary_frequencies(64, device=DEV)[0],
                   axis=torch.arange(32, device=DEV).to(torch.uint8) % 3 if axes == 3 else None)
    k, q = (torch.empty((0, h, D), dtype=torch.bfloat16, device=DEV) for h in (2, 4))
    pos = [None, torch.empty(0, dtype=torch.int32, device=DEV), None, torch.empty((3, 0), dtype=torch.int32, device=DEV)][axes]
    for kw in (dict(q=q), dict(q=q, q_out=q), dict()):
        if bits == 8:
            got = L.paged_append_rotary(cache, k, k, plan, rot, pos=pos, **kw)
        else:
            got = L.paged_mx_append(cache, k, k, plan, rot=rot, pos=pos, **kw)
        assert got.shape == q.shape if kw else got is None
    torch.cuda.synchronize()
    assert all(not bool(x.view(torch.uint8).any()) for x in cache)
