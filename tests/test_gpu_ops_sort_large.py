"""Plans of many slots and of very many clusters against a stable sort on the
device: every digit pass (one to three) and every length of tile (2, 4, 8 and
16 rounds of a block)."""
import pytest
import torch

import paper_1902_09527_amd as km

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("n,k", [
    (17_000_003, 3), (17_000_003, 1000), (4_194_305, 4095), (6_000_001, 4096), (5_000_011, 3_000_000),   # 16 rounds
    (3_000_001, 70_000), (900_001, 2 ** 20), (262_145, 2 ** 24 - 1),                                     # 8, 4: two passes
    (6145, 2 ** 24 + 1), (300_007, 2 ** 24 + 1), (5_000_011, 2 ** 25 + 7)])                              # three passes
def test_plan_against_a_stable_sort(n, k):
    print("case", n, k, flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(n + k)
    ids = torch.randint(0, k, (n,), generator=g, device=DEV, dtype=torch.int32)
    where = torch.rand(n, generator=g, device=DEV)
    ids = torch.where(where < 0.02, torch.where(where < 0.01, -5, 2 ** 31 - 1), ids).to(torch.int32)
    ids[: n // 50] = k - 1   # a long run of the last cluster
    plan = km.cluster_sort(ids, k)
    key = torch.where((ids < 0) | (ids >= k), k, ids)
    srt, order = torch.sort(key, stable=True)
    assert torch.equal(plan.order, order.to(torch.int32))
    pos = torch.empty_like(order)
    pos[order] = torch.arange(n, device=DEV)
    assert torch.equal(plan.pos, pos.to(torch.int32))
    assert torch.equal(plan.sorted_ids, torch.where(srt < k, srt, -1).to(torch.int32))
    offsets = torch.searchsorted(srt, torch.arange(k + 1, device=DEV, dtype=srt.dtype))
    assert torch.equal(plan.offsets, offsets.to(torch.int32))
