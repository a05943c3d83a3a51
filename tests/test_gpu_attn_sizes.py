"""PrefixBatch at the far end of what pc.h allows."""
import pytest
import torch

from paper_2608_01657_amd import device as dv

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def counts(batch):
    """Items of more than 16 rows, items of up to 16."""
    head = batch.workspace[:12].view(torch.int32).tolist()
    return head[1], head[2]


@pytest.mark.parametrize("new,at", [(17, 0), (1, 1)], ids=["wide", "narrow"])
def test_a_plan_of_more_work_than_32_bits_count(new, at):
    """4,096 requests of the longest sequence there is (one page in all of its table's 2^24 places): 2^34 blocks of
    work on 256 heads, so that none is split.  Only planned: nobody waits for such an attention."""
    R, heads = 4096, 256
    k = torch.zeros(1, 1, heads, 16, 64, dtype=torch.bfloat16, device=DEV)
    table = torch.zeros(1, 1 << 24, dtype=torch.int32, device=DEV)
    pool = dv.PagePool(k, k.clone(), table=table, length=i32([1 << 28]), refs=i32([1]))
    batch = dv.PrefixBatch(pool, R, R * new, heads)
    batch.plan(i32([0] * R), torch.arange(0, R * new + 1, new, dtype=torch.int32, device=DEV))
    assert int(pool.status) == 0
    n = counts(batch)
    assert n[at] == R * heads and n[1 - at] == 0
    del batch
    torch.cuda.empty_cache()
