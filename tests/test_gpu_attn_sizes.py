"""PrefixBatch at the far end of what pc.h allows."""
import pytest
import torch

from paper_2608_01657_amd import device as dv
from test_gpu_attn import Batch

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


@pytest.mark.parametrize("dim", [64])
def test_more_rows_than_a_grid_has_threads(dim):
    """2^26 + 5,000 queries of an empty sequence and of one that is not: zeros, a wave to a row, 2^32 threads."""
    T, new = (1 << 26) + 5000, 3000
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        torch.cuda.empty_cache()
    k = torch.ones(1, 4, 1, 16, dim, dtype=torch.bfloat16, device=DEV)
    pool = dv.PagePool(k, k.clone(), n_seqs=2, table_width=2)
    pool.extend(i32([1]), i32([20]))
    q = torch.zeros(T, 1, dim, dtype=torch.bfloat16, device=DEV)
    out = torch.full_like(q, 3.0)
    batch = dv.PrefixBatch(pool, 2, T, 1)
    batch.plan(i32([0, 1]), i32([0, T - new, T]), causal=False)
    lse = torch.full((T, 1), 3.0, device=DEV)
    batch.attend(0, q, out, lse)
    assert int(pool.status) == 0
    assert not out[:T - new].any() and (lse[:T - new] == -torch.inf).all()
    assert (out[T - new:] == 1).all()
    del batch, q, out, lse
    torch.cuda.empty_cache()


@pytest.mark.parametrize("R", [256, 257, 657, 658])
def test_batches_where_the_plan_changes_its_launch(R):
    """The last and first numbers of requests with fewer threads, and with LDS that is not asked for."""
    Batch([(i % 9 - 1, i % 9 if i % 9 else 0, 1 + i % 5, 1) for i in range(R)], 2, 1, 64, torch.float16).check()


def test_one_of_a_kind_has_any_stride():
    """One token, one head, one page: torch's strides of them are not multiples of 8."""
    k = torch.randn(1, 16, 1, 64, 1, device=DEV).to(torch.float16).permute(0, 4, 2, 1, 3)    # one page, one head
    v = torch.randn(1, 16, 1, 64, 1, device=DEV).to(torch.float16).permute(0, 4, 2, 1, 3)
    assert k.stride(1) == 1
    pool = dv.PagePool(k, v, n_seqs=1, table_width=1)
    pool.extend(i32([0]), i32([9]))
    new = torch.randn(1, 64, 1, device=DEV).to(torch.float16).permute(0, 2, 1)
    assert new.stride(1) == 1
    pool.write(0, i32([0]), i32([0, 1]), new, new)
    assert torch.equal(k[0, 0, 0, 8], new[0, 0]) and torch.equal(v[0, 0, 0, 8], new[0, 0])
    q = torch.randn(4, 64, 1, device=DEV).to(torch.float16).permute(2, 0, 1)     # one token
    out = torch.zeros(4, 64, 1, device=DEV, dtype=torch.float16).permute(2, 0, 1)
    assert q.stride(0) == 1
    batch = dv.PrefixBatch(pool, 1, 1, 4)
    for stream in (None, 0):
        batch.plan(i32([0]), i32([0, 1]), stream=stream)
        batch.attend(0, q, out, stream=stream)
    assert int(pool.status) == 0
    s = torch.softmax(q[0].double() @ k[0, 0, 0, :9].double().t() / 8, 1)
    o, mag = s @ v[0, 0, 0, :9].double(), s @ v[0, 0, 0, :9].double().abs()
    assert ((out[0].double() - o).abs() <= 2.0 ** -11 * (mag + o.abs()) + 2.0 ** -13 * mag).all()
