"""prefix_groups call after call, and what it leaves behind where it refuses."""
import random

import pytest
import torch

import paper_2608_01657_amd as P
from paper_2608_01657_amd import device as dv
from test_gpu_pages import plain_groups

pytestmark = pytest.mark.gpu
DEV = "cuda"


def upload(reqs):
    off = [0]
    for r in reqs:
        off.append(off[-1] + len(r))
    return (torch.tensor([k for r in reqs for k in r], dtype=torch.int64, device=DEV),
            torch.tensor(off, dtype=torch.int64, device=DEV))


def test_groups_of_one_between_large_ones():
    """A request's workgroup reads and writes the same word: of its first waves and of its last ones, in
    groups of one, of two and of many, the same results every time."""
    rng = random.Random(5)
    reqs = [[i % 3 + 1] * rng.randint(1, 1500) if i % 4 == 0 else [100 + i // 2 if i % 8 < 3 else 1000 + i]
            for i in range(1500)]
    keys, off = upload(reqs)
    order, goff, shared, n = plain_groups(reqs, 1)
    for _ in range(10):
        g = dv.prefix_groups(keys, off, 1)
        assert int(g.status) == 0 and int(g.n_groups) == n
        assert g.order.tolist() == order and g.group_off.tolist() == goff and g.shared.tolist() == shared


def test_refused_offsets_leave_no_groups_to_follow():
    """The arrays of a step's groups, used again by a step whose offsets are refused: the last step's
    groups are still in them, and a plan must not take them for its own."""
    prefix = torch.arange(40, dtype=torch.int64, device=DEV)
    keys, off = torch.cat([prefix, prefix]), torch.tensor([0, 40, 80], dtype=torch.int64, device=DEV)
    g = dv.prefix_groups(keys, off, 1)
    assert int(g.n_groups) == 1 and g.shared.tolist() == [40, 0]
    # two sequences that share nothing, long enough to be read together where they are said to
    pages, T = 82, 64
    k = torch.randn(1, pages, 1, 16, 64, device=DEV).to(torch.bfloat16)
    v = torch.randn(1, pages, 1, 16, 64, device=DEV).to(torch.bfloat16)
    table = torch.arange(pages, dtype=torch.int32, device=DEV).reshape(2, 41).contiguous()
    pool = dv.PagePool(k, v, table=table, length=torch.tensor([656, 656], dtype=torch.int32, device=DEV))
    q = torch.randn(2 * T, 1, 64, device=DEV).to(torch.bfloat16)
    seq = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    q_off = torch.tensor([0, T, 2 * T], dtype=torch.int32, device=DEV)
    batch = dv.PrefixBatch(pool, 2, 2 * T, 1)
    bad = torch.tensor([0, 50, 40], dtype=torch.int64, device=DEV)
    P.pc_prefix_groups(keys, bad, 1, *g)
    assert int(g.status) == P.PC_EINVAL and int(g.n_groups) == -1
    batch.plan(seq, q_off, *g[:4])
    out = torch.full_like(q, 3.0)
    batch.attend(0, q, out)
    assert int(pool.status) == P.PC_EINVAL and (out == 3).all()
    pool.status.zero_()
    P.pc_prefix_groups(keys, off, 1, *g)
    assert int(g.status) == 0 and int(g.n_groups) == 1
