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
