"""By which way the plan sends the batches of test_gpu_attn.py and others: read together or by each
request, split or whole, straight to the output or joined, taken from counters, in pairs.  A change of a rule that
leaves a way without a test fails here."""
import pytest
import torch

from test_gpu_attn import (DECODE, LONG, LONGER, MANY, MIXED, ODD, ONE, PACKED, PROMPTS, SHARED, Batch)

pytestmark = pytest.mark.gpu
SLOTS = 512     # workgroups of the items' kernel


class Plan:
    """The lists' lengths, and of each request how many parts its own tokens have (-1: none, they go straight to
    the output) and how many its group's."""

    def __init__(self, b):
        ws = b.batch.workspace
        _, self.wide, self.narrow = ws[:12].view(torch.int32).tolist()
        T, up = b.q.shape[0], lambda n: -(-n // 256) * 256
        at = 256 + up(8 * 32 * 4) + 2 * up(4 * T)
        rows = ws[at:at + 32 * T].view(torch.int32).reshape(T, 8).cpu()
        own, grp = torch.zeros(T, dtype=torch.int32), torch.zeros(T, dtype=torch.int32)
        own[rows[:, 0].long()], grp[rows[:, 0].long()] = rows[:, 1], rows[:, 4]
        first = [int(x) for x, y in zip(b.q_off[:-1], b.q_off[1:]) if y > x]
        self.own, self.grp = own[first].tolist(), grp[first].tolist()


def plan(rows, heads=8, kv_heads=2, dim=64, dtype=torch.bfloat16, grouped=True):
    b = Batch(rows, heads, kv_heads, dim, dtype)
    b.check(grouped)
    return Plan(b)


def test_short_decoding_requests_go_straight_to_the_output():
    for rows in (ONE, DECODE, ODD[:1] + DECODE):
        p = plan(rows)
        assert p.wide == 0 and set(p.own) <= {-1, 0} and not any(p.grp)


def test_prompts_and_decoding_requests_side_by_side():
    p = plan(PROMPTS)
    # the third request: 12 rows, four blocks of tokens, two to an item; the last: one block
    assert p.wide and p.narrow and p.own == [-1, -1, 2, -1, -1] and not any(p.grp)


def test_groups_that_are_read_together_and_others_that_are_not():
    # groups for which (tiles by themselves - tiles together) x tokens is above 1,024 x the ones + 256 x the others
    for rows, heads, kv_heads, expect in ((SHARED, 28, 4, set()), (SHARED, 4, 4, {3}), (LONGER, 28, 4, {0, 1, 2}),
                                          (LONGER, 4, 4, {0, 1, 2, 3}), (MIXED, 27, 9, {0, 1, 2})):
        p = plan(rows, heads, kv_heads)
        assert {g for (g, *_), n in zip([r for r in rows if r[3]], p.grp) if n} == expect
    p = plan([(0, 400, 5, 1), (0, 400, 9, 1)], 4, 4)        # of up to 16 rows together
    assert all(p.grp) and p.narrow and not p.wide
    assert not any(plan(LONGER, 28, 4, grouped=False).grp)


def test_long_ranges():
    p = plan(LONG, 16, 2)
    assert max(p.own) > 4 and min(p.own) in (-1, 1)
    p = plan([(-1, 0, 9000, 40)], 4, 2)
    assert p.wide > 2 and p.own[0] > 1      # of more than 16 rows
    p = plan([(0, 300, 9, 1)] * 24, 16, 2)
    assert max(p.grp) > 1                   # of shared tokens


@pytest.mark.parametrize("dim,dtype,heads,kv_heads", [(64, torch.bfloat16, 16, 16), (128, torch.float16, 27, 9)])
def test_many_items(dim, dtype, heads, kv_heads):
    p = plan(PACKED, heads, kv_heads, dim, dtype)
    assert p.wide > SLOTS and p.narrow == 0                                 # from counters
    p = plan(PACKED[:30], heads, kv_heads, dim, dtype)
    assert SLOTS // 2 < p.wide <= SLOTS and p.narrow == 0                   # in pairs
    p = plan(MIXED, heads, kv_heads, dim, dtype)
    assert p.wide > SLOTS // 2 and p.narrow                                 # from counters, narrow ones beside them


def test_many_groups_of_many_sizes():
    p = plan(MANY, 28, 4)
    assert p.narrow and not p.wide
    rows = [(i % 2, 130 + i % 2, 1 + 5 * i % 37, 1 + (i == 3) * 4) for i in range(80)]
    p = plan(rows)
    assert all(p.grp) and p.wide            # groups of 40: by a wave
    p = plan(rows[:32])
    assert all(p.grp)                       # of 16: by a thread
