"""The memory of PrefixBatch: what it held before, and which streams it is used on."""
import pytest
import torch

from paper_2608_01657_amd import device as dv
from test_gpu_attn import DECODE, DEV, PROMPTS, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [DECODE, PROMPTS], ids=["decode", "prompts"])
def test_memory_of_a_batch_that_is_gone(rows):
    """A new batch of the same shape gets the memory of the last one, with its plan in it: nothing is
    written before the new one has a plan of its own."""
    b = Batch(rows, 8, 2, 64, torch.bfloat16)
    pool = b.upload()
    R, T = len(rows), b.q.shape[0]
    q, seq, q_off, groups = b.q.to(DEV), b.seq.to(DEV), b.q_off.to(DEV), b.groups()
    old = dv.PrefixBatch(pool, R, T, 8)
    old.plan(seq, q_off, *groups)
    out = old.attend(1, q)
    at = old.workspace.data_ptr()
    torch.cuda.synchronize()
    del old
    new = dv.PrefixBatch(pool, R, T, 8)
    assert new.workspace.data_ptr() == at
    untouched = torch.full_like(q, 3.0)
    new.attend(1, q, untouched)
    assert (untouched == 3).all()
    new.plan(seq, q_off, *groups)
    assert torch.equal(new.attend(1, q), out)


def test_a_batch_made_while_a_graph_is_captured():
    b = Batch(DECODE, 8, 2, 64, torch.bfloat16)
    pool = b.upload()
    q, seq, q_off, groups = b.q.to(DEV), b.seq.to(DEV), b.q_off.to(DEV), b.groups()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        batch = dv.PrefixBatch(pool, len(b.rows), q.shape[0], 8)
        batch.plan(seq, q_off, *groups)
        batch.attend(1, q, out, lse)
    exact = b.exact()
    eager = dv.PrefixBatch(pool, len(b.rows), q.shape[0], 8)
    for _ in range(4):
        out.fill_(3)
        lse.fill_(3)
        graph.replay()
        b.near(out, lse, *exact)
        eager.plan(seq, q_off)
        eager.attend(1, q)
        torch.cuda.synchronize()
    assert int(pool.status) == 0
