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


def busy(stream):
    """Some milliseconds of work on the stream."""
    with torch.cuda.stream(stream):
        x = torch.ones(4096, 4096, device=DEV)
        for _ in range(40):
            x = x @ x * 1e-4
    return x


def test_results_on_a_raw_handle_belong_to_its_stream():
    """What a call allocates for a stream given by its handle is not handed out to the current one."""
    b = Batch(DECODE, 8, 2, 64, torch.bfloat16)
    pool = b.upload()
    q = b.q.to(DEV)
    batch = dv.PrefixBatch(pool, len(b.rows), q.shape[0], 8)
    seq, q_off, groups = b.seq.to(DEV), b.q_off.to(DEV), b.groups()
    keys, off = torch.arange(4, device=DEV), torch.arange(5, device=DEV)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for handle in (st.cuda_stream, st):
        batch.plan(seq, q_off, *groups, stream=handle)
        out = batch.attend(1, q, stream=handle)
        n_live = pool.compact(refs_to=torch.empty_like(pool.refs), table_to=torch.empty_like(pool.table), stream=handle)
        g = dv.prefix_groups(keys, off, 1, stream=handle)
        torch.cuda.synchronize()
        assert g.order.tolist() == [0, 1, 2, 3] and int(n_live) == 0
        o, _, tol, _ = b.exact()
        assert ((out.double().cpu() - o).abs() <= tol).all()
        at = {x.data_ptr() for x in (out, n_live, g.order)}
        sizes = [(x.shape, x.dtype) for x in (out, n_live)] + [((3 * 4 + 3,), torch.int32)]
        del out, n_live, g
        again = [torch.empty(s, dtype=t, device=DEV) for s, t in sizes for _ in range(3)]
        assert not at & {x.data_ptr() for x in again}
        pool.status.zero_()


@pytest.mark.parametrize("what", ["arguments", "batch", "pool"])
def test_what_is_dropped_while_its_calls_are_queued(what):
    """Memory that a call on another stream still reads is not handed out again, whoever dropped it."""
    b = Batch(PROMPTS, 8, 2, 64, torch.bfloat16)
    exact = b.exact()
    st = torch.cuda.Stream()
    pool = b.upload()
    batch = dv.PrefixBatch(pool, len(b.rows), b.q.shape[0], 8)
    q, seq, q_off, groups = b.q.to(DEV), b.seq.to(DEV), b.q_off.to(DEV), b.groups()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    torch.cuda.synchronize()
    keep = busy(st)
    batch.plan(seq, q_off, *groups, stream=st)
    batch.attend(1, q, out, lse, stream=st)
    dropped = {"arguments": (q, seq, q_off, *groups), "batch": (batch.workspace,),
               "pool": (batch.workspace, pool.k, pool.v, pool.table, pool.length)}[what]
    at = {x.data_ptr() for x in dropped}
    shapes = [(x.shape, x.dtype) for x in dropped]
    del dropped
    if what == "arguments":
        del q, seq, q_off, groups
    else:
        del batch
        b.pool = None
        if what == "pool":
            del pool
    again = [torch.zeros(s, dtype=t, device=DEV) for s, t in shapes]
    if not st.query():      # as long as the calls wait
        assert not at & {x.data_ptr() for x in again}
    torch.cuda.synchronize()
    b.near(out, lse, *exact)
    del keep


def test_arguments_are_refused_alike_on_a_stream():
    b = Batch(DECODE, 8, 2, 64, torch.bfloat16)
    pool = b.upload()
    batch = dv.PrefixBatch(pool, len(b.rows), b.q.shape[0], 8)
    st = torch.cuda.Stream()
    for s in (None, st, st.cuda_stream):
        for f in (lambda: batch.plan(b.seq, b.q_off.to(DEV), stream=s), lambda: batch.attend(1, b.q, stream=s),
                  lambda: pool.free(b.seq, stream=s), lambda: pool.extend(b.seq, b.seq, stream=s)):
            with pytest.raises(ValueError):
                f()
    assert int(pool.status) == 0
