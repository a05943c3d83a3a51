"""The status that calls on pages share: a call happens whole or not at all,
whenever another one sets it."""
import pytest
import torch

import paper_2608_01657_amd as P
from paper_2608_01657_amd import device as dv

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def pool_of(n_seqs, width, n_pages):
    k = torch.zeros(1, n_pages, 1, 16, 64, dtype=torch.bfloat16, device=DEV)
    return dv.PagePool(k, k.clone(), n_seqs=n_seqs, table_width=width)


@pytest.mark.parametrize("n,blocks", [(200, 90), (8, 300), (300, 3)])
def test_a_status_set_meanwhile_stops_a_fork_or_a_free_whole(n, blocks):
    """Another stream sets the status at some time or other while sequences are forked and freed: all
    children have all pages, or none has any."""
    pool = pool_of(2 * n, blocks, n * blocks)
    parent, child = torch.arange(n, dtype=torch.int32, device=DEV), torch.arange(n, 2 * n, dtype=torch.int32, device=DEV)
    pool.extend(parent, i32([16 * blocks] * n))
    assert int(pool.status) == 0
    pages = pool.table[:n].clone()
    here, there = torch.cuda.Stream(), torch.cuda.Stream()
    junk = torch.zeros(1 << 14, device=DEV)
    happened = set()
    torch.cuda.synchronize()
    for step in range(120):
        for what in ("fork", "free"):
            with torch.cuda.stream(there):
                for _ in range(step % 12):
                    junk.add_(1)
                pool.status.fill_(P.PC_EINVAL)
            if what == "fork":
                pool.fork(parent, child, stream=here)
            else:
                pool.free(child, stream=here)
            torch.cuda.synchronize()
            pool.status.zero_()
            held = int((pool.length[n:] > 0).sum())
            assert held in (0, n) and int((pool.length[n:] == 16 * blocks).sum()) == held
            assert (pool.length[:n] == 16 * blocks).all() and torch.equal(pool.table[:n], pages)
            assert (pool.refs == (2 if held else 1)).all()
            if held:
                assert torch.equal(pool.table[n:], pages)
            happened.add((what, held))
            if held and what == "free":     # was stopped
                pool.free(child)
            torch.cuda.synchronize()
    assert ("fork", n) in happened or ("fork", 0) in happened


@pytest.mark.parametrize("n,blocks", [(2, 3), (40, 100)])
def test_lengths_out_of_range_stay_so(n, blocks):
    """Refused and stopped calls leave every length that is in range, and none that is not becomes one."""
    pool = pool_of(n, blocks, n * blocks)
    pool.extend(torch.arange(n // 2, dtype=torch.int32, device=DEV), i32([16 * blocks] * (n // 2)))
    refs, table = pool.refs.clone(), pool.table.clone()
    good = pool.length.clone()
    for bad in (-1, -2 ** 31, 16 * blocks + 1, 2 ** 30, 2 ** 30 + 16, 2 ** 30 + 16 * blocks, 2 ** 31 - 1):
        for status in (0, P.PC_ENOPAGES):
            for f in (lambda: pool.free(torch.arange(n, dtype=torch.int32, device=DEV)),
                      lambda: pool.fork(torch.arange(n // 2, dtype=torch.int32, device=DEV),
                                        torch.arange(n // 2, n, dtype=torch.int32, device=DEV))):
                pool.length.copy_(good)
                pool.length[n - 1] = bad
                pool.status.fill_(status)
                f()
                assert int(pool.status) == (status or P.PC_EINVAL)
                assert torch.equal(pool.length[:n - 1], good[:n - 1])
                assert not 0 <= int(pool.length[n - 1]) <= 16 * blocks
                assert torch.equal(pool.refs, refs) and torch.equal(pool.table, table)
    pool.length.copy_(good)
    pool.status.zero_()
    pool.free(torch.arange(n, dtype=torch.int32, device=DEV))
    assert int(pool.status) == 0 and int(pool.refs.abs().sum()) == 0 and int(pool.length.abs().sum()) == 0


def test_a_batch_with_a_status_of_its_own():
    """What its plan refuses does not stop the pool's calls, nor theirs it."""
    pool = pool_of(4, 3, 12)
    seq = i32([0, 1])
    pool.extend(seq, i32([20, 30]))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    q = torch.ones(2, 1, 64, dtype=torch.bfloat16, device=DEV)
    batch = dv.PrefixBatch(pool, 2, 2, 1, status=status)
    batch.plan(i32([0, 4]), i32([0, 1, 2]))             # no such sequence
    pool.fork(seq, i32([2, 3]))
    assert int(status) == P.PC_EINVAL and int(pool.status) == 0 and pool.length.tolist() == [20, 30, 20, 30]
    status.zero_()
    pool.free(i32([0, 0]))
    batch.plan(seq, i32([0, 1, 2]))
    out = batch.attend(0, q)
    assert int(status) == 0 and int(pool.status) == P.PC_EINVAL and (out == 0).all()     # V of the pool is 0
    for bad in (torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(1, device=DEV),
                torch.zeros(1, dtype=torch.int32)):
        with pytest.raises(ValueError):
            dv.PrefixBatch(pool, 2, 2, 1, status=bad)


@pytest.mark.parametrize("n,blocks", [(3, 5), (30, 60), (40, 100), (2, 700)])
def test_forks_and_frees_in_a_graph(n, blocks):
    """Both ways of a fork and a free, captured, replayed between eager ones, stopped by a status that is set."""
    pool = pool_of(3 * n, blocks, n * blocks + 3)
    at = lambda i: torch.arange(i * n, (i + 1) * n, dtype=torch.int32, device=DEV)
    pool.extend(at(0), i32([16 * blocks - 5] * n))
    table = pool.table[:n].clone()
    graphs = []
    for f in (lambda: pool.fork(at0, at1), lambda: pool.free(at1)):
        at0, at1 = at(0), at(1)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f()
        graphs.append((graph, at0, at1))
    for step in range(4):
        graphs[0][0].replay()
        assert pool.length.tolist() == [16 * blocks - 5] * (2 * n) + [0] * n
        assert torch.equal(pool.table[n:2 * n], table) and pool.refs.tolist() == [2] * (n * blocks) + [0] * 3
        pool.fork(at(1), at(2))
        assert torch.equal(pool.table[2 * n:], table) and int(pool.refs.max()) == 3
        pool.status.fill_(P.PC_ENOPAGES)
        graphs[1][0].replay()
        assert pool.length.tolist() == [16 * blocks - 5] * (3 * n) and int(pool.status) == P.PC_ENOPAGES
        pool.status.zero_()
        graphs[1][0].replay()
        pool.free(at(2))
        assert pool.length.tolist() == [16 * blocks - 5] * n + [0] * (2 * n) and int(pool.refs.max()) == 1
        assert int(pool.status) == 0
