"""The pages of a cache (PagePool) and the groups of a keyed batch
(prefix_groups) against plain Python, every count, table entry and value."""
import random

import numpy as np
import pytest
import torch

import paper_2608_01657_amd as P
from paper_2608_01657_amd import device as dv
from paper_2608_01657_amd import tracegen as tg

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Model:
    """What include/pc.h says, in lists."""

    def __init__(self, n_pages, n_seqs, width):
        self.refs, self.pages, self.len = [0] * n_pages, [[] for _ in range(n_seqs)], [0] * n_seqs
        self.width = width

    def fork(self, parent, child):
        for p, c in zip(parent, child):
            self.pages[c], self.len[c] = list(self.pages[p]), self.len[p]
            for x in self.pages[p]:
                self.refs[x] += 1

    def free(self, seq):
        for s in seq:
            for x in self.pages[s]:
                self.refs[x] -= 1
            self.pages[s], self.len[s] = [], 0

    def extend(self, seq, add):
        """The pages copied, as (from, to), or None where the pool is short."""
        grow = {}
        for s, a in zip(seq, add):
            if a and self.len[s] % 16 and self.refs[self.pages[s][-1]] > 1:
                grow.setdefault(self.pages[s][-1], []).append(s)
        copied = {s for page, ss in grow.items() for s in (ss[1:] if len(ss) == self.refs[page] else ss)}
        need = [-(-(self.len[s] + a) // 16) - len(self.pages[s]) + (s in copied) for s, a in zip(seq, add)]
        free = [p for p, r in enumerate(self.refs) if r == 0]
        if sum(need) > len(free):
            return None
        moves = []
        for s, a, n in zip(seq, add, need):
            new, free = free[:n], free[n:]
            for x in new:
                self.refs[x] = 1
            if s in copied:
                old = self.pages[s].pop()
                self.refs[old] -= 1
                moves.append((old, new[0]))
            self.pages[s] += new
            self.len[s] += a
        return moves

    def compact(self):
        live = [p for p, r in enumerate(self.refs) if r]
        n = len(live)
        holes = [p for p in range(n) if not self.refs[p]]
        moves = list(zip([p for p in live if p >= n], holes))
        to = dict(moves)
        refs = list(self.refs)
        for a, b in moves:
            refs[b], refs[a] = refs[a], 0
        self.refs = refs
        self.pages = [[to.get(x, x) for x in s] for s in self.pages]
        return n, moves


class Pair:
    """A pool and its model, and the values that its pages should hold."""

    def __init__(self, n_pages, n_seqs, width, layers=2, heads=2, dim=64, dtype=torch.bfloat16, tokens_first=False, seed=0):
        torch.manual_seed(seed)
        shape = (layers, n_pages) + ((16, heads, dim) if tokens_first else (heads, 16, dim))
        k, v = (torch.randn(shape, device=DEV, dtype=dtype) for _ in range(2))
        self.pool = dv.PagePool(k, v, n_seqs=n_seqs, table_width=width, tokens_first=tokens_first)
        self.model = Model(n_pages, n_seqs, width)
        self.k, self.v = k.clone(), v.clone()

    def moved(self, moves):
        if moves:
            a, b = (torch.tensor(x, device=DEV) for x in zip(*moves))
            self.k[:, b], self.v[:, b] = self.k[:, a], self.v[:, a]

    def fork(self, parent, child):
        self.pool.fork(i32(parent), i32(child))
        self.model.fork(parent, child)

    def free(self, seq):
        self.pool.free(i32(seq))
        self.model.free(seq)

    def extend(self, seq, add):
        self.pool.extend(i32(seq), i32(add))
        moves = self.model.extend(seq, add)
        if moves is None:
            assert int(self.pool.status) == P.PC_ENOPAGES
            self.pool.status.zero_()
        else:
            self.moved(moves)

    def compact(self):
        n, moves = self.model.compact()
        assert int(self.pool.compact()) == n
        self.moved(moves)

    def check(self):
        m = self.model
        assert int(self.pool.status) == 0
        assert self.pool.refs.tolist() == m.refs
        assert self.pool.length.tolist() == m.len
        for row, pages in zip(self.pool.table.tolist(), m.pages):
            assert row[:len(pages)] == pages
        assert torch.equal(self.pool.k, self.k) and torch.equal(self.pool.v, self.v)


@pytest.mark.parametrize("seed", range(6))
def test_random_traffic(seed):
    rng = random.Random(seed)
    n_pages, n_seqs, width = ((40, 12, 6), (300, 40, 9), (4097, 70, 20), (9000, 300, 33), (64, 64, 3), (1, 2, 1))[seed]
    t = Pair(n_pages, n_seqs, width, layers=1 + seed % 3, heads=1 + seed % 4, dim=(64, 128)[seed % 2],
             dtype=(torch.bfloat16, torch.float16)[seed // 2 % 2], tokens_first=bool(seed % 2), seed=seed)
    m = t.model
    for _ in range(60):
        held = [s for s in range(n_seqs) if m.len[s]]
        empty = [s for s in range(n_seqs) if not m.len[s]]
        op = rng.random()
        if op < 0.3 and held and empty:
            child = rng.sample(empty, rng.randint(1, len(empty)))
            t.fork([rng.choice(held) for _ in child], child)
        elif op < 0.7:
            seq = rng.sample(range(n_seqs), rng.randint(1, n_seqs))
            t.extend(seq, [min(rng.choice([0, 1, 1, 5, 16, 17, 40]), 16 * width - m.len[s]) for s in seq])
        elif op < 0.85:
            t.free(rng.sample(range(n_seqs), rng.randint(1, n_seqs)))
        else:
            t.compact()
        t.check()


@pytest.mark.parametrize("n_pages", [63, 64, 65, 4095, 4096, 4097, 16383, 16384, 16385, 20481])
def test_pool_sizes(n_pages):
    """Both ways of scanning a pool, at the edges of its words, chunks and of the small pool; full and empty pools."""
    width = n_pages // 6 + 1
    t = Pair(n_pages, 9, width, layers=1, heads=1)
    sizes = [n_pages // 6, n_pages // 3 % width, 5, n_pages // 7]
    t.extend([3, 1, 0, 2], [16 * n for n in sizes])
    t.extend([4], [1])
    t.free([3, 0])
    t.compact()
    t.check()
    t.fork([1, 2, 4], [5, 6, 7])
    t.extend([5, 7, 8], [0, 3, 16 * (n_pages // 6)])
    t.free([1, 2])
    t.check()
    t.compact()
    t.check()
    left = sum(r == 0 for r in t.model.refs)
    while left:             # the last pages of the pool
        n = min(left, width)
        seq = next(s for s in range(9) if not t.model.len[s])
        t.extend([seq], [16 * n - 7])
        left -= n
    t.check()
    t.compact()             # nothing to move
    t.extend([4], [16])     # and none left
    t.free(list(range(9)))
    t.compact()
    t.check()


def test_who_copies_a_shared_page():
    """All holders grow: the first in the list keeps the page.  Some do not: every one that grows copies."""
    t = Pair(64, 8, 4)
    t.extend([0], [20])
    t.fork([0, 0, 0], [3, 1, 2])
    t.check()
    t.extend([2, 0, 3, 1], [1, 1, 1, 1])
    assert t.model.pages[2][1] == 1 and t.model.refs[1] == 1
    t.check()
    t.fork([2, 2], [5, 6])
    t.extend([5, 6, 0], [0, 3, 2])
    t.check()
    t.extend([5, 2], [9, 9])
    t.check()


def test_a_short_pool_is_left_as_it_was():
    t = Pair(6, 8, 8)
    t.extend([0], [50])         # four pages
    t.fork([0, 0, 0], [1, 2, 3])
    before = [x.clone() for x in (t.pool.refs, t.pool.table, t.pool.length)]
    for seq, add in (([0, 1, 2, 3], [1, 1, 1, 1]), ([1, 0], [1, 60]), ([4], [128])):
        t.extend(seq, add)      # three copies, or more, for two free pages
        assert all(torch.equal(a, b) for a, b in zip(before, (t.pool.refs, t.pool.table, t.pool.length)))
    t.extend([1, 0], [1, 1])    # two copies
    t.check()


def test_long_lists_and_wide_tables():
    """More sequences and blocks than one pass of a workgroup."""
    n = 3000
    t = Pair(70000, n, 300, layers=1, heads=1)
    t.extend(list(range(n - 1, -1, -1)), [1 + i % 37 for i in range(n)])
    t.extend([7], [4000])
    t.check()
    t.free(list(range(0, n, 2)))
    t.compact()
    t.fork([7] * (n // 2), list(range(0, n, 2)))
    t.extend(list(range(n)), [1] * n)
    t.check()
    t.free(list(range(n)))
    assert set(t.model.refs) == {0}
    t.compact()
    t.check()


def test_compaction_into_other_arrays():
    """The pool's own arrays, and the pages that moved, stay as they were."""
    t = Pair(200, 20, 12)
    t.extend(list(range(20)), [9 * i for i in range(20)])
    t.fork([19], [0])
    t.free([3, 7, 11, 12, 13])
    pool = t.pool
    refs, table = pool.refs.clone(), pool.table.clone()
    refs_to, table_to = torch.full_like(refs, -5), torch.full_like(table, -5)
    n_live = int(pool.compact(refs_to=refs_to, table_to=table_to))
    assert torch.equal(pool.refs, refs) and torch.equal(pool.table, table)
    old = [list(p) for p in t.model.pages]
    n, moves = t.model.compact()
    assert n == n_live and refs_to.tolist() == t.model.refs
    t.moved(moves)
    assert torch.equal(pool.k, t.k) and torch.equal(pool.v, t.v)
    for row, was, pages, before in zip(table_to.tolist(), table.tolist(), t.model.pages, old):
        assert row[:len(pages)] == pages and row[len(pages):] == was[len(pages):]
        for a, b in zip(before, pages):
            assert torch.equal(pool.k[:, a], pool.k[:, b])


@pytest.mark.parametrize("tokens_first", [False, True])
@pytest.mark.parametrize("dtype,dim,heads", [(torch.bfloat16, 128, 8), (torch.float16, 64, 1), (torch.float16, 128, 3)])
def test_write(tokens_first, dtype, dim, heads):
    t = Pair(400, 12, 40, layers=3, heads=heads, dim=dim, dtype=dtype, tokens_first=tokens_first)
    t.extend(list(range(11)), [1, 16, 17, 100, 333, 5, 31, 640, 2, 48, 20])
    t.fork([4], [11])
    t.extend([11, 4], [7, 1])
    t.check()
    seq = [7, 0, 11, 3, 9, 4, 5]
    new = [640, 1, 7, 40, 0, 1, 3]
    off = np.concatenate([[0], np.cumsum(new)]).tolist()
    wide = torch.randn(off[-1], 2, heads, dim, device=DEV).to(dtype)
    t.pool.write(1, i32(seq), i32(off), wide[:, 0], wide[:, 1])
    for i, s in enumerate(seq):
        for j in range(new[i]):
            pos = t.model.len[s] - new[i] + j
            page, at = t.model.pages[s][pos // 16], pos % 16
            for to, x in ((t.k, wide[off[i] + j, 0]), (t.v, wide[off[i] + j, 1])):
                if tokens_first:
                    to[1, page, at] = x
                else:
                    to[1, page, :, at] = x
    t.check()


def test_lists_that_are_refused_change_nothing():
    t = Pair(100, 10, 6)
    t.extend(list(range(6)), [10, 20, 30, 40, 50, 96])
    pool = t.pool

    def refused(f, code=P.PC_EINVAL):
        f()
        assert int(pool.status) == code
        f()                          # and nothing more while it is set
        pool.fork(i32([0]), i32([9]))
        pool.free(i32([0]))
        pool.extend(i32([0]), i32([1]))
        pool.status.zero_()
        t.check()

    refused(lambda: pool.fork(i32([0, 1]), i32([6, 6])))        # a child twice
    refused(lambda: pool.fork(i32([0]), i32([1])))              # not empty
    refused(lambda: pool.fork(i32([0, 6]), i32([6, 7])))        # a parent among the children
    refused(lambda: pool.fork(i32([0]), i32([10])))
    refused(lambda: pool.fork(i32([-1]), i32([6])))
    refused(lambda: pool.free(i32([2, 2])))
    refused(lambda: pool.free(i32([10])))
    refused(lambda: pool.extend(i32([1, 1]), i32([1, 1])))
    refused(lambda: pool.extend(i32([1]), i32([-1])))
    refused(lambda: pool.extend(i32([5]), i32([1])))            # wider than the table
    refused(lambda: pool.extend(i32([1]), i32([0x7fffffff])))
    refused(lambda: pool.extend(i32([-7]), i32([1])))
    page = int(pool.table[2, 1])                                # page numbers out of the pool
    for bad in (-1, 100, 0x7fffffff):
        pool.table[2, 1] = bad
        for f in (lambda: pool.fork(i32([2]), i32([6])), lambda: pool.free(i32([2])),
                  lambda: pool.extend(i32([2]), i32([1]))):
            f()
            assert int(pool.status) == P.PC_EINVAL
            pool.status.zero_()
        refs, table = torch.empty_like(pool.refs), torch.empty_like(pool.table)
        pool.compact(refs_to=refs, table_to=table)
        assert int(pool.status) == P.PC_EINVAL and int(table[2, 1]) == bad
        pool.status.zero_()
    pool.table[2, 1] = page
    t.model.compact(), t.moved([])
    pool.compact()
    t.check()


def test_writes_that_are_refused():
    t = Pair(100, 6, 6, heads=1)
    t.extend([0, 1, 2], [10, 20, 30])
    t.fork([1], [3])
    x = torch.randn(8, 1, 64, device=DEV).to(torch.bfloat16)
    pool = t.pool
    for seq, off in (([0, 0], [0, 2, 4]), ([9], [0, 1]), ([-1], [0, 1]), ([0], [0, 9]), ([0], [-1, 2]),
                     ([0, 2], [0, 3, 1]), ([1], [0, 2]), ([4], [0, 1])):     # the last two: a shared page, an empty one
        pool.write(0, i32(seq), i32(off), x, x)
        assert int(pool.status) == P.PC_EINVAL
        pool.status.zero_()
    assert torch.equal(pool.k[:, t.model.pages[1][1]], t.k[:, t.model.pages[1][1]])
    page = int(pool.table[2, 1])
    pool.table[2, 1] = 100
    pool.write(0, i32([2]), i32([0, 3]), x, x)
    assert int(pool.status) == P.PC_EINVAL
    pool.status.zero_()
    pool.table[2, 1] = page
    assert torch.equal(pool.k[1], t.k[1]) and torch.equal(pool.v[1], t.v[1])


# ------------------------------------------------------------------ groups

def plain_groups(reqs, w):
    first, leader = {}, []
    for i, ks in enumerate(reqs):
        leader.append(first.setdefault(ks[w - 1], i) if len(ks) >= w else i)
    order = sorted(range(len(reqs)), key=lambda i: (leader[i], i))
    off, shared = [], []
    for p, i in enumerate(order):
        if p == 0 or leader[i] != leader[order[p - 1]]:
            off.append(p)
            members = [j for j in range(len(reqs)) if leader[j] == leader[i]]
            n = min(len(reqs[j]) for j in members)
            same = 0
            while same < n and len({reqs[j][same] for j in members}) == 1:
                same += 1
            shared.append(same if len(members) > 1 else 0)
    R, n = len(reqs), len(off)
    return order, off + [R] * (R + 1 - n), shared + [0] * (R - n), n


def check_groups(reqs, w):
    off = np.concatenate([[0], np.cumsum([len(r) for r in reqs])]).astype(np.int64)
    keys = np.array([k for r in reqs for k in r], dtype=np.uint64).view(np.int64)
    g = dv.prefix_groups(torch.from_numpy(keys).to(DEV), torch.from_numpy(off).to(DEV), w)
    order, goff, shared, n = plain_groups(reqs, w)
    assert int(g.status) == 0 and int(g.n_groups) == n
    assert g.order.tolist() == order and g.group_off.tolist() == goff and g.shared.tolist() == shared


@pytest.mark.parametrize("R,longest,w", [(1, 5, 1), (2, 3, 1), (3, 9, 2), (64, 40, 1), (65, 300, 3), (1000, 60, 4),
                                         (1025, 5, 1), (4096, 30, 2), (17, 3000, 1), (40, 1025, 1024)])
def test_groups(R, longest, w):
    rng = random.Random(R * 31 + w)
    chains = [[rng.getrandbits(64) for _ in range(rng.randint(1, longest))] for _ in range(max(1, R // 6))]
    reqs = []
    for _ in range(R):
        c = rng.choice(chains)
        n = rng.choice([0, len(c), len(c), rng.randint(0, len(c))])
        reqs.append(c[:n] + [rng.getrandbits(64) for _ in range(rng.randint(0, longest - n))])
    check_groups(reqs, w)


def test_groups_with_all_or_no_keys_alike():
    check_groups([[5, 6, 7]] * 4096, 1)
    check_groups([[i] for i in range(4096)], 1)
    check_groups([[]] * 9, 1)
    check_groups([[0] * 2000, [0] * 2000, [0] * 1024 + [1]], 3)
    check_groups([[2 ** 64 - 1], [0], [2 ** 64 - 1]], 1)


def test_groups_of_keyed_traces():
    """Conversations keyed by pc_hash_blocks: turns of one conversation share their context."""
    tr = tg.workload("chat", seeds=[0], n_requests=900)[0][0]
    t = dv.cut_and_hash(dv.upload(tr))
    off = t.key_off.cpu().numpy()
    keys = t.keys.cpu().numpy().view(np.uint64)
    for a, b in ((0, 128), (300, 900)):
        reqs = [keys[off[i]:off[i + 1]].tolist() for i in range(a, b)]
        g = dv.prefix_groups(t.keys[:t.n_keys], t.key_off[a:b + 1].contiguous(), 2)
        order, goff, shared, n = plain_groups(reqs, 2)
        assert int(g.status) == 0 and int(g.n_groups) == n
        assert g.order.tolist() == order and g.group_off.tolist() == goff and g.shared.tolist() == shared
        assert max(shared) > 2


def test_offsets_that_are_refused():
    keys = torch.arange(10, dtype=torch.int64, device=DEV)
    for off in ([0, 5, 11], [0, 6, 5], [-1, 3, 5]):
        g = dv.prefix_groups(keys, torch.tensor(off, dtype=torch.int64, device=DEV), 1)
        assert int(g.status) == P.PC_EINVAL
    with pytest.raises(ValueError):
        dv.prefix_groups(keys, torch.zeros(3, dtype=torch.int32, device=DEV))
    with pytest.raises(P.PCError):
        dv.prefix_groups(keys, torch.zeros(3, dtype=torch.int64, device=DEV), 0)
