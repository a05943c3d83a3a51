"""Attention over shared prefixes (PrefixBatch) against the definition in 64
bits, request by request, on the values that the pool holds.

Tolerance, for a row with weights w (their sum 1), values v, u = half a step of
the type: the weights are rounded before the product with V (u sum w|v|), the
result once more (u |o|); 32-bit sums of D products in a score and of n terms
in a row add 2^-24 (2 D sum|q k| scale + 4 n + 64) sum w|v| at most.  Weights
below the type's normal range (fp16) lose at most 2^-25 each, times |v|."""
import math

import pytest
import torch

from paper_2608_01657_amd import device as dv

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


class Batch:
    """rows: per request (group or -1, shared blocks, own tokens, new tokens).  Everything that no
    query may see is NaN: pages nobody holds, places behind a length, other layers."""

    def __init__(self, rows, heads, kv_heads, dim, dtype, tokens_first=False, layers=2, layer=1, seed=0, spare=9,
                 strided=False):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.layer = rows, layer
        blocks = {}
        for grp, b, _, _ in rows:
            if grp >= 0:
                assert blocks.setdefault(grp, b) == b
        n_pages = sum(blocks.values()) + sum(-(-t // 16) for _, _, t, _ in rows) + spare
        ids = torch.randperm(n_pages, generator=g).tolist()
        shape = (16, kv_heads, dim) if tokens_first else (kv_heads, 16, dim)
        room = 3 if strided else 1
        pools = [torch.full((layers, n_pages, room) + shape, math.nan, dtype=dtype) for _ in range(2)]
        self.kp, self.vp = pools[0][:, :, room - 1], pools[1][:, :, room - 1]
        shared = {grp: [ids.pop() for _ in range(b)] for grp, b in blocks.items()}
        width = max(1, max(b * 16 + t for _, b, t, _ in rows) // 16 + 2)
        self.table = torch.full((len(rows) + 3, width), 0x7ffffff0, dtype=torch.int32)
        self.len = torch.zeros(len(rows) + 3, dtype=torch.int32)
        self.seq = torch.randperm(len(rows) + 3, generator=g)[:len(rows)].int()
        self.kv = []
        filled = {}
        for (grp, b, t, new), s in zip(rows, self.seq.tolist()):
            pages = shared.get(grp, []) + [ids.pop() for _ in range(-(-t // 16))]
            n = b * 16 + t if grp >= 0 else t
            self.table[s, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
            self.len[s] = n
            at = torch.arange(n)
            pg = torch.tensor(pages, dtype=torch.long)[at // 16] if n else at
            kv = []
            for pool in (self.kp, self.vp):
                x = torch.randn(n, kv_heads, dim, generator=g).to(dtype)
                if grp in filled:
                    old = filled[grp][len(kv)]
                    x[:len(old)] = old[:n]
                view = pool[layer] if tokens_first else pool[layer].transpose(1, 2)
                view[pg, at % 16] = x
                kv.append(x)
            if grp >= 0:
                filled[grp] = [x[:b * 16].clone() for x in kv]
            self.kv.append(kv)
        q_off = [0]
        for r in rows:
            q_off.append(q_off[-1] + r[3])
        self.q_off = torch.tensor(q_off, dtype=torch.int32)
        self.q = torch.randn(q_off[-1], heads, dim, generator=g).to(dtype)
        self.heads, self.kv_heads, self.dim, self.dtype, self.tokens_first = heads, kv_heads, dim, dtype, tokens_first

    def groups(self):
        first, leader = {}, []
        for r, row in enumerate(self.rows):
            leader.append(first.setdefault(row[0], r) if row[0] >= 0 else r)
        order = sorted(range(len(leader)), key=lambda r: (leader[r], r))
        off, shared = [], []
        for p, r in enumerate(order):
            if p == 0 or leader[r] != leader[order[p - 1]]:
                off.append(p)
                shared.append(self.rows[r][1] if leader.count(leader[r]) > 1 else 0)
        R, n = len(order), len(off)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
        return i32(order), i32(off + [R] * (R + 1 - n)), i32(shared + [0] * (R - n)), i32([n])

    def upload(self):
        # a copy that keeps the strides
        put = lambda x: torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=DEV).copy_(x)
        self.pool = dv.PagePool(put(self.kp), put(self.vp), table=self.table.to(DEV), length=self.len.to(DEV),
                                tokens_first=self.tokens_first)
        return self.pool

    def exact(self, causal=True, scale=None):
        """out, lse, and how far out may be off, all in 64 bits."""
        scale = scale or 1 / math.sqrt(self.dim)
        G = self.heads // self.kv_heads
        out = torch.zeros(self.q.shape, dtype=torch.float64)
        lse = torch.full(self.q.shape[:2], -math.inf, dtype=torch.float64)
        tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
        u = U[self.dtype]
        for r, (k, v) in enumerate(self.kv):
            a, b = int(self.q_off[r]), int(self.q_off[r + 1])
            n, new = k.shape[0], b - a
            if not new or not n:
                continue
            q = self.q[a:b].double()
            kk, vv = (x.double().repeat_interleave(G, 1).transpose(0, 1) for x in (k, v))     # [heads, n, dim]
            s = torch.matmul(q.transpose(0, 1), kk.transpose(1, 2)) * scale                   # [heads, new, n]
            size = torch.matmul(q.abs().transpose(0, 1), kk.abs().transpose(1, 2)).amax(2).t() * scale
            if causal:
                late = torch.arange(n) >= n - new + torch.arange(new)[:, None] + 1
                s = s.masked_fill(late, -math.inf)
            z = torch.logsumexp(s, 2)
            w = torch.exp(s - torch.where(z == -math.inf, torch.zeros_like(z), z)[..., None])
            o = torch.matmul(w, vv).transpose(0, 1)
            mag = torch.matmul(w, vv.abs()).transpose(0, 1)
            e32 = 2.0 ** -24 * (2 * self.dim * size + 4 * n + 64)
            out[a:b], lse[a:b] = o, z.t()
            tol[a:b] = u * (mag + o.abs()) + e32[..., None] * mag
            if self.dtype == torch.float16:
                tol[a:b] += n * 2.0 ** -25 * vv.abs().max() + 2.0 ** -25
            tol_lse[a:b] = e32 + 2.0 ** -22 * z.t().abs().nan_to_num(0, 0, 0)
        return out, lse, tol, tol_lse

    def run(self, grouped=True, causal=True, scale=None):
        pool = self.upload()
        b = dv.PrefixBatch(pool, len(self.rows), self.q.shape[0], self.heads)
        b.plan(self.seq.to(DEV), self.q_off.to(DEV), *(self.groups() if grouped else ()), causal=causal)
        lse = torch.full(self.q.shape[:2], 7.0, device=DEV)
        out = b.attend(self.layer, self.q.to(DEV), lse=lse, scale=scale)
        torch.cuda.synchronize()
        assert int(pool.status) == 0
        self.batch = b
        return out, lse

    def check(self, grouped=True, causal=True, scale=None):
        out, lse = self.run(grouped, causal, scale)
        self.near(out, lse, *self.exact(causal, scale))
        return out, lse

    @staticmethod
    def near(out, lse, o, z, tol, tol_z):
        out, lse = out.double().cpu(), lse.double().cpu()
        none = z == -math.inf
        assert torch.equal(lse == -math.inf, none)
        assert (out[none] == 0).all()
        off = ((out - o).abs() - tol).amax() if out.numel() else 0
        assert off <= 0, f"out is off by {float((out - o).abs().max())}, {float(off)} more than it may"
        bad = (lse - z)[~none].abs() - tol_z[~none]
        assert not bad.numel() or bad.max() <= 0, f"lse is off by {float((lse - z)[~none].abs().max())}"


# rows of a batch: (group, shared blocks, own tokens, new tokens)
ONE = [(-1, 0, 1, 1)]
DECODE = [(0, 7, 5, 1), (1, 3, 33, 1), (0, 7, 16, 1), (-1, 0, 70, 1), (0, 7, 1, 1), (1, 3, 17, 1), (2, 5, 40, 1)]
PROMPTS = [(0, 9, 40, 40), (-1, 0, 150, 130), (0, 9, 100, 3), (1, 2, 64, 64), (1, 2, 17, 1)]
ODD = [(-1, 0, 0, 1), (-1, 0, 3, 9), (0, 2, 0, 1), (0, 2, 0, 5), (-1, 0, 20, 0), (0, 2, 4, 40), (-1, 0, 16, 16),
       (1, 4, 1, 1)]
MANY = [(i % 5, 4 + i % 5, 1 + 7 * i % 45, 1) for i in range(75)]
LONG = [(-1, 0, 5000, 1), (0, 300, 9, 1), (0, 300, 2000, 1), (-1, 0, 3, 1)]
HEADS = [(1, 1), (4, 4), (8, 2), (12, 2), (28, 4), (32, 1), (20, 1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows", [ONE, DECODE, PROMPTS, ODD], ids=["one", "decode", "prompts", "odd"])
def test_batches(rows, dim, dtype):
    Batch(rows, 8, 2, dim, dtype, tokens_first=dim == 64).check()


@pytest.mark.parametrize("heads,kv_heads", HEADS)
@pytest.mark.parametrize("rows", [DECODE, PROMPTS, MANY], ids=["decode", "prompts", "many"])
def test_heads(rows, heads, kv_heads):
    Batch(rows, heads, kv_heads, 128, torch.bfloat16, seed=heads).check()
    Batch(rows, heads, kv_heads, 64, torch.float16, seed=heads, tokens_first=True).check()


# groups that share enough for one pass over it: pairs, several, more rows than a tile, queries that
# see only part of the shared tokens, one empty of own tokens
SHARED = [(0, 70, 5, 1), (1, 90, 33, 1), (0, 70, 16, 1), (-1, 0, 70, 1), (1, 90, 1, 1), (2, 30, 40, 1), (2, 30, 1, 1),
          (2, 30, 15, 3), (2, 30, 90, 2), (3, 65, 0, 9), (3, 65, 0, 1), (3, 65, 33, 33), (3, 65, 20, 60)]


@pytest.mark.parametrize("heads,kv_heads", HEADS)
@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.float16, 64), (torch.bfloat16, 64)])
def test_shared_prefixes(heads, kv_heads, dtype, dim):
    b = Batch(SHARED, heads, kv_heads, dim, dtype, seed=heads, tokens_first=heads % 3 == 0)
    b.check()
    b.check(causal=False)
    b.check(grouped=False)


# the same kinds of groups behind more tokens: two that decode, four, some that see only part of the shared ones
LONGER = [(0, 130, 5, 1), (1, 190, 33, 1), (0, 130, 16, 1), (-1, 0, 70, 1), (1, 190, 1, 1), (2, 100, 40, 1),
          (2, 100, 1, 1), (2, 100, 15, 3), (2, 100, 90, 2), (3, 165, 0, 9), (3, 165, 0, 1), (3, 165, 33, 33),
          (3, 165, 20, 60)]


@pytest.mark.parametrize("heads,kv_heads", HEADS)
@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.float16, 64), (torch.bfloat16, 64)])
def test_longer_shared_prefixes(heads, kv_heads, dtype, dim):
    b = Batch(LONGER, heads, kv_heads, dim, dtype, seed=heads, tokens_first=heads % 3 == 0)
    b.check()
    b.check(causal=False)


@pytest.mark.parametrize("members", [2, 3, 16, 17, 40])
def test_group_sizes(members):
    """Both ways that the plan goes through a group, tiles that are not full, the rule's both sides."""
    for blocks in (1, 9, 64, 130):
        rows = [(i % 2, blocks + i % 2, 1 + 5 * i % 37, 1 + (i == 3) * 4) for i in range(2 * members)] + [(-1, 0, 9, 1)]
        Batch(rows, 8, 2, 64, torch.bfloat16, seed=members).check()


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1023, 1025])
def test_lengths(length):
    for new in {1, min(length, 2), min(length, 17), length}:
        Batch([(-1, 0, length, new)], 4, 2, 64, torch.float16, seed=length).check()
        Batch([(0, 2, length, new), (0, 2, 3, 1), (0, 2, length, 1)], 6, 2, 128, torch.bfloat16, seed=length).check()


def test_long_ranges_are_split_and_joined():
    for dim, dtype in ((128, torch.bfloat16), (64, torch.float16)):
        b = Batch(LONG, 16, 2, dim, dtype)
        b.check()
        b.check(grouped=False)


@pytest.mark.parametrize("rows", [DECODE, PROMPTS, ODD], ids=["decode", "prompts", "odd"])
def test_without_mask_and_without_groups(rows):
    b = Batch(rows, 12, 4, 128, torch.bfloat16, tokens_first=True)
    b.check(causal=False)
    b.check(grouped=False)
    b.check(grouped=False, causal=False, scale=0.3)


def test_strided_pages_and_rows():
    """K and V of a page side by side in one tensor, queries and results inside wider ones."""
    b = Batch(DECODE + [(g + 10 if g >= 0 else g, n, t, q) for g, n, t, q in PROMPTS], 8, 2, 128, torch.bfloat16,
              strided=True)
    b.check()
    pool = b.pool
    both = torch.stack([pool.k, pool.v], 2)     # [layers, pages, 2, ...]
    pool = dv.PagePool(both[:, :, 0], both[:, :, 1], table=pool.table, length=pool.length)
    batch = dv.PrefixBatch(pool, len(b.rows), b.q.shape[0], b.heads)
    batch.plan(b.seq.to(DEV), b.q_off.to(DEV), *b.groups())
    wide = torch.full((b.q.shape[0], 3, b.heads, 128), 5.0, dtype=b.dtype, device=DEV)
    wide[:, 1] = b.q.to(DEV)
    q, out = wide[:, 1], wide[:, 2]
    lse = torch.empty(q.shape[:2], device=DEV)
    assert batch.attend(1, q, out, lse) is out
    b.near(out, lse, *b.exact())
    assert (wide[:, 0] == 5).all() and torch.equal(wide[:, 1].cpu(), b.q)
    turned = torch.empty(b.heads, b.q.shape[0], 128, dtype=b.dtype, device=DEV).transpose(0, 1)     # heads outside
    batch.attend(1, q, turned)
    assert torch.equal(turned, out)


def test_one_sequence_twice_and_same_results_every_time():
    b = Batch(DECODE, 8, 2, 128, torch.bfloat16)
    out, lse = b.check()
    seq = b.seq.clone()
    seq[4] = seq[0]
    b.rows = list(b.rows)
    b.rows[4], b.kv[4] = b.rows[0], b.kv[0]
    o, z, tol, tol_z = b.exact()
    batch = dv.PrefixBatch(b.pool, len(b.rows), b.q.shape[0], 8)
    batch.plan(seq.to(DEV), b.q_off.to(DEV), *b.groups())
    got = torch.empty(b.q.shape[:2], device=DEV)
    first = batch.attend(1, b.q.to(DEV), lse=got)
    b.near(first, got, o, z, tol, tol_z)
    for _ in range(5):
        assert torch.equal(batch.attend(1, b.q.to(DEV)), first)


def test_shared_blocks_behind_the_shortest_request():
    """Groups that name more shared blocks than the shortest member holds: the rest is read as its own."""
    b = Batch([(0, 6, 10, 1), (0, 6, 30, 4), (0, 6, 0, 2)], 8, 2, 64, torch.bfloat16)
    b.upload()
    b.len[b.seq[2].item()] = 37
    b.kv[2] = [x[:37] for x in b.kv[2]]
    b.check()


def test_values_at_the_edge_of_the_type():
    """Scores far apart, and a row whose greatest score comes last."""
    b = Batch([(0, 5, 50, 30), (0, 5, 40, 1), (-1, 0, 200, 1)], 8, 2, 128, torch.bfloat16)
    b.q *= 40
    b.check(scale=1.0)
    b = Batch([(0, 5, 50, 30), (0, 5, 40, 1)], 8, 2, 64, torch.float16)
    b.q.fill_(0)
    out, lse = b.check()


def test_far_pages():
    """Offsets past 32 bits: the pages of the batch lie behind 5.7 GB of others."""
    b = Batch(DECODE, 8, 2, 128, torch.bfloat16, layers=1, layer=0)
    pages = 700000
    n = b.kp.shape[1]
    big = [torch.empty((1, pages) + b.kp.shape[2:], dtype=b.dtype, device=DEV) for _ in range(2)]
    for to, x in zip(big, (b.kp, b.vp)):
        to[:, pages - n:] = x.to(DEV)
    held = torch.arange(b.table.shape[1]) < ((b.len + 15) // 16)[:, None]
    pool = dv.PagePool(*big, table=torch.where(held, b.table + (pages - n), b.table).to(DEV), length=b.len.to(DEV))
    batch = dv.PrefixBatch(pool, len(b.rows), b.q.shape[0], 8)
    batch.plan(b.seq.to(DEV), b.q_off.to(DEV), *b.groups())
    lse = torch.empty(b.q.shape[:2], device=DEV)
    b.near(batch.attend(0, b.q.to(DEV), lse=lse), lse, *b.exact())


def test_bad_batches_set_the_status_and_write_nothing():
    b = Batch(DECODE, 8, 2, 64, torch.bfloat16)
    pool = b.upload()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    order, off, shared, n = b.groups()
    R, T = len(b.rows), b.q.shape[0]
    seq, q_off = b.seq.to(DEV), b.q_off.to(DEV)
    change = lambda x, at, v: x.clone().index_put_((i32([at]).long(),), i32([v]))
    for args in ((change(seq, 0, 99), q_off, order, off, shared, n), (change(seq, 0, -1), q_off, order, off, shared, n),
                 (seq, change(q_off, 1, 5), order, off, shared, n), (seq, change(q_off, R, T + 1), order, off, shared, n),
                 (seq, change(q_off, 0, -1), order, off, shared, n), (seq, q_off, change(order, 0, 1), off, shared, n),
                 (seq, q_off, change(order, 0, R), off, shared, n), (seq, q_off, order, change(off, 0, 1), shared, n),
                 (seq, q_off, order, change(off, 1, R + 7), shared, n), (seq, q_off, order, off, shared, i32([R + 1])),
                 (seq, q_off, order, off, shared, i32([-1])), (seq, q_off, order, off, shared, i32([1]))):
        batch = dv.PrefixBatch(pool, R, T, 8)
        batch.plan(*args)
        out = torch.full_like(b.q, 3.0, device=DEV)
        batch.attend(1, b.q.to(DEV), out)
        assert int(pool.status) == -1 and (out == 3).all()
        pool.status.zero_()
    long_ = pool.length.clone()
    pool.length[int(seq[0])] = 16 * b.table.shape[1] + 1
    batch.plan(seq, q_off, order, off, shared, n)
    assert int(pool.status) == -1
    pool.length.copy_(long_)
    batch.plan(seq, q_off, order, off, shared, n)           # the status is still set
    out = torch.full_like(b.q, 3.0, device=DEV)
    batch.attend(1, b.q.to(DEV), out)
    assert (out == 3).all()
    pool.status.zero_()
    batch.plan(seq, q_off, order, off, shared, n)
    lse = torch.empty(b.q.shape[:2], device=DEV)
    b.near(batch.attend(1, b.q.to(DEV), lse=lse), lse, *b.exact())


def test_without_a_plan_of_this_batch_nothing_is_written():
    b = Batch(DECODE, 8, 2, 64, torch.bfloat16)
    pool = b.upload()
    R, T = len(b.rows), b.q.shape[0]
    q, seq, q_off = b.q.to(DEV), b.seq.to(DEV), b.q_off.to(DEV)
    batch = dv.PrefixBatch(pool, R, T, 8)
    batch.workspace.fill_(1)
    out = torch.full_like(q, 3.0)
    batch.attend(1, q, out)                                  # no plan
    assert (out == 3).all()
    batch.plan(seq, q_off, *b.groups())
    other = dv.PagePool(pool.k, pool.v, table=pool.table[:-1].contiguous(), length=pool.length[:-1].contiguous())
    batch.pool = other
    batch.attend(1, q, out)                                  # of a pool with fewer sequences
    assert (out == 3).all()
    batch.pool = pool
    batch.n_heads = 4
    wide = torch.full((T, 4, 64), 3.0, dtype=b.dtype, device=DEV)
    batch.attend(1, q[:, :4], wide)                          # with fewer heads
    assert (wide == 3).all()
    batch.n_heads = 8
    lse = torch.empty(q.shape[:2], device=DEV)
    b.near(batch.attend(1, q, lse=lse), lse, *b.exact())


def test_two_batches_of_a_pool_at_once():
    """Batches with workspaces of their own, on two streams, and each again by itself."""
    b = Batch(MANY, 16, 2, 128, torch.bfloat16)
    pool = b.upload()
    groups, q, seq, q_off = b.groups(), b.q.to(DEV), b.seq.to(DEV), b.q_off.to(DEV)
    batches = [dv.PrefixBatch(pool, len(b.rows), q.shape[0], 16) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(q) for _ in range(6)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(6):
        for x in range(2):
            batches[x].plan(seq, q_off, *(groups if x else ()), stream=streams[x])
            batches[x].attend(1, q, outs[x][i], stream=streams[x])
    torch.cuda.synchronize()
    assert int(pool.status) == 0
    o, z, tol, tol_z = b.exact()
    for x in range(2):
        assert all(torch.equal(outs[x][0], y) for y in outs[x])
        lse = torch.empty(q.shape[:2], device=DEV)
        again = batches[x].attend(1, q, lse=lse)
        assert torch.equal(again, outs[x][0])
        b.near(again, lse, o, z, tol, tol_z)


def test_a_plan_for_thousands_of_requests():
    """More requests than one pass of the planning workgroup; groups of two, many and one."""
    rows = [((i // 2) if i < 1000 else 600 if i < 2400 else -1, 1 if i < 1000 else 2 if i < 2400 else 0, 1 + i % 3, 1)
            for i in range(3000)]
    b = Batch(rows, 2, 1, 64, torch.float16)
    b.check()
    b.check(grouped=False)


def test_a_plan_for_thousands_of_requests_that_share_more():
    """The same, behind prefixes long enough to be read once for all: 300 pairs, 1,300 requests together."""
    rows = [((i // 2, 100, 1 + i % 3, 1) if i < 600 else (600, 24, 1 + i % 3, 1) if i < 1900 else (-1, 0, 1 + i % 3, 1))
            for i in range(2200)]
    Batch(rows, 2, 1, 64, torch.float16).check()


# prompts of many lengths: more tiles of more than 16 rows than there are workgroups, or up to two to a CU;
# beside them single tokens
PACKED = [(-1, 0, 40 + 61 * i % 300, 17 + 7 * i % 24) for i in range(70)]
MIXED = PACKED[:40] + [(i % 3, 40, 1 + 9 * i % 50, 1) for i in range(30)] + [(3, 120, 30, 30), (3, 120, 19, 19)]


@pytest.mark.parametrize("rows", [PACKED, PACKED[:30], MIXED], ids=["packed", "pairs", "mixed"])
@pytest.mark.parametrize("dim,dtype,heads,kv_heads", [(64, torch.bfloat16, 16, 16), (128, torch.float16, 27, 9)])
def test_many_items_of_many_lengths(rows, dim, dtype, heads, kv_heads):
    """Workgroups that take one after another, call after call and in a graph's replays: each item once."""
    b = Batch(rows, heads, kv_heads, dim, dtype)
    first, _ = b.check()
    b.check(grouped=False)
    batch = dv.PrefixBatch(b.pool, len(rows), b.q.shape[0], heads)
    q = b.q.to(DEV)
    batch.plan(b.seq.to(DEV), b.q_off.to(DEV), *b.groups())
    for _ in range(4):
        out = torch.full_like(q, math.nan)
        batch.attend(1, q, out)
        assert torch.equal(out, first)
    out.fill_(math.nan)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        batch.attend(1, q, out)
        batch.attend(1, q, out)
    for _ in range(4):
        out.fill_(math.nan)
        graph.replay()
        assert torch.equal(out, first)
        assert torch.equal(batch.attend(1, q), first)


def test_the_largest_batch():
    rows = [(-1 if i % 7 else i // 700, 3 if i % 7 == 0 else 0, 1 + i % 5, 1 + (i % 900 == 0) * (i % 5))
            for i in range(4096)]
    b = Batch(rows, 2, 1, 64, torch.bfloat16)
    b.check()


def test_arguments_that_python_refuses():
    b = Batch(DECODE, 8, 2, 64, torch.bfloat16)
    pool = b.upload()
    batch = dv.PrefixBatch(pool, len(b.rows), b.q.shape[0], 8)
    seq, q_off, q = b.seq.to(DEV), b.q_off.to(DEV), b.q.to(DEV)
    order, off, shared, n = b.groups()
    for f in (lambda: batch.plan(seq[:-1], q_off), lambda: batch.plan(seq.long(), q_off),
              lambda: batch.plan(b.seq, q_off), lambda: batch.plan(seq, q_off, order),
              lambda: batch.plan(seq, q_off, order, off[:-1], shared, n),
              lambda: batch.attend(1, q.half()), lambda: batch.attend(1, q[:-1]), lambda: batch.attend(1, q[:, :4]),
              lambda: batch.attend(1, q, lse=torch.empty(3, device=DEV)),
              lambda: dv.PagePool(pool.k.float(), pool.v.float(), n_seqs=1, table_width=1),
              lambda: dv.PagePool(pool.k, pool.v), lambda: dv.PagePool(pool.k[:, :, :, :8], pool.v[:, :, :, :8], 1, 1)):
        with pytest.raises(ValueError):
            f()
    assert int(pool.status) == 0
