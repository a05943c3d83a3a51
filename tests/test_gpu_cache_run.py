"""The operators together, as a serving loop uses them: prompts keyed by
pc_hash_blocks, their groups found, the shared blocks held once, the rest of
each prompt stored and attended to, then steps of decoding with branches
forked, freed and compacted; on streams, and in captured graphs."""
import math

import pytest
import torch

import paper_2608_01657_amd as P
from paper_2608_01657_amd import device as dv
from paper_2608_01657_amd import tracegen as tg

pytestmark = pytest.mark.gpu
DEV = "cuda"
HEADS, KV, D = 8, 2, 64


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Server:
    """Two layers; K and V of a token are a function of its sequence's tokens up to it, so requests
    that share a prefix share its K and V.  `hist` keeps what the pages should hold."""

    def __init__(self, prompts, n_seqs=24, pages=600, width=24, dtype=torch.bfloat16, seed=0):
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.dtype = dtype
        k = torch.full((2, pages, KV, 16, D), math.nan, device=DEV, dtype=dtype)
        self.pool = dv.PagePool(k, k.clone(), n_seqs=n_seqs, table_width=width)
        self.hist = {}
        self.known = {}
        self.prompts = prompts

    def kv(self, tokens):
        """K and V [2 layers, n, 2, KV, D] of a prompt, equal for equal beginnings."""
        out = []
        for n in range(1, len(tokens) + 1):
            key = tuple(tokens[:n])
            if key not in self.known:
                self.known[key] = torch.randn(2, 2, KV, D, device=DEV, generator=self.gen).to(self.dtype)
            out.append(self.known[key])
        return torch.stack(out, 1)

    def store(self, seqs, new):
        """new: per sequence [2 layers, n, 2, KV, D], its last tokens."""
        off = [0]
        for x in new:
            off.append(off[-1] + x.shape[1])
        cat = torch.cat(new, 1)
        for layer in range(2):
            self.pool.write(layer, i32(seqs), i32(off), cat[layer, :, 0], cat[layer, :, 1])
        for s, x in zip(seqs, new):
            self.hist[s] = torch.cat([self.hist[s], x], 1) if s in self.hist else x

    def expect(self, seqs, q, q_off, layer):
        out = []
        for i, s in enumerate(seqs):
            kv = self.hist[s][layer].double()
            k, v = (kv[:, j].repeat_interleave(HEADS // KV, 1).transpose(0, 1) for j in (0, 1))
            x = q[q_off[i]:q_off[i + 1]].double().transpose(0, 1)
            n, new = k.shape[1], x.shape[1]
            a = torch.matmul(x, k.transpose(1, 2).contiguous()) / math.sqrt(D)
            late = torch.arange(n, device=DEV) >= n - new + torch.arange(new, device=DEV)[:, None] + 1
            w = torch.softmax(a.masked_fill(late, -math.inf), 2)
            out.append((torch.matmul(w, v).transpose(0, 1), torch.matmul(w, v.abs()).transpose(0, 1)))
        return torch.cat([o for o, _ in out]), torch.cat([m for _, m in out])

    def near(self, out, seqs, q, q_off, layer):
        o, mag = self.expect(seqs, q, q_off, layer)
        # weights rounded, results rounded, 32-bit sums (see test_gpu_attn.py)
        tol = 2.0 ** -8 * (mag + o.abs()) + 2.0 ** -12 * mag
        assert ((out.double() - o).abs() <= tol).all(), float(((out.double() - o).abs() - tol).max())


def prompts(seed=3):
    """Two applications, each with a prompt of its own, and one request by itself."""
    tr = tg.onetouch_tiny(seed, 12)
    base = [tr.tokens[int(o):int(o) + 100].tolist() for o in tr.tok_off[:3]]
    body = lambda i: [100000 + 977 * i + j for j in range(5 + 9 * i % 41)]
    return [base[i % 2] + body(i) for i in range(9)] + [base[2][:7]]


def load(sv, stream=None):
    """Every prompt into the pool, the shared blocks of a group stored once and forked."""
    toks = sv.prompts
    flat = torch.tensor([t for p in toks for t in p], dtype=torch.int32, device=DEV)
    lens = [len(p) for p in toks]
    off = [sum(lens[:i]) for i in range(len(lens))]
    key_off = torch.empty(len(toks) + 1, dtype=torch.int64, device=DEV)
    P.pc_block_offsets(i32(lens), key_off)
    keys = torch.empty(sum(n // 16 for n in lens), dtype=torch.int64, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.pc_hash_blocks(flat, torch.tensor(off, dtype=torch.int64, device=DEV), i32(lens), i32([0] * len(lens)), key_off,
                     keys, status)
    g = dv.prefix_groups(keys, key_off, 1)
    assert int(status) == 0 and int(g.status) == 0
    order, goff, shared = g.order.tolist(), g.group_off.tolist(), g.shared.tolist()
    for i in range(int(g.n_groups)):
        members, n = order[goff[i]:goff[i + 1]], 16 * shared[i]
        if n:
            sv.pool.extend(i32(members[:1]), i32([n]))
            sv.store(members[:1], [sv.kv(toks[members[0]][:n])])
            if len(members) > 1:
                sv.pool.fork(i32([members[0]] * (len(members) - 1)), i32(members[1:]))
                for m in members[1:]:
                    sv.hist[m] = sv.hist[members[0]]
    new = [n - (sv.hist[s].shape[1] if s in sv.hist else 0) for s, n in enumerate(lens)]
    seqs = list(range(len(toks)))
    sv.pool.extend(i32(seqs), i32(new))
    sv.store(seqs, [sv.kv(p)[:, len(p) - n:] for p, n in zip(toks, new)])
    return g, seqs, new


def test_prompts_then_decoding_with_branches():
    sv = Server(prompts())
    g, seqs, new = load(sv)
    pool = sv.pool
    assert sorted(x for x in g.shared.tolist() if x) == [6, 6]
    assert int((pool.refs > 1).sum()) == 12                    # held once for all
    q_off = [0]
    for n in new:
        q_off.append(q_off[-1] + n)
    q = torch.randn(q_off[-1], HEADS, D, device=DEV, generator=sv.gen).to(sv.dtype)
    b = dv.PrefixBatch(pool, len(seqs), q_off[-1], HEADS)
    b.plan(i32(seqs), i32(q_off), *g[:4])
    for layer in range(2):
        sv.near(b.attend(layer, q), seqs, q, q_off, layer)
    # decoding: request 2 and 5 fork two branches each; request 0 ends
    pool.free(i32([0]))
    del sv.hist[0]
    pool.fork(i32([2, 2, 5, 5]), i32([10, 11, 12, 13]))
    for p, c in zip([2, 2, 5, 5], [10, 11, 12, 13]):
        sv.hist[c] = sv.hist[p]
    seqs = [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13]
    app = {s: (s if s < 9 else {9: 9, 10: 2, 11: 2, 12: 5, 13: 5}[s]) for s in seqs}
    part = lambda s: 2 if app[s] == 9 else app[s] % 2
    order = sorted(range(len(seqs)), key=lambda i: (min(j for j in range(len(seqs)) if part(seqs[j]) == part(seqs[i])), i))
    sizes = [sum(part(s) == part(seqs[order[0]]) for s in seqs), sum(part(s) == 1 - part(seqs[order[0]]) for s in seqs)]
    goff = [0, sizes[0], sizes[0] + sizes[1], 13]
    shared = [6, 6, 0]
    R = len(seqs)
    groups = [i32(order), i32(goff + [R] * (R + 1 - 4)), i32(shared + [0] * (R - 3)), i32([3])]
    b = dv.PrefixBatch(pool, R, R, HEADS)
    for step in range(20):
        if step % 7 == 5:
            pool.compact()
        pool.extend(i32(seqs), i32([1] * R))
        sv.store(seqs, [torch.randn(2, 1, 2, KV, D, device=DEV, generator=sv.gen).to(sv.dtype) for _ in seqs])
        q = torch.randn(R, HEADS, D, device=DEV, generator=sv.gen).to(sv.dtype)
        b.plan(i32(seqs), torch.arange(R + 1, dtype=torch.int32, device=DEV), *groups)
        for layer in range(2):
            sv.near(b.attend(layer, q), seqs, q, list(range(R + 1)), layer)
    pool.free(i32(seqs))
    assert int(pool.status) == 0 and int(pool.refs.abs().sum()) == 0


def test_a_captured_step_replayed_between_eager_work():
    """Growing, storing, grouping, planning and attending in one graph, replayed as the sequences
    grow; two graphs share the workspaces; eager calls on the same pool in between."""
    sv = Server(prompts(5))
    g, seqs, _ = load(sv)
    pool, R = sv.pool, len(seqs)
    one, off = i32([1] * R), torch.arange(R + 1, dtype=torch.int32, device=DEV)
    sq = i32(seqs)
    b = dv.PrefixBatch(pool, R, R, HEADS)
    kv = torch.zeros(2, R, 2, KV, D, device=DEV, dtype=sv.dtype)
    q = torch.zeros(R, HEADS, D, device=DEV, dtype=sv.dtype)
    out = [torch.zeros_like(q) for _ in range(2)]

    def grow():
        pool.extend(sq, one)
        for layer in range(2):
            pool.write(layer, sq, off, kv[layer, :, 0], kv[layer, :, 1])

    def attend():
        b.plan(sq, off, *g[:4])
        for layer in range(2):
            b.attend(layer, q, out[layer])

    graphs = []
    for f in (grow, attend):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f()
        graphs.append(graph)
    for step in range(18):
        kv.copy_(torch.randn(kv.shape, device=DEV, generator=sv.gen))
        q.copy_(torch.randn(q.shape, device=DEV, generator=sv.gen))
        for s in seqs:
            sv.hist[s] = torch.cat([sv.hist[s], kv[:, s:s + 1]], 1)
        for graph in graphs:
            graph.replay()
        if step % 3 == 0:
            torch.cuda.synchronize()
        for layer in range(2):
            sv.near(out[layer], seqs, q, list(range(R + 1)), layer)
        if step % 5 == 4:       # eager work on the same pool and workspaces
            pool.fork(i32([1, 4]), i32([20, 21]))
            pool.extend(i32([20]), i32([3]))
            pool.free(i32([20, 21]))
            pool.compact()
            again = [torch.empty_like(q) for _ in range(2)]
            b.plan(sq, off)
            for layer in range(2):
                b.attend(layer, q, again[layer])
                sv.near(again[layer], seqs, q, list(range(R + 1)), layer)
    assert int(pool.status) == 0


def test_groups_in_a_captured_graph():
    toks = prompts(6)
    lens = [len(p) // 16 for p in toks]
    keys = torch.randint(-2 ** 62, 2 ** 62, (sum(lens),), device=DEV)
    off = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g = dv.prefix_groups(keys, off, 1)
    for step in range(4):
        keys.copy_(torch.randint(0, 3, (sum(lens),), device=DEV))
        graph.replay()
        eager = dv.prefix_groups(keys, off, 1)
        assert all(torch.equal(a, b) for a, b in zip(g, eager))


def test_the_largest_batches_in_captured_graphs():
    """More LDS than a kernel has without asking: 4,096 requests grouped, 3,000 planned and attended to."""
    keys = torch.randint(0, 900, (4096 * 2,), device=DEV)
    off = torch.arange(0, 4096 * 2 + 1, 2, dtype=torch.int64, device=DEV)
    R, pages = 3000, 3000
    k = torch.randn(1, pages, 1, 16, 64, device=DEV).to(torch.bfloat16)
    v = torch.randn(1, pages, 1, 16, 64, device=DEV).to(torch.bfloat16)
    table = torch.randperm(pages, device=DEV).int().reshape(R, 1).contiguous()
    length = torch.randint(1, 17, (R,), device=DEV).int()
    pool = dv.PagePool(k, v, table=table, length=length)
    q = torch.randn(R, 2, 64, device=DEV).to(torch.bfloat16)
    seq, q_off = torch.arange(R, device=DEV).int(), torch.arange(R + 1, device=DEV).int()
    b, out = dv.PrefixBatch(pool, R, R, 2), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g = dv.prefix_groups(keys, off, 1)
        b.plan(seq, q_off)
        b.attend(0, q, out)
    for _ in range(3):
        keys.random_(0, 900)
        q.normal_()
        length.random_(1, 17)
        graph.replay()
        eager = dv.prefix_groups(keys, off, 1)
        assert all(torch.equal(x, y) for x, y in zip(g, eager)) and int(g.status) == 0 and int(pool.status) == 0
        kk, vv = k[0, table[:, 0].long(), 0].double(), v[0, table[:, 0].long(), 0].double()
        s = torch.matmul(q.double(), kk.transpose(1, 2).contiguous()) / 8
        w = torch.softmax(s.masked_fill((torch.arange(16, device=DEV) >= length[:, None])[:, None], -math.inf), 2)
        o, mag = torch.matmul(w, vv), torch.matmul(w, vv.abs())
        assert ((out.double() - o).abs() <= 2.0 ** -8 * (mag + o.abs()) + 2.0 ** -12 * mag).all()


def test_on_another_stream():
    """All calls on a stream that is not the current one, after work on it that they depend on."""
    st = torch.cuda.Stream()
    sv = Server(prompts(7))
    g, seqs, _ = load(sv)
    R = len(seqs)
    q = torch.randn(R, HEADS, D, device=DEV, generator=sv.gen).to(sv.dtype)
    kv = torch.randn(2, R, 2, KV, D, device=DEV, generator=sv.gen).to(sv.dtype)
    sq, one, off = i32(seqs), i32([1] * R), torch.arange(R + 1, dtype=torch.int32, device=DEV)
    b = dv.PrefixBatch(sv.pool, R, R, HEADS)
    for s in seqs:
        sv.hist[s] = torch.cat([sv.hist[s], kv[:, s:s + 1]], 1)
    late_q, late_kv = torch.zeros_like(q), torch.zeros_like(kv)
    big = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        for _ in range(10):
            big = big @ big * 1e-3
        late_q.copy_(q)
        late_kv.copy_(kv)
    sv.pool.extend(sq, one, stream=st)
    for layer in range(2):
        sv.pool.write(layer, sq, off, late_kv[layer, :, 0], late_kv[layer, :, 1], stream=st)
    b.plan(sq, off, *g[:4], stream=st)
    out = [b.attend(layer, late_q, stream=st) for layer in range(2)]
    st.synchronize()
    for layer in range(2):
        sv.near(out[layer], seqs, q, list(range(R + 1)), layer)
    assert int(sv.pool.status) == 0
