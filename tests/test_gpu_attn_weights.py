"""How exact the weights of PrefixBatch are before the product with V: a
request with up to 16 rows a KV head has the same precision in its shared
tokens, whoever else reads them, as in its own.

Tolerance, u = half a step of the type: a K of one element a token makes every
score one exact product, so that 32 bits leave 2^-24 (16 |s| + 4 n + 64) of a
weight (the scale, the exponential, sums of n terms, joins).  A weight in two
pieces is off by u^2 at most, the result by u |o| more.  In one piece it would
be off by up to u: with some ten weights that count, 5e-4 in the mean (bf16)
where results near 0 may be off by 1e-4."""
import math

import pytest
import torch

from paper_2608_01657_amd import device as dv
from test_gpu_attn import DEV, U, Batch

pytestmark = pytest.mark.gpu


def batch(rows, heads, kv_heads, dim, dtype, seed=0):
    b = Batch(rows, heads, kv_heads, dim, dtype, seed=seed)
    # one element of K a token, by its place, so that shared tokens stay alike
    for (k, _), s in zip(b.kv, b.seq.tolist()):
        n = k.shape[0]
        at = torch.arange(n)
        k *= torch.nn.functional.one_hot(at * 7 % dim, dim).to(dtype)[:, None]
        if n:
            pages = b.table[s, :-(-n // 16)].long()
            b.kp[b.layer].transpose(1, 2)[pages[at // 16], at % 16] = k
    b.q *= 2
    return b


def counts(b):
    """Items of more than 16 rows, items of up to 16."""
    head = b.batch.workspace[:12].view(torch.int32).tolist()
    return head[1], head[2]


def check(b, few, grouped=True):
    """`few`: requests with up to 16 rows a KV head."""
    out, lse = b.run(grouped, scale=1.0)
    o, z, tol, _ = b.exact(scale=1.0)
    u, G = U[b.dtype], b.heads // b.kv_heads
    for r, (k, v) in enumerate(b.kv):
        if r not in few:
            continue
        rows = slice(int(b.q_off[r]), int(b.q_off[r + 1]))
        n, new = k.shape[0], rows.stop - rows.start
        s = torch.matmul(b.q[rows].double().transpose(0, 1),
                         k.double().repeat_interleave(G, 1).permute(1, 2, 0)).transpose(0, 1)    # [new, heads, n]
        s = s.masked_fill((torch.arange(n) >= n - new + torch.arange(new)[:, None] + 1)[:, None], -math.inf)
        w = torch.softmax(s, 2)
        mag = torch.einsum("qhn,nhd->qhd", w, v.double().abs().repeat_interleave(G, 1))
        top = s.masked_fill(s == -math.inf, 0).abs().amax(2)
        tol[rows] = (u * u + 2.0 ** -24 * (16 * top + 4 * n + 64))[..., None] * mag * (1 + u) + u * o[rows].abs()
        if b.dtype == torch.float16:
            tol[rows] += n * 2.0 ** -25 * v.abs().max() + 2.0 ** -25
    off = ((out.double().cpu() - o).abs() - tol).amax((1, 2))
    for r in range(len(b.rows)):
        x = off[int(b.q_off[r]):int(b.q_off[r + 1])]
        assert not x.numel() or x.max() <= 0, f"request {r} {b.rows[r]}: {float(x.max())} more than it may"


TYPES = [(torch.bfloat16, 128), (torch.float16, 64), (torch.bfloat16, 64), (torch.float16, 128)]


@pytest.mark.parametrize("dtype,dim", TYPES)
def test_own_tokens(dtype, dim):
    b = batch([(-1, 0, n, 1) for n in (1, 16, 33, 200, 384)] + [(-1, 0, 60, 4)], 8, 2, dim, dtype)
    check(b, range(6), grouped=False)
    assert counts(b)[0] == 0


@pytest.mark.parametrize("dtype,dim", TYPES)
@pytest.mark.parametrize("heads,kv_heads", [(8, 2), (6, 1), (4, 4), (16, 1)])
def test_shared_tokens(heads, kv_heads, dtype, dim):
    """Forty requests that decode behind tokens read once for all."""
    new = lambda i: 1 + i % 2 * (heads // kv_heads <= 8)
    # 16 heads a KV head: 40 tiles apart, 5 together, from 439 tokens on
    blocks = 24 if heads // kv_heads <= 8 else 28
    b = batch([(0, blocks, 1 + i % 37, new(i)) for i in range(40)], heads, kv_heads, dim, dtype, seed=heads)
    check(b, range(40))
    assert counts(b)[0] >= kv_heads


@pytest.mark.parametrize("dtype,dim", TYPES)
def test_shared_tokens_of_prompts_and_decoding_requests(dtype, dim):
    """Between the rows of prompts in the same tiles, some of prompts alone, and requests without a query."""
    rows = [(0, 40, 20, 5), (0, 40, 9, 1), (0, 40, 70, 70), (0, 40, 5, 0), (0, 40, 33, 2), (0, 40, 90, 90), (0, 40, 4, 4)]
    rows += [(0, 40, 1 + i, 1) for i in range(30)] + [(0, 40, 40, 0)]
    b = batch(rows, 8, 2, dim, dtype)
    check(b, [r for r, x in enumerate(rows) if x[3] <= 4])
    assert counts(b)[0] >= 2


@pytest.mark.parametrize("dtype,dim", TYPES[:2])
def test_the_same_answer_alone_and_in_a_group(dtype, dim):
    """A request's result in a group and by itself: both within half a step and what 32 bits leave."""
    rows = [(0, 24, 3 + i, 1) for i in range(40)]
    b = batch(rows, 8, 2, dim, dtype)
    check(b, range(40))
    check(b, range(40), grouped=False)


@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 64), (torch.float16, 64), (torch.float16, 128)])
@pytest.mark.parametrize("new", [1, 40], ids=["decode", "prompt"])
def test_many_small_weights_behind_a_great_one(new, dtype, dim):
    """The first token takes nearly all of each row and has V = 0; 20,000 others, each with 2^-25.4 of its weight,
    have V = 1, so that the result is their share, some 2^-11.1.  Requests enough (all of one sequence) that none is
    split along its tokens.  Off by at most: 2^-32 of the first weight for each token (what a type of few exponents
    loses), u for the weights, u for the result, 2^-24 (16 |s| + 4 n + 64)."""
    R, n, score = 512, 20000 + new, 17.625      # 25.43 powers of two
    pages = -(-n // 16)
    k = torch.zeros(1, pages, 2, 16, dim, dtype=dtype, device=DEV)
    v = torch.ones_like(k)
    k[0, 0, :, 0, 0] = 1
    v[0, 0, :, 0] = 0
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    pool = dv.PagePool(k, v, table=torch.arange(pages, dtype=torch.int32, device=DEV)[None].contiguous(), length=i32([n]))
    q = torch.zeros(R * new, 4, dim, dtype=dtype, device=DEV)
    q[:, :, 0] = score
    b = dv.PrefixBatch(pool, R, R * new, 4)
    b.plan(i32([0] * R), torch.arange(0, R * new + 1, new, dtype=torch.int32, device=DEV))
    out = b.attend(0, q, scale=1.0).double().reshape(R, new, 4 * dim)
    assert int(pool.status) == 0
    seen = torch.arange(n - new, n, dtype=torch.float64, device=DEV)[:, None]     # tokens behind the first
    o = seen * math.exp(-score) / (1 + seen * math.exp(-score))
    u = U[dtype]
    tol = n * 2.0 ** -32 + o * (2 * u + u * u + 2.0 ** -24 * (16 * score + 4 * n + 64))
    assert ((out - o).abs() <= tol).all(), float((out / o - 1).abs().max())
