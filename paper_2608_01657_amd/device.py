"""Device-side driver of the hot path: upload a trace, cut and hash it, replay
a batch of instances; and of the cache itself: pages of K and V (PagePool), the
groups of a keyed batch (prefix_groups) and attention that reads a group's
shared prefix once (PrefixBatch).  Only allocation and argument marshalling
happen here; all work runs in libpcreplay's kernels on the current HIP stream
of the tensors' device, or the one given."""
from __future__ import annotations

import contextlib
import math
from dataclasses import dataclass
from typing import List, NamedTuple, Optional, Sequence

import numpy as np
import torch

from . import (make_instance_desc, make_pages, make_rows, phase_counters, make_trace_desc, pc_attn, pc_attn_plan,
               pc_attn_workspace_bytes, pc_block_offsets, pc_get_stats, pc_hash_blocks, pc_pages_compact,
               pc_pages_extend, pc_pages_fork, pc_pages_free, pc_pages_workspace_bytes, pc_pages_write,
               pc_prefix_groups, pc_replay_batch, pc_replay_route_offset, pc_replay_workspace_bytes, pc_replay_workspace_min_bytes,
               stats_to_dicts, PC_ATTN_HEAD_BYTES, PC_BLOCK_TOKENS, PC_ROUTE_GENERAL, PC_STATS_RECORD_BYTES)


@dataclass
class DeviceTrace:
    tokens: torch.Tensor        # int32 [T]
    tok_off: torch.Tensor       # int64 [R]
    length: torch.Tensor        # int32 [R]
    ns: torch.Tensor            # int32 [R] namespace (= accounting group)
    group: torch.Tensor         # uint8 [R]
    contract: torch.Tensor      # uint8 [R]
    prefix: torch.Tensor        # int32 [R] (uint32 values)
    tick: Optional[torch.Tensor]
    n_groups: int
    n_prefix: int
    max_req_blocks: int
    key_off: Optional[torch.Tensor] = None   # int64 [R+1]
    keys: Optional[torch.Tensor] = None      # int64 [K] (uint64 bit patterns)
    status: Optional[torch.Tensor] = None
    n_keys: int = 0

    @property
    def n_req(self) -> int:
        return int(self.length.numel())

    @property
    def n_tokens(self) -> int:
        return int(self.tokens.numel())


def upload(trace, device="cuda") -> DeviceTrace:
    """Copy a tracegen.Trace to device memory."""
    dev = torch.device(device)
    tok = torch.from_numpy(np.ascontiguousarray(trace.tokens, np.int32))
    # allocations from torch's caching allocator are at least 256-byte aligned
    t = DeviceTrace(
        tokens=tok.to(dev),
        tok_off=torch.from_numpy(np.ascontiguousarray(trace.tok_off, np.int64)).to(dev),
        length=torch.from_numpy(np.ascontiguousarray(trace.length, np.int32)).to(dev),
        ns=torch.from_numpy(np.ascontiguousarray(trace.group, np.int32)).to(dev),
        group=torch.from_numpy(np.ascontiguousarray(trace.group, np.uint8)).to(dev),
        contract=torch.from_numpy(np.ascontiguousarray(trace.contract, np.uint8)).to(dev),
        prefix=torch.from_numpy(np.ascontiguousarray(trace.prefix, np.uint32).view(np.int32)).to(dev),
        tick=None if trace.tick is None else torch.from_numpy(np.ascontiguousarray(trace.tick, np.int64)).to(dev),
        n_groups=int(trace.n_groups), n_prefix=int(trace.n_prefix),
        max_req_blocks=int(trace.length.max() // 16) if trace.n_req else 0,
    )
    return t


def alloc_keys(t: DeviceTrace, stream=None):
    """Allocate key_off and keys (sizes come from the host-side lengths)."""
    dev = t.tokens.device
    t.key_off = torch.empty(t.n_req + 1, dtype=torch.int64, device=dev)
    t.status = torch.zeros(1, dtype=torch.int32, device=dev)
    return t


def cut_and_hash(t: DeviceTrace, n_keys: Optional[int] = None, stream=None) -> DeviceTrace:
    """Block offsets then chained keys, on the device."""
    if t.key_off is None:
        alloc_keys(t)
    pc_block_offsets(t.length, t.key_off, stream)
    if t.keys is None:
        if n_keys is None:
            n_keys = int(t.key_off[-1].item())      # one 8-byte read to size the key buffer
        t.n_keys = n_keys
        t.keys = torch.empty(max(n_keys, 1), dtype=torch.int64, device=t.tokens.device)
    t.status.zero_()
    pc_hash_blocks(t.tokens, t.tok_off, t.length, t.ns, t.key_off, t.keys[:t.n_keys] if t.n_keys else t.keys[:0],
                   t.status, stream)
    return t


@dataclass
class KeyDeviceTrace:
    """A replay input given directly as keys (tests craft these)."""
    keys: torch.Tensor
    key_off: torch.Tensor
    group: torch.Tensor
    contract: torch.Tensor
    prefix: torch.Tensor
    tick: Optional[torch.Tensor]
    n_groups: int
    n_prefix: int
    max_req_blocks: int
    n_keys: int


def upload_keys(kt, device="cuda") -> KeyDeviceTrace:
    dev = torch.device(device)
    keys = np.ascontiguousarray(kt.keys, np.uint64).view(np.int64)
    off = np.ascontiguousarray(kt.key_off, np.int64)
    mx = int(np.diff(off).max()) if len(off) > 1 else 0
    return KeyDeviceTrace(
        keys=torch.from_numpy(keys if keys.size else np.zeros(1, np.int64)).to(dev),
        key_off=torch.from_numpy(off).to(dev),
        group=torch.from_numpy(np.ascontiguousarray(kt.group, np.uint8)).to(dev),
        contract=torch.from_numpy(np.ascontiguousarray(kt.contract, np.uint8)).to(dev),
        prefix=torch.from_numpy(np.ascontiguousarray(kt.prefix, np.uint32).view(np.int32)).to(dev),
        tick=None if kt.tick is None else torch.from_numpy(np.ascontiguousarray(kt.tick, np.int64)).to(dev),
        n_groups=int(kt.n_groups), n_prefix=int(kt.n_prefix), max_req_blocks=mx, n_keys=int(keys.size))


def trace_desc(t):
    keys = t.keys[:t.n_keys] if t.n_keys else t.keys[:0]
    return make_trace_desc(keys, t.key_off, t.group, t.contract, t.prefix, t.n_groups, t.n_prefix,
                           t.max_req_blocks, t.tick)


class ReplayBatch:
    """Holds the descriptors, workspace and stats buffer of one batch so the
    same replay can be launched repeatedly (each launch starts from an empty
    cache).  Where device memory has no room for the trace analysis, the
    workspace is allocated without it (the general kernels then replay the
    batch)."""

    def __init__(self, dtraces: Sequence, instances: Sequence, per_request: bool = False):
        self.dtraces = list(dtraces)
        self.instances = list(instances)
        self.tdesc = [trace_desc(t) for t in self.dtraces]
        self.idesc = [make_instance_desc(i) for i in self.instances]
        dev = self.dtraces[0].key_off.device
        empty = lambda nbytes: torch.empty((nbytes + 255) // 256 * 32, dtype=torch.int64, device=dev)
        try:
            self.workspace = empty(pc_replay_workspace_bytes(self.tdesc, self.idesc))
        except torch.OutOfMemoryError:
            self.workspace = empty(pc_replay_workspace_min_bytes(self.tdesc, self.idesc))
        self.stats = torch.zeros(len(self.instances) * PC_STATS_RECORD_BYTES // 8, dtype=torch.int64, device=dev)
        self.per_request = None
        if per_request:
            n = sum(4 * int(self.dtraces[i.trace].key_off.numel() - 1) for i in self.instances)
            self.per_request = torch.zeros(max(n, 1), dtype=torch.int32, device=dev)

    def launch(self, stream=None):
        pc_replay_batch(self.tdesc, self.idesc, self.workspace, self.stats, self.per_request, stream)

    def results(self, stream=None):
        G, S = pc_get_stats(self.stats, len(self.instances), -1, 64, stream)
        ng = [self.dtraces[i.trace].n_groups for i in self.instances]
        return stats_to_dicts(G, S, ng)

    def routes(self) -> List[int]:
        """How the last launch replayed each instance (PC_ROUTE_*)."""
        n, at = len(self.instances), pc_replay_route_offset(self.tdesc, self.idesc, self.workspace.numel() * 8)
        if at == 0:
            return [PC_ROUTE_GENERAL] * n
        torch.cuda.synchronize(self.workspace.device)
        return self.workspace.view(torch.int32)[at // 4:at // 4 + n].tolist()

    def phase_counters(self, stream=None) -> List[dict]:
        """Per-instance phase cycles and event counts (phase-counter library
        only; see paper_2608_01657_amd.use_phase_counters)."""
        G, S = pc_get_stats(self.stats, len(self.instances), -1, 64, stream)
        full = stats_to_dicts(G, S, [64] * len(self.instances))
        return [phase_counters(groups) for groups, _, _ in full]

    def per_request_arrays(self) -> List[np.ndarray]:
        assert self.per_request is not None
        host = self.per_request.cpu().numpy()
        out, off = [], 0
        for i in self.instances:
            n = int(self.dtraces[i.trace].key_off.numel() - 1)
            out.append(host[off:off + 4 * n].reshape(n, 4))
            off += 4 * n
        return out


@dataclass
class TraceView:
    """One trace of a TraceSet as the replay reads it: its requests' rows of
    the set's arrays, with key offsets into the set's whole key buffer."""
    keys: torch.Tensor
    key_off: torch.Tensor
    group: torch.Tensor
    contract: torch.Tensor
    prefix: torch.Tensor
    tick: Optional[torch.Tensor]
    n_groups: int
    n_prefix: int
    max_req_blocks: int
    n_keys: int


class TraceSet:
    """Several traces in one set of device buffers, so that block offsets and
    keys of all of them take one pc_block_offsets and one pc_hash_blocks
    call.  Requests keep their own trace's namespace (group) and token view;
    `views` are what ReplayBatch takes, one per trace."""

    def __init__(self, traces: Sequence, device="cuda"):
        dev = torch.device(device)
        tok_base = np.cumsum([0] + [int(tr.tokens.size) for tr in traces[:-1]], dtype=np.int64)
        self.req_base = np.cumsum([0] + [tr.n_req for tr in traces], dtype=np.int64)
        cat = lambda xs, dt: torch.from_numpy(np.ascontiguousarray(np.concatenate(xs), dt)).to(dev)
        any_tick = any(tr.tick is not None for tr in traces)
        self.dt = DeviceTrace(
            tokens=cat([tr.tokens for tr in traces], np.int32),
            tok_off=cat([np.asarray(tr.tok_off, np.int64) + b for tr, b in zip(traces, tok_base)], np.int64),
            length=cat([tr.length for tr in traces], np.int32),
            ns=cat([tr.group for tr in traces], np.int32),
            group=cat([tr.group for tr in traces], np.uint8),
            contract=cat([tr.contract for tr in traces], np.uint8),
            prefix=cat([np.asarray(tr.prefix, np.uint32).view(np.int32) for tr in traces], np.int32),
            # a trace without ticks counts time in requests (tick = request index)
            tick=cat([tr.tick if tr.tick is not None else np.arange(tr.n_req, dtype=np.int64) for tr in traces],
                     np.int64) if any_tick else None,
            n_groups=max(int(tr.n_groups) for tr in traces), n_prefix=max(int(tr.n_prefix) for tr in traces),
            max_req_blocks=max(int(tr.length.max() // 16) if tr.n_req else 0 for tr in traces))
        self.meta = [(int(tr.n_groups), int(tr.n_prefix), int(tr.length.max() // 16) if tr.n_req else 0)
                     for tr in traces]
        self.views: List[TraceView] = []

    def hash(self, stream=None):
        """Offsets and keys of every trace (one call each); views are made on
        the first call."""
        t = self.dt
        cut_and_hash(t, n_keys=t.n_keys if t.keys is not None else None, stream=stream)
        if not self.views:
            for j, (ng, npfx, mx) in enumerate(self.meta):
                r0, r1 = int(self.req_base[j]), int(self.req_base[j + 1])
                self.views.append(TraceView(
                    keys=t.keys[:t.n_keys] if t.n_keys else t.keys[:0], key_off=t.key_off[r0:r1 + 1],
                    group=t.group[r0:r1], contract=t.contract[r0:r1], prefix=t.prefix[r0:r1],
                    tick=None if t.tick is None else t.tick[r0:r1], n_groups=ng, n_prefix=npfx, max_req_blocks=mx,
                    n_keys=t.n_keys))
        return self

    def trace_keys(self, j) -> np.ndarray:
        """Keys of trace j (host copy)."""
        k0, k1 = int(self.dt.key_off[int(self.req_base[j])].item()), int(self.dt.key_off[int(self.req_base[j + 1])].item())
        return self.dt.keys[k0:k1].cpu().numpy().view(np.uint64)

    def trace_key_off(self, j) -> np.ndarray:
        """Key offsets of trace j relative to its own first key (host copy)."""
        o = self.dt.key_off[int(self.req_base[j]):int(self.req_base[j + 1]) + 1].cpu().numpy()
        return o - o[0]


# ---------------------------------------------------------------------------
# Pages of K and V, and attention over them
# ---------------------------------------------------------------------------

def _need(ok, message):
    if not ok:
        raise ValueError(message)


def _list(x, dev, what, dtype=torch.int32):
    if not (x.dtype is dtype and x.get_device() == dev.index and x.dim() == 1 and x.is_contiguous()):
        raise ValueError(f"{what}: a contiguous one-dimensional {dtype} tensor on {dev}")
    return x


@contextlib.contextmanager
def _other(dev, stream, owner, tensors):
    """`dev` is the current device, and `stream` the one that new tensors belong to.  What a call uses there
    is not handed out again before the stream is done with it: its arguments, and the owner's tensors.  (Of a
    raw handle nobody says how long it lives, so there the caller keeps them; a captured graph's user does so
    anyway.)"""
    with torch.cuda.device(dev):
        if stream is None:
            yield
            return
        known = isinstance(stream, torch.cuda.Stream)
        if not known:
            stream = torch.cuda.ExternalStream(getattr(stream, "cuda_stream", stream), device=dev)
        with torch.cuda.stream(stream):
            if known and not torch.cuda.is_current_stream_capturing():
                if owner is not None:
                    owner._used_on(stream)
                for x in tensors:
                    if x is not None and x.is_cuda:     # others are refused by the call
                        x.record_stream(stream)
            yield


_here = contextlib.nullcontext()


def _on(dev, stream, owner, *tensors):
    return (_here if stream is None and torch.cuda.current_device() == dev.index
            else _other(dev, stream, owner, tensors))


class _Owner:
    """Tensors that belong to an object, kept for the streams that it is used on."""

    def _used_on(self, stream):
        if stream.cuda_stream not in self._streams:
            self._streams.add(stream.cuda_stream)
            for x in self._tensors():
                x.record_stream(stream)


class PagePool(_Owner):
    """The pages of a KV cache and the sequences that hold them: 16 tokens a
    page, K and V [layers, pages, heads, 16, dim], or [layers, pages, 16,
    heads, dim] with tokens_first; the layers and pages may be strided, a page
    is contiguous.  Sequences have numbers 0 .. n_seqs-1.

    The arrays are the pool's: `table` [n_seqs, table_width], `length` and
    `refs` [pages] (holders), all int32; made empty unless given.  `status`
    collects what the calls find wrong on the device (PC_EINVAL, PC_ENOPAGES):
    once it is set, further calls do nothing until it is zeroed.  Every call
    is asynchronous and can be captured into a graph.

    A call goes to the current stream, or to the one given: a torch.cuda.Stream,
    or a raw handle, whose calls' tensors the caller keeps until they are done."""

    def __init__(self, k, v, n_seqs: Optional[int] = None, table_width: Optional[int] = None, table=None, length=None,
                 refs=None, tokens_first: bool = False):
        _need(k.dim() == 5 and k.shape == v.shape and k.dtype == v.dtype and k.device == v.device
              and k.stride() == v.stride(), "k and v: [layers, pages, .., .., dim], alike in shape, type and strides")
        _need(k.is_cuda, "k and v: on a GPU")
        _need(k.dtype in (torch.bfloat16, torch.float16), f"k and v: bfloat16 or float16, not {k.dtype}")
        _need(k.shape[2 if tokens_first else 3] == PC_BLOCK_TOKENS, f"a page has {PC_BLOCK_TOKENS} tokens")
        _need(k[0, 0].is_contiguous(), "a page is contiguous")
        dev = self.device = k.device
        self.k, self.v, self.tokens_first = k, v, tokens_first
        if table is None:
            _need(n_seqs is not None and table_width is not None, "n_seqs and table_width, or table")
            table = torch.full((n_seqs, table_width), -1, dtype=torch.int32, device=dev)
        _need(table.dim() == 2 and table.is_contiguous() and table.dtype == torch.int32 and table.device == dev,
              f"table: a contiguous int32 matrix on {dev}")
        zeros = lambda n: torch.zeros(n, dtype=torch.int32, device=dev)
        self.table = table
        self.length = _list(zeros(table.shape[0]) if length is None else length, dev, "length")
        self.refs = _list(zeros(k.shape[1]) if refs is None else refs, dev, "refs")
        _need(self.length.numel() == table.shape[0], "length: one for each row of the table")
        _need(self.refs.numel() == k.shape[1], "refs: one for each page")
        self.status = zeros(1)
        self.desc = make_pages(k, v, self.refs, self.table, self.length, tokens_first)
        n = pc_pages_workspace_bytes(self.desc, table.shape[0])
        self.workspace = torch.empty(n, dtype=torch.uint8, device=dev)
        self._streams = set()

    def _tensors(self):
        return self.k, self.v, self.table, self.length, self.refs, self.status, self.workspace

    @property
    def n_heads(self) -> int:
        return self.desc.n_kv_heads

    def fork(self, parent, child, stream=None):
        """Sequences child[i], empty, take over parent[i]'s pages and length."""
        _need(parent.numel() == child.numel(), "as many parents as children")
        with _on(self.device, stream, self, parent, child):
            pc_pages_fork(self.desc, _list(parent, self.device, "parent"), _list(child, self.device, "child"),
                          self.status, stream)

    def extend(self, seq, add, stream=None):
        """Sequences seq[i] grow by add[i] tokens: new pages, and a copy of a
        last page that others hold too."""
        _need(seq.numel() == add.numel(), "a length for each sequence")
        with _on(self.device, stream, self, seq, add):
            pc_pages_extend(self.desc, _list(seq, self.device, "seq"), _list(add, self.device, "add"), self.workspace,
                            self.status, stream)

    def free(self, seq, stream=None):
        """Sequences seq[i] give up their pages and are empty."""
        with _on(self.device, stream, self, seq):
            pc_pages_free(self.desc, _list(seq, self.device, "seq"), self.status, stream)

    def compact(self, refs_to=None, table_to=None, stream=None):
        """Pages in use move to the lowest numbers; counts and tables are
        rewritten in place, or to refs_to and table_to.  Returns the number of
        pages in use (a tensor; of no meaning where the status was set)."""
        refs_to = self.refs if refs_to is None else _list(refs_to, self.device, "refs_to")
        table_to = self.table if table_to is None else table_to
        _need(refs_to.numel() == self.refs.numel(), "refs_to: one for each page")
        _need(table_to.shape == self.table.shape and table_to.is_contiguous() and table_to.dtype == torch.int32
              and table_to.device == self.device, "table_to: like the table")
        with _on(self.device, stream, self, refs_to, table_to):
            n_live = torch.empty(1, dtype=torch.int32, device=self.device)
            pc_pages_compact(self.desc, refs_to, table_to, n_live, self.workspace, self.status, stream)
        return n_live

    def write(self, layer: int, seq, new_off, k_new, v_new, stream=None):
        """Rows new_off[i] .. new_off[i+1]-1 of k_new and v_new [tokens, heads,
        dim] become K and V of sequence seq[i]'s last tokens."""
        for x in (k_new, v_new):
            self._rows(x, self.desc.n_kv_heads, "k_new and v_new")
        _need(k_new.shape == v_new.shape, "k_new and v_new are alike")
        _need(new_off.numel() == seq.numel() + 1, "new_off: one more than sequences")
        with _on(self.device, stream, self, seq, new_off, k_new, v_new):
            pc_pages_write(self.desc, layer, _list(seq, self.device, "seq"), _list(new_off, self.device, "new_off"),
                           k_new.shape[0], make_rows(k_new), make_rows(v_new), self.status, stream)

    def _rows(self, x, heads, what):
        dim = self.desc.head_dim
        if not (x.dim() == 3 and x.shape[1] == heads and x.shape[2] == dim and x.dtype is self.k.dtype
                and x.get_device() == self.device.index and x.stride(2) == 1):
            raise ValueError(f"{what}: [tokens, {heads}, {dim}] of {self.k.dtype} on {self.device}, "
                             "the last dimension contiguous")


class PrefixGroups(NamedTuple):
    """A batch in groups that share leading blocks (see pc_prefix_groups)."""
    order: torch.Tensor         # int32 [R] requests, group by group
    group_off: torch.Tensor     # int32 [R+1] where each group begins; R behind the last
    shared: torch.Tensor        # int32 [R] blocks that a group's requests share
    n_groups: torch.Tensor      # int32 [1]
    status: torch.Tensor        # int32 [1]


def prefix_groups(keys, key_off, min_blocks: int = 1, stream=None) -> PrefixGroups:
    """Groups of the requests whose block keys (cut_and_hash: keys, key_off)
    are alike for min_blocks blocks or more, and how many leading blocks each
    group shares."""
    dev = key_off.device
    _need(dev.type == "cuda", "keys and key_off: on a GPU")
    _list(key_off, dev, "key_off", torch.int64)
    _list(keys, dev, "keys", torch.int64)
    R = key_off.numel() - 1
    _need(R >= 1, "key_off: n_req + 1 offsets")
    with _on(dev, stream, None, keys, key_off):
        g = PrefixGroups(*torch.empty(3 * R + 3, dtype=torch.int32, device=dev).split((R, R + 1, R, 1, 1)))
        pc_prefix_groups(keys, key_off, min_blocks, *g, stream)
    return g


class PrefixBatch(_Owner):
    """Attention of a batch over a PagePool: n_req requests with n_tokens
    queries in all, of n_heads heads.  plan() once for the lengths that the
    sequences then have, attend() for every layer.  What plan() finds wrong goes
    to `status` (int32 [1], zeroed), the pool's unless given: a batch that is
    planned on another stream than the pool's calls has one of its own, or its
    errors stop them, and theirs it."""

    def __init__(self, pool: PagePool, n_req: int, n_tokens: int, n_heads: int, status=None):
        self.pool, self.n_req, self.n_tokens, self.n_heads = pool, n_req, n_tokens, n_heads
        if status is not None:
            _need(_list(status, pool.device, "status").numel() == 1, "status: one word")
        self.status = status
        n = pc_attn_workspace_bytes(pool.desc, n_req, n_tokens, n_heads)
        self.workspace = torch.empty(n, dtype=torch.uint8, device=pool.device)
        self.workspace[:PC_ATTN_HEAD_BYTES].zero_()     # memory of a batch that is gone may hold its plan
        self._streams = set()

    def _tensors(self):
        return (self.workspace,) if self.status is None else (self.workspace, self.status)

    def _used_on(self, stream):
        super()._used_on(stream)
        self.pool._used_on(stream)

    def plan(self, seq, q_off, order=None, group_off=None, shared=None, n_groups=None, causal: bool = True,
             stream=None):
        """Request r is sequence seq[r] with the queries q_off[r] ..
        q_off[r+1]-1, its last tokens; order .. n_groups: its groups, as
        prefix_groups gives them, or none."""
        pool, R = self.pool, self.n_req
        _need(seq.numel() == R and q_off.numel() == R + 1, "seq: one for each request, q_off: one more")
        given = [x for x in (order, group_off, shared, n_groups) if x is not None]
        if given:
            _need(len(given) == 4, "groups: all of order, group_off, shared and n_groups, or none")
            _need([x.numel() for x in given] == [R, R + 1, R, 1], "groups of as many requests")
            for x in given:
                _list(x, pool.device, "groups")
        with _on(pool.device, stream, self, seq, q_off, *given):
            pc_attn_plan(pool.desc, _list(seq, pool.device, "seq"), _list(q_off, pool.device, "q_off"), self.n_tokens,
                         self.n_heads, causal, order, group_off, shared, n_groups, self.workspace,
                         pool.status if self.status is None else self.status, stream)

    def attend(self, layer: int, q, out=None, lse=None, scale: Optional[float] = None, stream=None):
        """softmax(scale q K^T) V for q [n_tokens, n_heads, dim], each query
        over the tokens it sees; scale: 1 / sqrt(dim) unless given.  lse
        (float32 [n_tokens, n_heads]): log of each row's sum of exponentials.  Without
        a plan, or one that was refused, out and lse stay as they are."""
        pool = self.pool
        with _on(pool.device, stream, self, q, out, lse):
            if out is None:
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            for x in (q, out):
                pool._rows(x, self.n_heads, "q and out")
                _need(x.shape[0] == self.n_tokens, "q and out: as many tokens as the batch has")
            _need(lse is None or (lse.shape == q.shape[:2] and lse.dtype == torch.float32 and lse.is_contiguous()
                                  and lse.device == pool.device), "lse: a contiguous float32 [tokens, heads]")
            if scale is None:
                scale = 1.0 / math.sqrt(q.shape[2])
            pc_attn(pool.desc, layer, make_rows(q), self.n_req, self.n_tokens, self.n_heads, scale, make_rows(out),
                    lse, self.workspace, stream)
        return out
