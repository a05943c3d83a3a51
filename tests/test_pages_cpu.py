"""The page operators, the groups and the attention without a GPU: what the
host refuses, and with which code, before any device work."""
import ctypes

import pytest

import paper_2608_01657_amd as P

FAKE = 0x10000


def _pool(**kw):
    d = dict(d_k=FAKE, d_v=FAKE, d_refs=FAKE, d_table=FAKE, d_len=FAKE, page_stride=16 * 2 * 64,
             layer_stride=16 * 2 * 64 * 100, n_layers=2, n_pages=100, n_seqs=10, table_width=8, n_kv_heads=2,
             head_dim=64, dtype=P.PC_BF16, layout=P.PC_HEADS_FIRST)
    d.update(kw)
    return P.pc_pages(**d)


def _rows(**kw):
    d = dict(d_data=FAKE, token_stride=128, head_stride=64)
    d.update(kw)
    return P.pc_rows(**d)


BIG = 1 << 40


def _fork(p, parent=FAKE, child=FAKE, n=2, status=FAKE):
    return P.lib().pc_pages_fork(p, parent, child, n, status, None)


def _extend(p, seq=FAKE, add=FAKE, n=2, ws=FAKE, size=BIG, status=FAKE):
    return P.lib().pc_pages_extend(p, seq, add, n, ws, size, status, None)


def _free(p, seq=FAKE, n=2, status=FAKE):
    return P.lib().pc_pages_free(p, seq, n, status, None)


def _compact(p, refs=FAKE, table=FAKE, n_live=FAKE, ws=FAKE, size=BIG, status=FAKE):
    return P.lib().pc_pages_compact(p, refs, table, n_live, ws, size, status, None)


def _write(p, layer=0, seq=FAKE, off=FAKE, n=2, tokens=4, k=None, v=None, status=FAKE):
    return P.lib().pc_pages_write(p, layer, seq, off, n, tokens, k or _rows(), v or _rows(), status, None)


def _groups(keys=FAKE, n_keys=10, off=FAKE, n=2, w=1, out=FAKE, status=FAKE):
    return P.lib().pc_prefix_groups(keys, n_keys, off, n, w, out, FAKE, FAKE, FAKE, status, None)


def _plan(p, seq=FAKE, q_off=FAKE, n=2, tokens=4, heads=4, causal=1, g=(FAKE,) * 4, ws=FAKE, size=BIG, status=FAKE):
    return P.lib().pc_attn_plan(p, seq, q_off, n, tokens, heads, causal, *g, ws, size, status, None)


def _attn(p, layer=0, q=None, n=2, tokens=4, heads=4, scale=0.1, out=None, ws=FAKE, size=BIG):
    return P.lib().pc_attn(p, layer, q or _rows(), n, tokens, heads, scale, out or _rows(), FAKE, ws, size, None)


CALLS = {"fork": _fork, "extend": _extend, "free": _free, "compact": _compact, "write": _write, "plan": _plan,
         "attn": _attn}


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("field,value,code", [
    ("n_pages", 0, P.PC_EINVAL), ("n_pages", P.PC_MAX_POOL_PAGES + 1, P.PC_EINVAL),
    ("n_seqs", 0, P.PC_EINVAL), ("n_seqs", P.PC_MAX_SEQS + 1, P.PC_EINVAL),
    ("table_width", 0, P.PC_EINVAL), ("table_width", (1 << 24) + 1, P.PC_EINVAL),
    ("n_layers", 0, P.PC_EINVAL), ("n_kv_heads", 0, P.PC_EINVAL), ("n_kv_heads", 257, P.PC_EINVAL),
    ("head_dim", 80, P.PC_EUNSUPPORTED), ("head_dim", 0, P.PC_EUNSUPPORTED),
    ("dtype", 2, P.PC_EINVAL), ("dtype", -1, P.PC_EINVAL), ("layout", 2, P.PC_EINVAL),
    ("page_stride", 16 * 2 * 64 - 8, P.PC_EINVAL), ("page_stride", 16 * 2 * 64 + 4, P.PC_EINVAL),
    ("layer_stride", 4, P.PC_EINVAL), ("d_table", None, P.PC_EINVAL), ("d_len", None, P.PC_EINVAL),
    ("d_refs", None, P.PC_EINVAL), ("d_k", None, P.PC_EINVAL), ("d_v", FAKE + 8, P.PC_EINVAL),
    ("d_len", FAKE + 2, P.PC_EINVAL)])
def test_pools_that_are_refused(call, field, value, code):
    assert CALLS[call](_pool(**{field: value})) == code
    assert P.pc_last_error()


@pytest.mark.parametrize("rc", [
    lambda p: _fork(p, n=-1), lambda p: _fork(p, n=11), lambda p: _fork(p, parent=None), lambda p: _fork(p, child=None),
    lambda p: _fork(p, status=None), lambda p: _free(p, n=11), lambda p: _free(p, seq=None),
    lambda p: _free(p, status=FAKE + 1), lambda p: _extend(p, n=11), lambda p: _extend(p, add=None),
    lambda p: _extend(p, ws=None), lambda p: _extend(p, ws=FAKE + 16), lambda p: _compact(p, refs=None),
    lambda p: _compact(p, table=None), lambda p: _compact(p, n_live=None), lambda p: _compact(p, ws=None),
    lambda p: _write(p, layer=2), lambda p: _write(p, layer=-1), lambda p: _write(p, tokens=-1),
    lambda p: _write(p, k=_rows(d_data=None)), lambda p: _write(p, v=_rows(d_data=FAKE + 8)),
    lambda p: _write(p, v=_rows(token_stride=12)), lambda p: _write(p, off=None),
    lambda p: _plan(p, n=0), lambda p: _plan(p, heads=3), lambda p: _plan(p, heads=0), lambda p: _plan(p, tokens=-1),
    lambda p: _plan(p, seq=None), lambda p: _plan(p, q_off=None), lambda p: _plan(p, causal=2),
    lambda p: _plan(p, g=(FAKE, FAKE, None, FAKE)), lambda p: _plan(p, ws=None), lambda p: _plan(p, status=None),
    lambda p: _attn(p, layer=2), lambda p: _attn(p, scale=0.0), lambda p: _attn(p, scale=-1.0),
    lambda p: _attn(p, scale=float("nan")), lambda p: _attn(p, scale=float("inf")),
    lambda p: _attn(p, q=_rows(d_data=None)), lambda p: _attn(p, out=_rows(head_stride=60)),
    lambda p: _attn(p, ws=FAKE + 128)])
def test_arguments_that_are_refused(rc):
    assert rc(_pool()) == P.PC_EINVAL
    assert P.pc_last_error()


def test_what_is_not_implemented():
    assert _plan(_pool(), n=P.PC_MAX_BATCH + 1, tokens=P.PC_MAX_BATCH + 1) == P.PC_EUNSUPPORTED
    assert _plan(_pool(), tokens=1 << 28, heads=64) == P.PC_EUNSUPPORTED     # over 2^31 partial rows
    assert _groups(n=P.PC_MAX_BATCH + 1) == P.PC_EUNSUPPORTED
    assert _extend(_pool(n_seqs=P.PC_MAX_BATCH + 1), n=P.PC_MAX_BATCH + 1) == P.PC_EUNSUPPORTED


@pytest.mark.parametrize("kw", [dict(n=0), dict(w=0), dict(n_keys=-1), dict(keys=None), dict(keys=FAKE + 4),
                                dict(off=None), dict(out=None), dict(status=None)])
def test_groups_refuse(kw):
    assert _groups(**kw) == P.PC_EINVAL


def test_workspaces():
    p = _pool()
    L = P.lib()
    need = L.pc_pages_workspace_bytes(p, 5)
    assert need > 0 and _extend(p, n=5, size=need - 1) == P.PC_ENOMEM
    assert _compact(p, size=L.pc_pages_workspace_bytes(p, 0) - 1) == P.PC_ENOMEM
    need = L.pc_attn_workspace_bytes(p, 2, 4, 4)
    assert need > 0 and _plan(p, size=need - 1) == P.PC_ENOMEM and _attn(p, size=need - 1) == P.PC_ENOMEM
    assert L.pc_pages_workspace_bytes(p, 11) == P.PC_EINVAL
    assert L.pc_attn_workspace_bytes(p, 0, 4, 4) == P.PC_EINVAL


def test_calls_of_nothing_do_nothing():
    p = _pool()
    assert _fork(p, parent=None, child=None, n=0) == P.PC_OK
    assert _free(p, seq=None, n=0) == P.PC_OK
    assert _extend(p, seq=None, add=None, n=0) == P.PC_OK
    assert _write(p, tokens=0) == P.PC_OK
    assert _attn(p, tokens=0) == P.PC_OK
    assert P.pc_last_error() == ""


def test_struct_sizes():
    assert ctypes.sizeof(P.pc_pages) == 88 and ctypes.sizeof(P.pc_rows) == 24
