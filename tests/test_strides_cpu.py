"""Strides of what there is one of: torch gives them any value, and no address depends on them."""
import pytest

import paper_2608_01657_amd as P
from test_pages_cpu import _attn, _pool, _rows, _write



@pytest.mark.parametrize("stride", [1, 0, -3, 64])
def test_one_token_or_head_of_any_stride(stride):
    p, one = _pool(), _pool(n_kv_heads=1)
    for rc in (_attn(p, tokens=1, q=_rows(token_stride=stride), size=0), _attn(p, tokens=1, out=_rows(token_stride=stride), size=0),
               _attn(one, heads=1, q=_rows(head_stride=stride), size=0),
               _attn(one, heads=1, out=_rows(head_stride=stride), size=0)):
        assert rc == P.PC_ENOMEM
    if stride % 8:
        for rc in (_attn(p, tokens=2, q=_rows(token_stride=stride), size=0),
                   _attn(p, tokens=1, heads=2, out=_rows(head_stride=stride), size=0),
                   _write(p, tokens=1, v=_rows(head_stride=stride)), _write(p, tokens=2, k=_rows(token_stride=stride))):
            assert rc == P.PC_EINVAL


@pytest.mark.parametrize("stride", [1, 0, 8])
def test_one_page_of_any_stride(stride):
    L = P.lib()
    assert L.pc_pages_workspace_bytes(_pool(n_pages=1, page_stride=stride), 1) > 0
    assert L.pc_pages_workspace_bytes(_pool(n_pages=2, page_stride=stride), 1) == P.PC_EINVAL
