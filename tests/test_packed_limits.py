"""How long tables may be that drafted trees are verified over: both sides of the limit that the header states."""
import ctypes as C

import pytest

from test_kv_ops_args import lib  # noqa: F401
from test_kv_ops_ranges import apart
from test_packed_args import tree


def places(B, T, hkv, group, D, slots):
    R = min(64, T) * group
    chunks = -(-R // (128 if D == 256 else 256))
    front, each = (10, 3 if R > 128 else 2) if D == 64 else (4, 1)
    return min(B, T) * hkv * chunks * (front + each * -(-slots // 128))


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("B,T,hkv,group", [(1024, 1, 8, 16), (1024, 7, 8, 16), (1024, 5000, 8, 16), (1024, 5000, 8, 1), (1024, 1 << 30, 256, 16),
                                           (1000, 1000, 200, 3), (300, 64, 256, 2)])
def test_both_sides_of_the_longest_list(lib, D, B, T, hkv, group):  # noqa: F811
    page, hq = 128, hkv * group

    def cache(pages):
        kv = apart(batch=B, n_kv_heads=hkv, head_dim=D, page_size=page, max_pages=pages, n_pages=1, stride_slot=D, stride_head=page * D,
                   stride_page=hkv * page * D)
        need = lib.pbd_op_tree_attention_workspace_bytes(C.byref(kv), T, hq)
        s = tree(lib, kv, T=T, hq=hq, qs=hq * D, ks=hkv * D, ws=None)  # (no workspace: refused for that at the latest)
        return need, s, lib.pbd_op_last_error()
    room = (1 << 30) // page
    fits = max(n for n in range(0, 24) if (1 << n) <= room and places(B, T, hkv, group, D, page << n) < (1 << 31) - 1)
    lo, hi = 1 << fits, min(room, 2 << fits)
    while hi - lo > 1:  # the most pages that fit
        mid = (lo + hi) // 2
        if places(B, T, hkv, group, D, page * mid) < (1 << 31) - 1:
            lo = mid
        else:
            hi = mid
    if places(B, T, hkv, group, D, page * hi) < (1 << 31) - 1:
        lo = hi
    need, s, why = cache(lo)
    assert need > 0 and s == 2 and b"workspace" in why
    if lo < room:
        need, s, why = cache(lo + 1)
        assert need == 0 and s == 3 and b"places" in why


def test_the_table_of_a_large_server_takes_one_row(lib):  # noqa: F811
    """One row behind tables of 2.8 million slots a sequence, 1024 of them on 8 KV heads: what the call's own rows count."""
    kv = apart(batch=1024, n_kv_heads=8, head_dim=64, page_size=16, max_pages=175000, n_pages=1, stride_slot=64, stride_head=1024, stride_page=8192)
    assert lib.pbd_op_tree_attention_workspace_bytes(C.byref(kv), 1, 128) > 0
    assert lib.pbd_op_tree_attention_workspace_bytes(C.byref(kv), 1 << 20, 128) == 0
