"""What the entry points of the operators on packed rows and pages refuse, before they touch a GPU."""
import ctypes as C

import pytest

from paper_2607_12422_gb300 import pbd
from test_kv_ops_args import A, BAD, BAD_POINTERS, cache, lib  # noqa: F401
from test_kv_ops_ranges import G, OVER, apart

NAN, INF = float("nan"), float("inf")


def assign(lib, B=3, mp=4, ps=16, n=20, lens=A, new=A + G, table=A + 2 * G, held=A + 3 * G, free=A + 4 * G, nf=A + 5 * G, most=10,  # noqa: F811
           starts=A + 6 * G, slots=A + 7 * G, pos=A + 8 * G, ws=A + 9 * G, nb=1024):
    return lib.pbd_op_assign_pages(B, mp, ps, n, lens, new, table, held, free, nf, most, starts, slots, pos, ws, nb, None)


def prompt(lib, T=100, B=3, hq=4, hkv=2, D=128, dt=pbd.PBD_BF16, scale=1.0, q=A + 10 * G, qs=512, k=A + 11 * G, v=A + 12 * G, ks=256,  # noqa: F811
           starts=A + 13 * G, kv=None, slots=None, out=A + 14 * G, lse=A + 15 * G, ws=A + 16 * G, nb=1 << 40):
    return lib.pbd_op_prompt_attention(T, B, hq, hkv, D, dt, scale, q, qs, k, v, ks, starts, C.byref(kv) if kv else None, slots, out, lse, ws,
                                       nb, None)


def tree(lib, kv, T=100, hq=4, scale=1.0, q=A + 10 * G, qs=512, k=A + 11 * G, v=A + 12 * G, ks=256, starts=A + 13 * G, par=A + 17 * G,  # noqa: F811
         pos=A + 18 * G, out=A + 14 * G, lse=A + 15 * G, ws=A + 16 * G, nb=1 << 40):
    return lib.pbd_op_tree_attention(C.byref(kv) if kv else None, T, hq, scale, q, qs, k, v, ks, starts, par, pos, out, lse, ws, nb, None)


def commit(lib, kv, path=A + 10 * G, most=8, took=A + 11 * G, ws=A + 12 * G, nb=1 << 40):  # noqa: F811
    return lib.pbd_op_commit_path(C.byref(kv) if kv else None, path, most, took, ws, nb, None)


def test_assign_arguments(lib):  # noqa: F811
    for kw in (dict(B=0), dict(B=1025), dict(mp=0), dict(ps=0), dict(n=0), dict(mp=1 << 16, ps=1 << 15), dict(most=-1), dict(most=(1 << 30) + 1),
               dict(lens=None), dict(new=None), dict(table=None), dict(held=None), dict(free=None), dict(nf=None), dict(starts=None),
               dict(slots=None), dict(lens=A + 2), dict(new=A + G + 1), dict(table=A + 2), dict(held=A + 2), dict(free=A + 2), dict(nf=A + 2),
               dict(starts=A + 2), dict(pos=A + 2), dict(slots=A + 7 * G + 4)):
        assert assign(lib, **kw) == 1 and b"pbd_op_assign_pages" in lib.pbd_op_last_error(), kw
    for kw in (dict(ws=None), dict(ws=A + 9 * G + 8), dict(nb=1023)):
        assert assign(lib, **kw) == 2, kw
    assert lib.pbd_op_assign_pages_workspace_bytes(1024) == 1024
    assert lib.pbd_op_assign_pages_workspace_bytes(0) == 0 and lib.pbd_op_assign_pages_workspace_bytes(1025) == 0


@pytest.mark.parametrize("a,b", [("table", "lens"), ("table", "new"), ("held", "lens"), ("free", "held"), ("nf", "free"), ("starts", "new"),
                                 ("slots", "free"), ("pos", "slots"), ("ws", "lens"), ("ws", "starts")])
def test_assign_ranges(lib, a, b):  # noqa: F811
    at = dict(lens=A, new=A + G, table=A + 2 * G, held=A + 3 * G, free=A + 4 * G, nf=A + 5 * G, starts=A + 6 * G, slots=A + 7 * G, pos=A + 8 * G)
    where = (at[b] + 1023) // 1024 * 1024 if a == "ws" else at[b]
    assert assign(lib, **{a: where}) == 1 and b"lies over" in lib.pbd_op_last_error()


def test_prompt_arguments(lib):  # noqa: F811
    for kw in (dict(T=0), dict(T=(1 << 30) + 1), dict(B=0), dict(B=1025), dict(hkv=0), dict(hkv=257, hq=257), dict(hq=3), dict(hq=1), dict(hq=0),
               dict(hq=8192), dict(D=96), dict(D=0), dict(dt=pbd.PBD_FP32), dict(dt=9), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN),
               dict(scale=INF), dict(q=None), dict(k=None), dict(v=None), dict(starts=None), dict(out=None), dict(q=A + 8), dict(k=A + 8),
               dict(v=A + 4), dict(out=A + 2), dict(starts=A + 2), dict(lse=A + 2), dict(qs=504), dict(qs=516), dict(ks=248), dict(ks=260),
               dict(qs=1 << 38), dict(ks=1 << 40), dict(kv=apart()), dict(slots=A + 20 * G)):
        assert prompt(lib, **kw) == 1 and b"pbd_op_prompt_attention" in lib.pbd_op_last_error(), kw
    for kw in (dict(ws=None), dict(ws=A + 16 * G + 16), dict(nb=1023)):
        assert prompt(lib, **kw) == 2, kw
    for sizes in ((0, 1, 2, 1, 128), (1, 0, 2, 1, 128), (1, 1, 3, 2, 128), (1, 1, 2, 1, 100), ((1 << 30) + 1, 1, 2, 1, 128)):
        assert lib.pbd_op_prompt_attention_workspace_bytes(*sizes) == 0
    assert lib.pbd_op_prompt_attention_workspace_bytes(100, 3, 4, 2, 128) > 0


@pytest.mark.parametrize("bad", BAD + BAD_POINTERS, ids=str)
def test_caches_that_are_refused(lib, bad):  # noqa: F811
    kv = cache(**bad)
    assert prompt(lib, kv=kv, slots=A + 20 * G) == 1 and b"pbd_op_prompt_attention" in lib.pbd_op_last_error()
    assert tree(lib, kv) == 1 and b"pbd_op_tree_attention" in lib.pbd_op_last_error()
    assert commit(lib, kv) == 1 and b"pbd_op_commit_path" in lib.pbd_op_last_error()
    sizes = bad in BAD
    assert (lib.pbd_op_tree_attention_workspace_bytes(C.byref(kv), 64, 4) == 0) == sizes
    assert (lib.pbd_op_commit_path_workspace_bytes(C.byref(kv), 8) == 0) == sizes


@pytest.mark.parametrize("strides", OVER, ids=str)
def test_written_rows_that_lie_over_one_another_are_refused(lib, strides):  # noqa: F811
    kv = apart(**dict(zip(("stride_page", "stride_head", "stride_slot"), strides)))
    for s in (prompt(lib, kv=kv, slots=A + 20 * G), tree(lib, kv), commit(lib, kv)):
        assert s == 1 and b"rows" in lib.pbd_op_last_error()


def test_cached_prompt_arguments(lib):  # noqa: F811
    for kw in (dict(dtype=pbd.PBD_FP16), dict(head_dim=64), dict(n_kv_heads=4)):
        assert prompt(lib, kv=apart(**kw), slots=A + 20 * G) == 1 and b"not k's and v's" in lib.pbd_op_last_error(), kw
    assert prompt(lib, kv=apart(), slots=A + 20 * G + 4) == 1
    assert prompt(lib, kv=apart(d_v=A + G), slots=A + 20 * G) == 1 and b"K and V" in lib.pbd_op_last_error()
    for kw in (dict(out=A + G), dict(lse=A + 2 * G), dict(q=A + G), dict(k=A + G), dict(v=A + 2 * G), dict(ws=A + G), dict(slots=A + G),
               dict(starts=A + 2 * G)):
        assert prompt(lib, kv=apart(), **dict(dict(slots=A + 20 * G), **kw)) == 1 and b"lies over" in lib.pbd_op_last_error(), kw


def test_prompt_ranges(lib):  # noqa: F811
    for kw in (dict(out=A + 10 * G), dict(out=A + 11 * G + 16), dict(lse=A + 12 * G), dict(lse=A + 13 * G), dict(ws=A + 14 * G), dict(out=A + 15 * G)):
        assert prompt(lib, **kw) == 1 and b"lies over" in lib.pbd_op_last_error(), kw


def test_tree_arguments(lib):  # noqa: F811
    kv = apart()
    assert tree(lib, None) == 1
    for kw in (dict(T=0), dict(T=(1 << 30) + 1), dict(hq=3), dict(hq=1), dict(hq=0), dict(hq=8192), dict(scale=0.0), dict(scale=NAN), dict(scale=INF),
               dict(q=None), dict(k=None), dict(v=None), dict(starts=None), dict(out=None), dict(q=A + 8), dict(k=A + 8), dict(v=A + 4), dict(out=A + 2),
               dict(starts=A + 2), dict(par=A + 2), dict(pos=A + 2), dict(lse=A + 2), dict(qs=504), dict(qs=516), dict(ks=248), dict(ks=260),
               dict(qs=1 << 38), dict(ks=1 << 40)):
        assert tree(lib, kv, **kw) == 1 and b"pbd_op_tree_attention" in lib.pbd_op_last_error(), kw
    need = lib.pbd_op_tree_attention_workspace_bytes(C.byref(kv), 100, 4)
    assert need > 0
    for kw in (dict(ws=None), dict(ws=A + 16 * G + 16), dict(nb=need - 1)):
        assert tree(lib, kv, **kw) == 2, kw
    for T, hq in ((0, 4), ((1 << 30) + 1, 4), (10, 3), (10, 0)):
        assert lib.pbd_op_tree_attention_workspace_bytes(C.byref(kv), T, hq) == 0
    for kw in (dict(out=A + 10 * G), dict(out=A + G), dict(out=A + 11 * G), dict(lse=A + 2 * G), dict(lse=A + 13 * G), dict(lse=A + 17 * G),
               dict(ws=A + 3 * G), dict(ws=A + 14 * G), dict(q=A + G), dict(k=A + 2 * G), dict(v=A + G), dict(par=A + 2 * G), dict(pos=A + 6 * G),
               dict(out=A + 18 * G), dict(starts=A + G)):
        at = {n: (x + 1023) // 1024 * 1024 if n == "ws" else x for n, x in kw.items()}
        assert tree(lib, kv, **at) == 1 and b"lies over" in lib.pbd_op_last_error(), kw
    assert tree(lib, apart(d_v=A + G)) == 1 and b"K and V" in lib.pbd_op_last_error()


def test_commit_arguments(lib):  # noqa: F811
    kv = apart()
    assert commit(lib, None) == 1
    for kw in (dict(most=0), dict(most=65), dict(most=-1), dict(path=None), dict(took=None), dict(path=A + 2), dict(took=A + 1)):
        assert commit(lib, kv, **kw) == 1 and b"pbd_op_commit_path" in lib.pbd_op_last_error(), kw
    for kw in (dict(ws=None), dict(ws=A + 12 * G + 16), dict(nb=1023)):
        assert commit(lib, kv, **kw) == 2, kw
    assert lib.pbd_op_commit_path_workspace_bytes(C.byref(kv), 65) == 0 and lib.pbd_op_commit_path_workspace_bytes(C.byref(kv), 0) == 0
    for kw in (dict(path=A + G), dict(took=A + 2 * G), dict(path=A + 5 * G), dict(took=A + 6 * G), dict(ws=A + G)):
        at = {n: (x + 1023) // 1024 * 1024 if n == "ws" else x for n, x in kw.items()}
        assert commit(lib, kv, **at) == 1 and b"lies over" in lib.pbd_op_last_error(), kw
    assert commit(lib, apart(d_v=A + G)) == 1 and b"K and V" in lib.pbd_op_last_error()


def test_the_binding_refuses(lib):  # noqa: F811
    import torch
    table = torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(pbd.PbdError, match="on a GPU"):
        pbd.PagePool(table, 16, 10)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(pbd.PbdError, match="on a GPU"):
        pbd.pbd_op_prompt_attention(x, x, x, torch.zeros(2, dtype=torch.int32))
    assert pbd.assign_pages_workspace_bytes(1 << 40) == 0
    assert pbd.prompt_attention_workspace_bytes(1 << 40, 1, 2, 1, 128) == 0
