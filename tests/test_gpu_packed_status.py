"""The status codes of the operators on packed rows, pages and paths, as the header gives them, and which one is said where there
are several faults."""
import ctypes as C

import pytest

from test_gpu_packed import env, i32  # noqa: F401

pytestmark = pytest.mark.gpu

BAD_LENGTH, BAD_PAGE, NO_PAGES, BAD_TREE = 5, 7, 8, 9


def code_of(torch, pbd, ws):
    code = C.c_int32(-1)
    s = pbd.load().pbd_op_status(ws.ptr, torch.cuda.current_stream().cuda_stream, C.byref(code))
    assert (s == 0) == (code.value == 0) and s in (0, 6)
    return code.value


# a pool of 6 pages of 4 slots; two sequences, of which the first needs no more and the second one
POOL = dict(table=[[3, 5, 0], [1, 0, 0]], held=[2, 1], free=[0, 2, 4, 9, 9, 9], n_free=3, lens=[7, 3], new=[1, 4], most=8)


@pytest.mark.parametrize("pad", [0, 9000, 40000])  # one CTA, a cluster, rows by a second kernel
@pytest.mark.parametrize("code,kw", [
    (0, dict()),
    (BAD_LENGTH, dict(lens=[-1, 3])), (BAD_LENGTH, dict(new=[1, -1])), (BAD_LENGTH, dict(lens=[12, 3])), (BAD_LENGTH, dict(new=[1, 10])),
    (BAD_LENGTH, dict(new=[1 << 30, 4])), (BAD_LENGTH, dict(lens=[(1 << 31) - 1, 3], new=[(1 << 31) - 1, 4])),
    (BAD_PAGE, dict(held=[2, -1])), (BAD_PAGE, dict(held=[2, 4])), (BAD_PAGE, dict(n_free=-1)), (BAD_PAGE, dict(n_free=7)),
    (BAD_PAGE, dict(n_free=4)), (BAD_PAGE, dict(held=[3, 1])), (BAD_PAGE, dict(free=[0, 2, 6, 9, 9, 9])), (BAD_PAGE, dict(free=[0, 2, -1, 9, 9, 9])),
    (BAD_PAGE, dict(table=[[3, 6, 0], [1, 0, 0]], lens=[0, 3], new=[0, 4])),
    (BAD_PAGE, dict(table=[[3, 6, 0], [1, 0, 0]], lens=[6, 3], new=[1, 1])),  # one held before: rows get no slot
    (NO_PAGES, dict(lens=[12, 12], new=[0, 0], n_free=2)), (NO_PAGES, dict(lens=[7, 3], new=[5, 9], n_free=2, most=14)),
    # several: a length before a page, both before a shortage
    (BAD_LENGTH, dict(lens=[-1, 3], held=[2, 4])), (BAD_LENGTH, dict(lens=[12, 12], new=[0, 1], n_free=2)),
    (BAD_PAGE, dict(lens=[12, 12], new=[0, 0], n_free=2, held=[2, -1])),
], ids=str)
def test_pages(env, code, kw, pad):  # noqa: F811
    torch, pbd = env
    c = dict(POOL, **kw)
    pool = pbd.PagePool(i32(torch, c["table"]), 4, 6, held=i32(torch, c["held"]), free=i32(torch, c["free"]), n_free=i32(torch, [c["n_free"]]))
    ws = pbd.op_workspace(1024)
    pbd.pbd_op_assign_pages(pool, i32(torch, c["lens"]), i32(torch, c["new"]), c["most"] + pad, workspace=ws, sync=False)
    assert code_of(torch, pbd, ws) == code


def test_more_new_tokens_than_rows(env):  # noqa: F811
    torch, pbd = env
    pool = pbd.PagePool(i32(torch, POOL["table"]), 4, 6, held=i32(torch, POOL["held"]), free=i32(torch, POOL["free"]), n_free=i32(torch, [3]))
    ws = pbd.op_workspace(1024)
    pbd.pbd_op_assign_pages(pool, i32(torch, POOL["lens"]), i32(torch, POOL["new"]), 4, workspace=ws, sync=False)
    assert code_of(torch, pbd, ws) == BAD_LENGTH


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("code,starts,slot", [
    (0, [0, 20, 40, 60], 0), (0, [0, 20, 40, 60], -5),
    (BAD_LENGTH, [0, 20, 10, 60], 0), (BAD_LENGTH, [0, 20, 40, 61], 0), (BAD_LENGTH, [-1, 20, 40, 60], 0), (BAD_LENGTH, [5, 5, 5, 70], 0),
    (BAD_PAGE, [0, 20, 40, 60], 80), (BAD_PAGE, [0, 20, 40, 60], 1 << 40),
    (BAD_LENGTH, [0, 20, 40, 61], 80),  # both: the bounds
], ids=str)
def test_prompts(env, code, starts, slot, D):  # noqa: F811
    torch, pbd = env
    q, k, v = (torch.ones(60, n, D, dtype=torch.bfloat16, device="cuda") for n in (4, 2, 2))
    ck, cv = (torch.zeros(5, 2, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slots = torch.arange(60, device="cuda")
    slots[7] = 79 if slot == 0 else slot
    ws = pbd.op_workspace(1024)
    pbd.pbd_op_prompt_attention(q, k, v, i32(torch, starts), kv=pbd.PagedKV(ck, cv, i32(torch, [[0]] * 3), i32(torch, [0] * 3)), slots=slots,
                                workspace=ws, sync=False)
    assert code_of(torch, pbd, ws) == code


LENGTH, PAGE, NODE_PAGE, PARENT = dict(lens=[50, 1 << 20, 20]), dict(page=2), dict(page=6), dict(parent=4)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("code,kw", [
    (0, dict()), (BAD_LENGTH, LENGTH), (BAD_LENGTH, dict(lens=[50, -1, 20])), (BAD_LENGTH, dict(starts=[0, 10, 5, 35])),
    (BAD_LENGTH, dict(starts=[0, 10, 30, 36])), (BAD_LENGTH, dict(starts=[0, 0, 0, 65], T=65)), (BAD_PAGE, PAGE), (BAD_PAGE, NODE_PAGE),
    (BAD_TREE, PARENT), (BAD_TREE, dict(parent=-2)), (BAD_TREE, dict(parent=1 << 30)),
    # several, of one sequence or of two: a length before a page before a parent
    (BAD_LENGTH, dict(LENGTH, parent=4)), (BAD_LENGTH, dict(PAGE, lens=[-1, 90, 20])), (BAD_PAGE, dict(PAGE, **PARENT)),
    (BAD_LENGTH, dict(NODE_PAGE, lens=[-1, 90, 20], parent=4)),
], ids=str)
def test_trees(env, code, kw, D):  # noqa: F811
    torch, pbd = env
    lens, starts, page, T = kw.get("lens", [50, 90, 20]), kw.get("starts", [0, 10, 30, 35]), 16, kw.get("T", 35)
    per, hkv = 7, 1
    table = torch.arange(3 * per, dtype=torch.int32).view(3, per)
    if "page" in kw:
        table[1, kw["page"]] = 3 * per
    parents = torch.full((T,), -1, dtype=torch.int32)
    parents[10 + 4] = kw.get("parent", -1)
    q, kn, vn = (torch.ones(T, n, D, dtype=torch.bfloat16, device="cuda") for n in (2, hkv, hkv))
    ck, cv = (torch.ones(3 * per, hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kv = pbd.PagedKV(ck, cv, table.cuda(), i32(torch, lens))
    ws = pbd.op_workspace(pbd.tree_attention_workspace_bytes(kv, T, 2))
    pbd.pbd_op_tree_attention(q, kv, kn, vn, i32(torch, starts), parents.cuda(), workspace=ws, sync=False)
    assert code_of(torch, pbd, ws) == code


@pytest.mark.parametrize("code,path,n,lens,page", [
    (0, [[2, 5, 9], [1, 2, 3]], [3, 3], [20, 30], None),
    (BAD_TREE, [[2, 5, 9], [3, 3, 4]], [3, 3], [20, 30], None), (BAD_TREE, [[2, 5, 9], [3, 2, 4]], [3, 2], [20, 30], None),
    (BAD_TREE, [[2, 5, 9], [-1, 2, 4]], [3, 2], [20, 30], None), (BAD_TREE, [[2, 5, 9], [1, 2, 64]], [3, 3], [20, 30], None),
    (BAD_TREE, [[2, 5, 9], [1, 2, 27]], [3, 3], [20, 30], None),
    (BAD_LENGTH, [[2, 5, 9], [1, 2, 3]], [3, 4], [20, 30], None), (BAD_LENGTH, [[2, 5, 9], [1, 2, 3]], [3, -1], [20, 30], None),
    (BAD_LENGTH, [[2, 5, 9], [1, 2, 3]], [3, 3], [20, -1], None), (BAD_LENGTH, [[2, 5, 9], [1, 2, 3]], [3, 3], [20, 57], None),
    (BAD_PAGE, [[2, 5, 9], [1, 5, 12]], [3, 3], [20, 30], 4),
    # of one sequence: what its path says before its pages
    (BAD_TREE, [[2, 5, 9], [5, 5, 12]], [3, 3], [20, 30], 4),
], ids=str)
def test_paths(env, code, path, n, lens, page):  # noqa: F811
    torch, pbd = env
    table = torch.arange(14, dtype=torch.int32).view(2, 7)
    if page is not None:
        table[1, page] = 1 << 30
    ck, cv = (torch.ones(14, 2, 8, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kv = pbd.PagedKV(ck, cv, table.cuda(), i32(torch, lens))
    ws = pbd.op_workspace(1024)
    pbd.pbd_op_commit_path(kv, i32(torch, path), i32(torch, n), workspace=ws, sync=False)
    assert code_of(torch, pbd, ws) == code
