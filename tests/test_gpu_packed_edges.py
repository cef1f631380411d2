"""Calls of the operators on packed rows that a program may make and others seldom do: offsets beyond 32 bits, outputs at odd
addresses, caches with gaps, many sequences of one and of two tiles in turn, one workspace for a whole step on another stream."""
import math

import pytest

import _kv_oracle as kvref
import _packed_oracle as ref
from test_gpu_packed import env, i32, same_bits, to_gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def room_for(torch, gib):
    if torch.cuda.mem_get_info()[0] < (gib + 4) << 30:
        pytest.skip("not enough memory")


@pytest.mark.parametrize("D,group", [(128, 2), (256, 3)])
def test_rows_of_prompts_far_apart(env, D, group):  # noqa: F811
    """q, k and v in one buffer whose last row begins beyond 2^32 values."""
    torch, pbd = env
    room_for(torch, 10)
    T, hkv, stride = 140, 1, 1 << 25
    hq = hkv * group
    q, k, v = ref.rows(torch, T, hq, hkv, D, torch.bfloat16, False)
    flat = torch.empty((T - 1) * stride + (hq + 2 * hkv) * D, dtype=torch.bfloat16, device="cuda")
    big = flat.as_strided((T, hq + 2 * hkv, D), (stride, D, 1))
    gq, gk, gv = big[:, :hq], big[:, hq:hq + hkv], big[:, hq + hkv:]
    gq.copy_(q), gk.copy_(k), gv.copy_(v)
    out, lse = pbd.pbd_op_prompt_attention(gq, gk, gv, i32(torch, [0, 3, T]), want_lse=True)
    for a, b in ((0, 3), (3, T)):
        ref.check(torch, ref.attend(torch, q[a:b], k[a:b], v[a:b], ref.causal(torch, b - a)), out[a:b], lse[a:b], "bf16")


def test_the_last_of_very_many_rows(env):  # noqa: F811
    """Packed rows whose outputs lie beyond 2^32 values, of a prompt and of a tree; the rows before belong to nobody."""
    torch, pbd = env
    room_for(torch, 22)
    hkv, group, D, n, page = 1, 64, 256, 30, 16
    hq, dt = hkv * group, torch.bfloat16
    T = (1 << 32) // (hq * D) + n
    q, k, v = ref.rows(torch, n, hq, hkv, D, dt, False)
    gq, gk, gv = (torch.empty(T, x.shape[1], D, dtype=dt, device="cuda") for x in (q, k, v))
    for x, y in ((gq, q), (gk, k), (gv, v)):
        x[T - n:] = y.cuda()
    out, lse = torch.empty(T, hq, D, dtype=dt, device="cuda"), torch.empty(T, hq, device="cuda")
    out[:T - n].fill_(7.0)
    pbd.pbd_op_prompt_attention(gq, gk, gv, i32(torch, [T - n, T]), out=out, lse=lse)
    ref.check(torch, ref.attend(torch, q, k, v, ref.causal(torch, n)), out[T - n:], lse[T - n:], "bf16")
    assert (out[T - n - 1] == 7).all() and (out[0] == 7).all()
    c = ref.tree_case(torch, [45], [n], hkv, D, page, dt, "heads")
    g = to_gpu(torch, c)
    out[T - n:].fill_(7.0)
    pbd.pbd_op_tree_attention(gq, pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"]), gk, gv, i32(torch, [T - n, T]), out=out, lse=lse)
    ref.check(torch, ref.tree_attention(torch, c, 0, q, k, v, None), out[T - n:], lse[T - n:], "bf16")
    assert (out[T - n - 1] == 7).all()


@pytest.mark.parametrize("page,layout", [(16, "heads"), (16, "tokens"), (5, "heads")])
def test_pages_beyond_32_bits(env, page, layout):  # noqa: F811
    """Prompt rows stored into pages behind 2^32 values of a cache, read there by a tree, whose path is then moved."""
    torch, pbd = env
    room_for(torch, 20)
    hkv, group, D, dt = 2, 2, 128, torch.bfloat16
    hq = hkv * group
    n_pages = (1 << 32) // (hkv * page * D) + 40
    shape = (n_pages, hkv, page, D) if layout == "heads" else (n_pages, page, hkv, D)
    k, v = (torch.empty(shape, dtype=dt, device="cuda") for _ in range(2))
    if layout != "heads":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    n, m, per = 150, 20, 40
    table = n_pages - 1 - torch.randperm(40, generator=torch.Generator().manual_seed(2)).to(torch.int32).view(1, per)
    lens = i32(torch, [n])
    kv = pbd.PagedKV(k, v, table.cuda(), lens)
    q, kp, vp = ref.rows(torch, n, hq, hkv, D, dt, False)
    at = torch.arange(n)
    slots = table[0, at // page].long() * page + at % page
    pbd.pbd_op_prompt_attention(q.cuda(), kp.cuda(), vp.cuda(), i32(torch, [0, n]), kv=kv, slots=slots.cuda())
    q, kn, vn = ref.rows(torch, m, hq, hkv, D, dt, False, seed=2)
    parents = ref.trees(torch, [m])
    out, lse = pbd.pbd_op_tree_attention(q.cuda(), kv, kn.cuda(), vn.cuda(), i32(torch, [0, m]), parents.cuda(), want_lse=True)
    sees = torch.cat([torch.ones(m, n, dtype=torch.bool), ref.ancestors(torch, parents.tolist())], 1)
    ref.check(torch, ref.attend(torch, q, torch.cat([kp, kn]), torch.cat([vp, vn]), sees), out, lse, "bf16")
    path = [1, 4, 5, 19]
    pbd.pbd_op_commit_path(kv, i32(torch, [path]), i32(torch, [4]))
    at = torch.arange(n + m)
    pages, places = table[0, at // page].long().cuda(), (at % page).cuda()
    for x, old, new in ((k, kp, kn), (v, vp, vn)):
        want = torch.cat([old, new])
        want[n:n + 4] = new[path]
        assert same_bits(torch, x[pages, :, places], want)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_outputs_at_odd_addresses(env, D):  # noqa: F811
    """out 16-byte aligned, but not 32; lse 4-byte aligned."""
    torch, pbd = env
    lens, nodes, hkv, group, page = [70, 0, 300], [20, 3, 64], 1, 3, 16
    hq, dt, T = hkv * group, torch.bfloat16, 87
    q, k, v = (x.cuda() for x in ref.rows(torch, T, hq, hkv, D, dt, False))
    starts = ref.starts_of(torch, nodes).cuda()

    def odd():
        out = torch.zeros(8 + T * hq * D, dtype=dt, device="cuda")[8:].view(T, hq, D)
        assert out.data_ptr() % 32 == 16
        return out, torch.zeros(1 + T * hq, device="cuda")[1:].view(T, hq)
    out, lse = odd()
    want = pbd.pbd_op_prompt_attention(q, k, v, starts, want_lse=True)
    pbd.pbd_op_prompt_attention(q, k, v, starts, out=out, lse=lse)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    g = to_gpu(torch, ref.tree_case(torch, lens, nodes, hkv, D, page, dt, "heads"))
    kv = pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"])
    out, lse = odd()
    want = pbd.pbd_op_tree_attention(q, kv, k, v, starts, want_lse=True)
    pbd.pbd_op_tree_attention(q, kv, k, v, starts, out=out, lse=lse)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


# gaps behind a row of a head, a head's rows, a page's heads; heads
@pytest.mark.parametrize("page", [8, 16, 96, 12])
@pytest.mark.parametrize("gaps", [(8, 0, 0, 2), (0, 1, 0, 2), (0, 0, 1, 3), (16, 2, 1, 1), (0, 0, 0, 1)])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_caches_with_gaps(env, page, gaps, layout):  # noqa: F811
    torch, pbd = env
    lens, nodes, group, D, dt = [300, 17, 0, 128], [9, 30, 64, 1], 3, 64, torch.float16
    row, inner, outer, hkv = gaps
    c = ref.tree_case(torch, lens, nodes, hkv, D, page, dt, layout)
    n_pages = c["k"].shape[0]
    a, b = (hkv, page) if layout == "heads" else (page, hkv)

    def spread(x):
        y = torch.full((n_pages, a + outer, b + inner, D + row), math.nan, dtype=dt, device="cuda")[:, :a, :b, :D]
        y = y if layout == "heads" else y.transpose(1, 2)
        return y.copy_(x)
    g = dict(to_gpu(torch, c), k=spread(c["k"]), v=spread(c["v"]))
    hq, T = hkv * group, sum(nodes)
    q, kn, vn = ref.rows(torch, T, hq, hkv, D, dt, False)
    starts, parents = ref.starts_of(torch, nodes), ref.trees(torch, nodes)
    kv = pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"])
    out, lse = pbd.pbd_op_tree_attention(q.cuda(), kv, kn.cuda(), vn.cuda(), starts.cuda(), parents.cuda(), want_lse=True)
    for i, m in enumerate(nodes):
        at = slice(int(starts[i]), int(starts[i + 1]))
        ref.check(torch, ref.tree_attention(torch, c, i, q[at], kn[at], vn[at], parents[at]), out[at], lse[at], "fp16")
        for j in range(m):
            p, o = int(c["table"][i, (lens[i] + j) // page]), (lens[i] + j) % page
            c["k"][p, :, o], c["v"][p, :, o] = kn[at][j], vn[at][j]
    assert same_bits(torch, g["k"], c["k"].contiguous()) and same_bits(torch, g["v"], c["v"].contiguous())
    pbd.pbd_op_commit_path(kv, i32(torch, [[2, 5], [7, 29], [1, 3], [0, 0]]), i32(torch, [2, 2, 1, 1]))
    for i, path in enumerate([[2, 5], [7, 29], [1], []]):
        for j, x in enumerate(path):
            s, d = lens[i] + x, lens[i] + j
            for n in ("k", "v"):
                c[n][int(c["table"][i, d // page]), :, d % page] = c[n][int(c["table"][i, s // page]), :, s % page].clone()
    assert same_bits(torch, g["k"], c["k"].contiguous()) and same_bits(torch, g["v"], c["v"].contiguous())


@pytest.mark.parametrize("D,page", [(64, 32), (128, 16), (128, 8), (256, 64), (64, 6)])
def test_pages_outside_the_cache_among_whole_blocks(env, D, page):  # noqa: F811
    """Pages that the table names wrongly far in front of the nodes: their slots take no part, the rest does."""
    torch, pbd = env
    lens, nodes, hkv, group, dt = [1000, 700], [5, 64], 2, 2, torch.bfloat16
    c = ref.tree_case(torch, lens, nodes, hkv, D, page, dt, "heads")
    T = sum(nodes)
    q, kn, vn = ref.rows(torch, T, hkv * group, hkv, D, dt, False)
    starts, parents = ref.starts_of(torch, nodes), ref.trees(torch, nodes)
    g = to_gpu(torch, c)
    lost = [[0, 3, 500 // page], [128 // page, 640 // page]]
    for b, pages in enumerate(lost):
        for i, p in enumerate(pages):
            g["table"][b, p] = (-1, c["k"].shape[0], 0x7fffffff)[i]
    kv = pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"])
    out, lse = torch.zeros(T, hkv * group, D, dtype=dt, device="cuda"), torch.zeros(T, hkv * group, device="cuda")
    with pytest.raises(pbd.PbdError, match="PBD_ERR_DEVICE"):
        pbd.pbd_op_tree_attention(q.cuda(), kv, kn.cuda(), vn.cuda(), starts.cuda(), parents.cuda(), out=out, lse=lse)
    for b, (n, m) in enumerate(zip(lens, nodes)):
        at = slice(int(starts[b]), int(starts[b + 1]))
        sees = torch.cat([torch.ones(m, n, dtype=torch.bool), ref.ancestors(torch, parents[at].tolist())], 1)
        for p in lost[b]:
            sees[:, p * page:(p + 1) * page] = False
        k, v = (torch.cat([kvref.rows_of(c, c[x], b, n).transpose(0, 1), new[at].double()]) for x, new in (("k", kn), ("v", vn)))
        ref.check(torch, ref.attend(torch, q[at], k, v, sees), out[at], lse[at], "bf16")


@pytest.mark.parametrize("D,page", [(64, 32), (128, 16), (64, 7)])
def test_odd_values_in_units_of_one_and_two_tiles_in_turn(env, D, page):  # noqa: F811
    """Short sequences, many a CTA, some of more than 128 rows, whose nodes hold values of V that are infinite or NaN here and
    there: each sequence keeps its own."""
    torch, pbd = env
    group, hkv, dt, B = 7, 2, torch.float16, 600
    gen = torch.Generator().manual_seed(D + page)
    nodes = torch.where(torch.rand(B, generator=gen) < 0.2, torch.randint(20, 37, (B,), generator=gen), torch.randint(0, 8, (B,), generator=gen)).tolist()
    lens = torch.randint(0, 90, (B,), generator=gen).tolist()
    c = ref.tree_case(torch, lens, nodes, hkv, D, page, dt, "tokens")
    T, hq = sum(nodes), hkv * group
    q, kn, vn = ref.rows(torch, T, hq, hkv, D, dt, False)
    where = torch.randperm(T, generator=gen)[:T // 40]
    for i, t in enumerate(where.tolist()):
        vn[t, i % hkv, (7 * i) % D] = (math.inf, math.nan, -math.inf)[i % 3]
    starts, parents = ref.starts_of(torch, nodes), ref.trees(torch, nodes)
    g = to_gpu(torch, c)
    out, lse = pbd.pbd_op_tree_attention(q.cuda(), pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"]), kn.cuda(), vn.cuda(), starts.cuda(),
                                         parents.cuda(), want_lse=True)
    out, lse = out.cpu(), lse.cpu()
    for b, m in enumerate(nodes):
        if m:
            at = slice(int(starts[b]), int(starts[b + 1]))
            ref.check(torch, ref.tree_attention(torch, c, b, q[at], kn[at], vn[at], parents[at]), out[at], lse[at], "fp16")


def test_one_workspace_on_another_stream(env):  # noqa: F811
    """Pages, a prompt that fills them, a tree and its path in turn on a stream of their own, nothing waited for in between."""
    torch, pbd = env
    hkv, group, D, page, dt, T = 2, 4, 128, 16, torch.bfloat16, 200
    hq = hkv * group
    stream = torch.cuda.Stream()
    q, k, v = ref.rows(torch, T, hq, hkv, D, dt, False)
    tq, tk, tv = ref.rows(torch, 40, hq, hkv, D, dt, False, seed=2)
    parents, path = ref.trees(torch, [30, 10]), [[0, 3, 9], [1, 2, 8]]
    data = [x.cuda() for x in (q, k, v, tq, tk, tv, parents)]
    cache = [torch.zeros(40, hkv, page, D, dtype=dt, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        pool = pbd.PagePool(torch.zeros(2, 20, dtype=torch.int32, device="cuda"), page, 40)
        lens = i32(torch, [0, 0])
        kv = pbd.PagedKV(*cache, pool.page_table, lens)
        ws = pbd.op_workspace(max(pbd.tree_attention_workspace_bytes(kv, T, hq), pbd.prompt_attention_workspace_bytes(T, 2, hq, hkv, D), 1024))
        counts, nodes, took = i32(torch, [150, 50]), i32(torch, [30, 10]), i32(torch, [3, 3])
        torch.cuda._sleep(2_000_000)
        got = pbd.pbd_op_assign_pages(pool, lens, counts, T, workspace=ws, sync=False)
        out1 = pbd.pbd_op_prompt_attention(*data[:3], got.starts, kv=kv, slots=got.slots, workspace=ws, sync=False)[0]
        lens.add_(counts)
        got = pbd.pbd_op_assign_pages(pool, lens, nodes, 40, workspace=ws, sync=False)
        out2 = pbd.pbd_op_tree_attention(data[3], kv, *data[4:6], got.starts, data[6], workspace=ws, sync=False)[0]
        pbd.pbd_op_commit_path(kv, i32(torch, path), took, workspace=ws, sync=False)
        lens.add_(took)
    pbd_status = pbd.pbd_op_status
    with torch.cuda.stream(stream):
        pbd_status(ws)
    table = pool.page_table.tolist()
    for b, (a, e, s, t) in enumerate(((0, 150, 0, 30), (150, 200, 30, 40))):
        ref.check(torch, ref.attend(torch, q[a:e], k[a:e], v[a:e], ref.causal(torch, e - a)), out1[a:e], None, "bf16")
        n, m = e - a, t - s
        sees = torch.cat([torch.ones(m, n, dtype=torch.bool), ref.ancestors(torch, parents[s:t].tolist())], 1)
        ref.check(torch, ref.attend(torch, tq[s:t], torch.cat([k[a:e], tk[s:t]]), torch.cat([v[a:e], tv[s:t]]), sees), out2[s:t], None, "bf16")
        for x, old, new in ((cache[0], k, tk), (cache[1], v, tv)):
            for i in range(n + 3):
                want = old[a + i] if i < n else new[s + path[b][i - n]]
                assert torch.equal(x[table[b][i // page], :, i % page].cpu(), want)


def test_a_pool_keeps_its_tensors(env):  # noqa: F811
    torch, pbd = env
    pool = pbd.PagePool(torch.zeros(2, 5, dtype=torch.int32, device="cuda"), 16, 8)
    for name in ("page_table", "held", "free", "n_free"):
        with pytest.raises(pbd.PbdError, match="PBD_ERR_INVALID_ARG"):
            setattr(pool, name, getattr(pool, name).clone())
        setattr(pool, name, getattr(pool, name))
    pool.held += 0  # (in place)
    assert pool.n_free.tolist() == [8]


def test_all_of_them_at_once_on_streams_of_their_own(env):  # noqa: F811
    """A prompt, trees of two caches and the paths of a third, none waiting for another: what each gives alone."""
    torch, pbd = env
    hkv, group, page, dt = 2, 4, 16, torch.bfloat16
    hq = hkv * group
    prompts = [x.cuda() for x in ref.rows(torch, 900, hq, hkv, 128, dt, False)]
    starts = i32(torch, [0, 700, 900])
    lens, nodes = [400, 90, 1000, 0], [64, 20, 33, 5]
    T = sum(nodes)
    trees, fresh = [], []
    for D in (128, 64):
        c = ref.tree_case(torch, lens, nodes, hkv, D, page, dt, "heads")
        trees.append((c, [x.cuda() for x in ref.rows(torch, T, hq, hkv, D, dt, False, seed=D)]))
        fresh.append([to_gpu(torch, c) for _ in range(2)])
    node_starts = ref.starts_of(torch, nodes).cuda()
    third = kvref.make_cache(torch, [n + 64 for n in lens], hkv, 128, page, dt, extra=0)
    third["lens"] = torch.tensor(lens, dtype=torch.int32)
    paths, took = i32(torch, [list(range(1, 64, 2))] * 4), i32(torch, [32, 7, 0, 31])

    def calls(turn, where):
        out = []
        copies = [f[turn] for f in fresh]
        moved = to_gpu(torch, third)
        torch.cuda.synchronize()

        def prompt():
            out.append(pbd.pbd_op_prompt_attention(*prompts, starts, sync=False)[0])

        def tree(i):
            g, (q, kn, vn) = copies[i], trees[i][1]
            out.append(pbd.pbd_op_tree_attention(q, pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"]), kn, vn, node_starts, sync=False)[0])

        def commit():
            pbd.pbd_op_commit_path(pbd.PagedKV(moved["k"], moved["v"], moved["table"], moved["lens"]), paths, took, sync=False)
        for f, s in zip((prompt, lambda: tree(0), lambda: tree(1), commit), where):
            with torch.cuda.stream(s):
                f()
        torch.cuda.synchronize()
        return out + [x[n] for x in copies + [moved] for n in ("k", "v")]
    alone = calls(0, [torch.cuda.current_stream()] * 4)
    for x, y in zip(alone, calls(1, [torch.cuda.Stream() for _ in range(4)])):
        assert torch.equal(x.contiguous().view(torch.int16), y.contiguous().view(torch.int16))


@pytest.mark.parametrize("D,group", [(64, 11), (128, 13), (128, 15), (256, 9), (64, 26), (128, 14), (64, 6)])
def test_prompts_of_groups_that_leave_rows_over(env, D, group):  # noqa: F811
    """Heads a KV head that do not divide a tile's 128 rows, two KV heads, prompts around a tile's tokens and a block of keys; the
    rows behind the prompts are NaN."""
    torch, pbd = env
    tile = 128 // group
    lens, hkv, dt = [1, tile, 0, tile + 1, 2 * tile - 1, 129, 2 * tile + 1, 300], 2, torch.bfloat16
    hq, T = hkv * group, sum(lens) + 3
    q, k, v = ref.rows(torch, T, hq, hkv, D, dt, True, lens)
    starts = ref.starts_of(torch, lens)
    out, lse = torch.full((T, hq, D), 7.0, dtype=dt, device="cuda"), torch.full((T, hq), 7.0, device="cuda")
    pbd.pbd_op_prompt_attention(*ref.fused_to_gpu(torch, q, k, v), starts.cuda(), out=out, lse=lse)
    for i, n in enumerate(lens):
        if n:
            at = slice(int(starts[i]), int(starts[i + 1]))
            ref.check(torch, ref.attend(torch, q[at], k[at], v[at], ref.causal(torch, n)), out[at], lse[at], "bf16")
    assert (out[T - 3:] == 7).all() and (lse[T - 3:] == 7).all()


def test_the_most_heads_and_sequences(env):  # noqa: F811
    """4096 query heads on one KV head; 1024 sequences, many of them empty."""
    torch, pbd = env
    dt = torch.bfloat16
    for lens, nodes, hkv, group, D, page in (([40], [3], 1, 4096, 64, 16), ([i % 37 for i in range(1024)], [i % 3 for i in range(1024)], 1, 2, 128, 8)):
        hq, T = hkv * group, sum(nodes)
        q, kn, vn = ref.rows(torch, T, hq, hkv, D, dt, False)
        starts = ref.starts_of(torch, nodes)
        gpu = [x.cuda() for x in (q, kn, vn)]
        out, lse = (x.cpu() for x in pbd.pbd_op_prompt_attention(*gpu, starts.cuda(), want_lse=True))
        c = ref.tree_case(torch, lens, nodes, hkv, D, page, dt, "heads")
        g = to_gpu(torch, c)
        kv = pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"])
        out2, lse2 = (x.cpu() for x in pbd.pbd_op_tree_attention(gpu[0], kv, *gpu[1:], starts.cuda(), want_lse=True))
        for b, m in enumerate(nodes):
            if m:
                at = slice(int(starts[b]), int(starts[b + 1]))
                ref.check(torch, ref.attend(torch, q[at], kn[at], vn[at], ref.causal(torch, m)), out[at], lse[at], "bf16")
                ref.check(torch, ref.tree_attention(torch, c, b, q[at], kn[at], vn[at], None), out2[at], lse2[at], "bf16")


def test_a_first_call_within_a_capture(env):  # noqa: F811
    """In a process of its own, whose first calls of all four are captured as one step."""
    import os
    import subprocess
    import sys
    code = """
import sys
sys.path[:0] = ["tests", "."]
import torch, _packed_oracle as ref
from paper_2607_12422_gb300 import pbd
hkv, group, D, page, n, m = 2, 2, 128, 16, 150, 20
dt = torch.bfloat16
q, k, v = (x.cuda() for x in ref.rows(torch, n, hkv * group, hkv, D, dt, False))
tq, tk, tv = (x.cuda() for x in ref.rows(torch, m, hkv * group, hkv, D, dt, False, seed=2))
cache = [torch.zeros(20, hkv, page, D, dtype=dt, device="cuda") for _ in range(2)]
pool = pbd.PagePool(torch.zeros(1, 20, dtype=torch.int32, device="cuda"), page, 20)
lens, none = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
new, nodes, took = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (n, m, 2))
path = torch.tensor([[1, 7]], dtype=torch.int32, device="cuda")
kv = pbd.PagedKV(*cache, pool.page_table, lens)
ws = pbd.op_workspace(max(pbd.tree_attention_workspace_bytes(kv, m, hkv * group), 4096))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = pbd.pbd_op_assign_pages(pool, lens, new, n, workspace=ws, sync=False)
    out1 = pbd.pbd_op_prompt_attention(q, k, v, got.starts, kv=kv, slots=got.slots, workspace=ws, sync=False)[0]
    lens.add_(new)
    got = pbd.pbd_op_assign_pages(pool, lens, nodes, m, workspace=ws, sync=False)
    out2 = pbd.pbd_op_tree_attention(tq, kv, tk, tv, got.starts, workspace=ws, sync=False)[0]
    pbd.pbd_op_commit_path(kv, path, took, workspace=ws, sync=False)
graph.replay()
pbd.pbd_op_status(ws)
ref.check(torch, ref.attend(torch, q.cpu(), k.cpu(), v.cpu(), ref.causal(torch, n)), out1, None, "bf16")
sees = torch.cat([torch.ones(m, n, dtype=torch.bool), ref.causal(torch, m)], 1)
ref.check(torch, ref.attend(torch, tq.cpu(), torch.cat([k, tk]).cpu(), torch.cat([v, tv]).cpu(), sees), out2, None, "bf16")
table = pool.page_table[0].tolist()
for i, x in ((n, 1), (n + 1, 7)):
    assert torch.equal(cache[0][table[i // page], :, i % page], tk[x]) and torch.equal(cache[1][table[i // page], :, i % page], tv[x])
print("done")
"""
    got = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300,
                         cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert got.returncode == 0 and got.stdout.strip().endswith("done"), got.stderr[-2000:]
