"""Attention over packed prompts and drafted trees, pages from lengths and accepted paths, against the same in 64 bits and in
plain Python."""
import math

import pytest

import _kv_oracle as kvref
import _packed_oracle as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_12422_gb300 import pbd
    pbd.load()
    return torch, pbd


def to_gpu(torch, c):
    def move(x):
        y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
        return y.copy_(x)
    return {n: move(c[n]) for n in ("k", "v", "table", "lens", "weights", "positions")}


def same_bits(torch, x, y):
    return torch.equal(x.cpu().contiguous().view(torch.int16), y.contiguous().view(torch.int16))


def i32(torch, x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ prompts

PROMPTS = [
    # lens, hkv, group, D
    ([1], 1, 1, 64),
    ([2, 0, 1], 1, 2, 128),
    ([31, 32, 33, 0, 127, 128, 129], 2, 2, 128),
    ([63, 64, 65, 255, 256, 257, 5], 2, 4, 128),
    ([300, 17], 1, 1, 128),
    ([513, 3], 2, 3, 64),
    ([700], 1, 7, 64),
    ([140, 141], 1, 16, 128),
    ([90, 0, 0, 411], 1, 12, 64),
    ([70], 1, 40, 128),
    ([385, 1, 64], 1, 2, 256),
    ([129, 40], 2, 5, 256),
    ([1025], 1, 8, 128),
    ([9] * 70, 1, 2, 64),
    ([i % 40 for i in range(200)], 2, 1, 128),
]


@pytest.mark.parametrize("store", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", PROMPTS, ids=lambda s: "%dx%s-%s" % (len(s[0]), max(s[0]), "-".join(map(str, s[1:]))))
def test_prompts_match_64_bits(env, shape, dtype, store):
    """Rows of no sequence hold NaN and stay as they are; with `store` q, k and v are parts of one buffer."""
    torch, pbd = env
    lens, hkv, group, D = shape
    dt, hq, pad, page = getattr(torch, ref.DT[dtype]), hkv * group, 3, 24
    T = sum(lens) + pad
    q, k, v = ref.rows(torch, T, hq, hkv, D, dt, store, lens)
    gq, gk, gv = ref.fused_to_gpu(torch, q, k, v)
    starts = ref.starts_of(torch, lens)
    out, lse = torch.full((T, hq, D), 7.0, dtype=dt, device="cuda"), torch.full((T, hq), 7.0, device="cuda")
    kw = {}
    if store:
        c = kvref.make_cache(torch, lens, hkv, D, page, dt, "tokens" if group % 2 else "heads", extra=0)
        g = to_gpu(torch, c)
        slots = torch.full((T,), -1, dtype=torch.int64)
        for b, n in enumerate(lens):
            for i in range(n):
                slots[int(starts[b]) + i] = int(c["table"][b, i // page]) * page + i % page
        if sum(lens) > 2:
            slots[sum(lens) // 2] = -1  # one row that is not to be stored
        kw = dict(kv=pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"]), slots=slots.cuda())
    ws = pbd.op_workspace(pbd.prompt_attention_workspace_bytes(T, len(lens), hq, hkv, D))
    pbd.pbd_op_prompt_attention(gq, gk, gv, starts.cuda(), out=out, lse=lse, workspace=ws, **kw)
    for b, n in enumerate(lens):
        if n:
            at = slice(int(starts[b]), int(starts[b + 1]))
            ref.check(torch, ref.attend(torch, q[at], k[at], v[at], ref.causal(torch, n)), out[at], lse[at], dtype)
    assert (out[sum(lens):] == 7).all() and (lse[sum(lens):] == 7).all()
    out2, lse2 = pbd.pbd_op_prompt_attention(gq, gk, gv, starts.cuda(), want_lse=True, workspace=ws)
    n = sum(lens)
    assert torch.equal(out2[:n], out[:n]) and torch.equal(lse2[:n], lse[:n])  # the same bits on every call
    if store:
        for x, y, new in ((g["k"], c["k"], k), (g["v"], c["v"], v)):
            for t, s in enumerate(slots.tolist()):
                if s >= 0:
                    y[s // page, :, s % page] = new[t]
            assert same_bits(torch, x, y)


@pytest.mark.parametrize("D,group", [(128, 2), (64, 7), (256, 1)])
def test_values_that_a_row_does_not_see_do_not_touch_it(env, D, group):
    """NaN and infinities in V (and K) of later rows and of other sequences; they reach the rows that see them, in their
    dimension alone."""
    torch, pbd = env
    lens, hkv = [200, 333, 64], 2
    T = sum(lens)
    q, k, v = ref.rows(torch, T, hkv * group, hkv, D, torch.bfloat16, False)
    for t, h, d, x in ((150, 0, 3, math.inf), (151, 0, 4, math.nan), (199, 1, D - 1, -math.inf), (200 + 130, 1, 0, math.nan),
                       (200 + 332, 0, D // 2, math.inf), (533 + 63, 1, 9, math.inf)):
        v[t, h, d] = x
    starts = ref.starts_of(torch, lens)
    out, lse = pbd.pbd_op_prompt_attention(q.cuda(), k.cuda(), v.cuda(), starts.cuda(), want_lse=True)
    for b, n in enumerate(lens):
        at = slice(int(starts[b]), int(starts[b + 1]))
        want = ref.attend(torch, q[at], k[at], v[at], ref.causal(torch, n))
        ref.check(torch, want, out[at], lse[at], "bf16")
    # a key that is NaN: the rows from it on are NaN, the others as before
    k[170] = math.nan
    out2, lse2 = pbd.pbd_op_prompt_attention(q.cuda(), k.cuda(), v.cuda(), starts.cuda(), want_lse=True)
    assert torch.equal(out2[:150], out[:150]) and torch.equal(lse2[:170], lse[:170])
    assert torch.isnan(out2[170:200]).all() and torch.isnan(lse2[170:200]).all()
    assert torch.equal(out2[533:, :, :9], out[533:, :, :9])


def test_prompts_of_large_scores_and_equal_keys(env):
    torch, pbd = env
    for dtype in ("bf16", "fp16"):
        q, k, v = ref.rows(torch, 400, 4, 2, 128, getattr(torch, ref.DT[dtype]), False)
        k *= 20
        q[200:] = 0  # the mean of the values so far
        starts = ref.starts_of(torch, [200, 200])
        out, lse = pbd.pbd_op_prompt_attention(q.cuda(), k.cuda(), v.cuda(), starts.cuda(), scale=0.3, want_lse=True)
        for at in (slice(0, 200), slice(200, 400)):
            ref.check(torch, ref.attend(torch, q[at], k[at], v[at], ref.causal(torch, 200), 0.3), out[at], lse[at], dtype)
    # scores that rise from key to key: the running maximum follows all the way
    q, k, v = ref.rows(torch, 600, 2, 1, 64, torch.bfloat16, False)
    q[:], k[:] = 1.0, (torch.arange(600)[:, None, None] / 8.0).to(torch.bfloat16)
    starts = ref.starts_of(torch, [600])
    out, lse = pbd.pbd_op_prompt_attention(q.cuda(), k.cuda(), v.cuda(), starts.cuda(), scale=0.5, want_lse=True)
    ref.check(torch, ref.attend(torch, q, k, v, ref.causal(torch, 600), 0.5), out, lse, "bf16")
    k = -k
    out, lse = pbd.pbd_op_prompt_attention(q.cuda(), k.cuda(), v.cuda(), starts.cuda(), scale=0.5, want_lse=True)
    ref.check(torch, ref.attend(torch, q, k, v, ref.causal(torch, 600), 0.5), out, lse, "bf16")


def test_masked_scores_of_minus_infinity(env):
    """Rows all of whose scores are -inf give zeros and -inf, as rows that see nothing."""
    torch, pbd = env
    q, k, v = ref.rows(torch, 140, 2, 1, 64, torch.bfloat16, False)
    q[:], k[:] = 1.0, 0.0
    k[:130, :, 0] = -math.inf
    out, lse = pbd.pbd_op_prompt_attention(q.cuda(), k.cuda(), v.cuda(), ref.starts_of(torch, [140]).cuda(), want_lse=True)
    assert (out[:130] == 0).all() and (lse[:130] == -math.inf).all()
    want = ref.attend(torch, q[130:], k[130:], v[130:], ref.causal(torch, 10))
    ref.check(torch, want, out[130:], lse[130:], "bf16")


def test_bad_bounds_and_slots_of_prompts(env):
    torch, pbd = env
    hkv, D, page = 2, 64, 16
    q, k, v = (x.cuda() for x in ref.rows(torch, 60, 4, hkv, D, torch.bfloat16, False))
    want, _ = pbd.pbd_op_prompt_attention(q, k, v, i32(torch, [0, 20, 40, 60]))
    for starts, touched in (([0, 20, 10, 60], None), ([0, 20, 40, 61], 40), ([-1, 20, 40, 60], None), ([5, 5, 5, 70], 0)):
        out = torch.full_like(q, 7.0)
        ws = pbd.op_workspace(1 << 16)
        with pytest.raises(pbd.PbdError, match="PBD_ERR_DEVICE"):
            pbd.pbd_op_prompt_attention(q, k, v, i32(torch, starts), out=out, workspace=ws)
        if touched is not None:
            assert torch.equal(out[:touched], want[:touched]) and (out[touched:] == 7).all()
        pbd.pbd_op_prompt_attention(q, k, v, i32(torch, [0, 20, 40, 60]), out=out, workspace=ws)  # the workspace works again
        assert torch.equal(out, want)
    ck, cv = (torch.zeros(5, hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kv = pbd.PagedKV(ck, cv, i32(torch, [[0]]), i32(torch, [0]))
    slots = torch.arange(60, device="cuda")
    slots[7], slots[8], slots[9] = 80, 1 << 40, -(1 << 40)
    out = torch.empty_like(q)
    with pytest.raises(pbd.PbdError, match="PBD_ERR_DEVICE"):
        pbd.pbd_op_prompt_attention(q, k, v, i32(torch, [0, 20, 40, 60]), kv=kv, slots=slots, out=out)
    assert torch.equal(out, want)
    flat = ck.transpose(1, 2).reshape(80, hkv, D)
    keep = torch.tensor([i for i in range(60) if i not in (7, 8, 9)], device="cuda")
    assert torch.equal(flat[keep], k[keep]) and (flat[[7, 8, 9]] == 0).all() and (flat[60:] == 0).all()


# ------------------------------------------------------------------ trees

TREES = [
    # lens, nodes, hkv, group, D, page, layout
    ([1], [1], 1, 1, 64, 16, "heads"),
    ([512], [17], 8, 2, 128, 16, "heads"),
    ([0, 1, 15, 16, 17, 31, 33, 100], [64, 0, 1, 5, 33, 64, 17, 2], 2, 3, 128, 16, "heads"),
    ([0, 0], [1, 0], 2, 2, 64, 8, "tokens"),
    ([700, 0, 0, 3, 1300], [9, 3, 0, 30, 64], 2, 8, 64, 16, "tokens"),
    ([257, 90, 128], [64, 33, 64], 2, 7, 64, 24, "tokens"),
    ([129, 64, 1], [64, 64, 64], 1, 16, 128, 8, "heads"),
    ([200, 31], [7, 64], 2, 9, 256, 32, "heads"),
    ([77, 300], [20, 3], 1, 40, 128, 64, "tokens"),
    ([45], [10], 1, 33, 256, 1, "heads"),
    ([2500], [13], 1, 4, 256, 16, "tokens"),
    ([20000], [64], 1, 2, 128, 16, "heads"),
    ([37] * 150, [3] * 150, 2, 2, 64, 16, "heads"),
    ([0, 1, 17, 300, 64] * 40, [5, 0, 1, 16, 2] * 40, 1, 2, 64, 16, "heads"),
    ([30000, 10, 500, 0], [4, 64, 1, 2], 2, 7, 64, 5, "tokens"),
    ([127, 128, 129, 63, 64, 191], [1, 1, 64, 65 - 1, 64, 2], 1, 4, 128, 16, "heads"),
    # units of one and of two tiles of rows in turns, many to a CTA
    ([300, 20, 0, 700] * 24, [1, 26, 64, 3] * 24, 2, 7, 64, 32, "tokens"),
    ([130, 0, 500, 40, 260] * 30, [64, 2, 1, 33, 40] * 30, 2, 4, 128, 16, "heads"),
    ([1000, 90] * 40, [17, 64] * 40, 1, 16, 128, 8, "heads"),
]


@pytest.mark.parametrize("chain", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", TREES, ids=lambda s: "%dx%s-%s" % (len(s[0]), max(s[0]), "-".join(map(str, s[2:]))))
def test_trees_match_64_bits(env, shape, dtype, chain):
    """Slots that no sequence holds are NaN, and table entries behind a sequence lie outside the cache."""
    torch, pbd = env
    lens, nodes, hkv, group, D, page, layout = shape
    dt, hq = getattr(torch, ref.DT[dtype]), hkv * group
    c = ref.tree_case(torch, lens, nodes, hkv, D, page, dt, layout)
    g = to_gpu(torch, c)
    T = sum(nodes) + 2
    q, kn, vn = ref.rows(torch, T, hq, hkv, D, dt, chain, nodes)
    gq, gk, gv = ref.fused_to_gpu(torch, q, kn, vn)
    parents = torch.cat([ref.trees(torch, nodes), torch.full((2,), 99, dtype=torch.int32)])
    starts = ref.starts_of(torch, nodes)
    pos = torch.arange(T, dtype=torch.int32) + 1000
    kv = pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"], weights=g["weights"], positions=g["positions"])
    out, lse = torch.full((T, hq, D), 7.0, dtype=dt, device="cuda"), torch.full((T, hq), 7.0, device="cuda")
    args = (gq, kv, gk, gv, starts.cuda(), None if chain else parents.cuda())
    pbd.pbd_op_tree_attention(*args, new_positions=pos.cuda(), out=out, lse=lse)
    want_pos = c["positions"].clone()
    for b, m in enumerate(nodes):
        at = slice(int(starts[b]), int(starts[b + 1]))
        if m:
            ref.check(torch, ref.tree_attention(torch, c, b, q[at], kn[at], vn[at], None if chain else parents[at]), out[at], lse[at], dtype)
        for i in range(m):
            j = lens[b] + i
            p, o = int(c["table"][b, j // page]), j % page
            c["k"][p, :, o], c["v"][p, :, o] = kn[at][i], vn[at][i]
            want_pos[b, :, j] = pos[at][i]
    assert (out[sum(nodes):] == 7).all() and (lse[sum(nodes):] == 7).all()
    assert same_bits(torch, g["k"], c["k"]) and same_bits(torch, g["v"], c["v"])
    assert torch.equal(g["positions"].cpu(), want_pos) and torch.equal(g["weights"].cpu(), c["weights"])
    out2, lse2 = pbd.pbd_op_tree_attention(*args, want_lse=True)
    n = sum(nodes)
    assert torch.equal(out2[:n], out[:n]) and torch.equal(lse2[:n], lse[:n])  # the same bits on every call


def test_a_tree_of_one_node_is_a_decoding_step(env):
    """One node a sequence: what pbd_op_decode_attention computes, to the rounding of p."""
    torch, pbd = env
    lens, hkv, group, D, page = [40, 0, 333, 129], 2, 4, 128, 16
    c = ref.tree_case(torch, lens, [1] * 4, hkv, D, page, torch.bfloat16, "heads")
    q, kn, vn = (x.cuda() for x in ref.rows(torch, 4, hkv * group, hkv, D, torch.bfloat16, False))
    a, b = to_gpu(torch, c), to_gpu(torch, c)
    out, lse = pbd.pbd_op_tree_attention(q, pbd.PagedKV(a["k"], a["v"], a["table"], a["lens"]), kn, vn, i32(torch, range(5)), want_lse=True)
    out2, lse2 = pbd.pbd_op_decode_attention(q, pbd.PagedKV(b["k"], b["v"], b["table"], b["lens"]), kn, vn, want_lse=True)
    assert same_bits(torch, a["k"], b["k"].cpu()) and same_bits(torch, a["v"], b["v"].cpu())
    for i, n in enumerate(lens):
        want = ref.tree_attention(torch, c, i, q[i:i + 1].cpu(), kn[i:i + 1].cpu(), vn[i:i + 1].cpu(), None)
        for o, l in ((out, lse), (out2, lse2)):
            ref.check(torch, want, o[i:i + 1], l[i:i + 1], "bf16")


@pytest.mark.parametrize("D,group", [(128, 2), (64, 7), (256, 4)])
def test_nodes_that_a_row_does_not_see_do_not_touch_it(env, D, group):
    torch, pbd = env
    lens, nodes, hkv, page = [100, 0, 290], [40, 64, 7], 2, 16
    c = ref.tree_case(torch, lens, nodes, hkv, D, page, torch.bfloat16, "heads")
    T = sum(nodes)
    q, kn, vn = ref.rows(torch, T, hkv * group, hkv, D, torch.bfloat16, False)
    parents = ref.trees(torch, nodes)
    for t, h, d, x in ((5, 0, 1, math.inf), (20, 1, 2, math.nan), (39, 0, D - 1, -math.inf), (44, 1, 0, math.nan), (103, 0, 7, math.inf),
                       (105, 1, D // 2, math.nan)):
        vn[t, h, d] = x
    # and one of the cached tokens of the last sequence
    p = int(c["table"][2, 3])
    c["v"][p, 0, 2, 5] = math.inf
    g = to_gpu(torch, c)
    starts = ref.starts_of(torch, nodes)
    out, lse = pbd.pbd_op_tree_attention(q.cuda(), pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"]), kn.cuda(), vn.cuda(), starts.cuda(),
                                         parents.cuda(), want_lse=True)
    for b in range(3):
        at = slice(int(starts[b]), int(starts[b + 1]))
        ref.check(torch, ref.tree_attention(torch, c, b, q[at], kn[at], vn[at], parents[at]), out[at], lse[at], "bf16")


def test_bad_trees(env):
    """Lengths, bounds, pages and parents that lie outside: reported, and no harm done to the other sequences."""
    torch, pbd = env
    lens, nodes, hkv, group, D, page = [50, 90, 20], [10, 20, 5], 1, 2, 64, 16
    T, dt = sum(nodes), torch.bfloat16
    q, kn, vn = ref.rows(torch, T, hkv * group, hkv, D, dt, False)
    starts, parents = ref.starts_of(torch, nodes), ref.trees(torch, nodes)
    good = ref.tree_case(torch, lens, nodes, hkv, D, page, dt, "heads")

    def call(c, starts, parents, code=True):
        g = to_gpu(torch, c)
        out, lse = torch.full((T, hkv * group, D), 7.0, dtype=dt, device="cuda"), torch.full((T, hkv * group), 7.0, device="cuda")
        args = (q.cuda(), pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"]), kn.cuda(), vn.cuda(), starts.cuda(), parents.cuda())
        if code:
            with pytest.raises(pbd.PbdError, match="PBD_ERR_DEVICE"):
                pbd.pbd_op_tree_attention(*args, out=out, lse=lse)
        else:
            pbd.pbd_op_tree_attention(*args, out=out, lse=lse)
        return out, lse, g
    want, _, _ = call(good, starts, parents, False)
    rest = [slice(0, 10), slice(30, 35)]
    # a length outside the table
    for n in (-1, good["cap"] - 19, 1 << 30):
        c = dict(good, lens=torch.tensor([50, n, 20], dtype=torch.int32))
        out, lse, g = call(c, starts, parents)
        assert all(torch.equal(out[at], want[at]) for at in rest) and (out[10:30] == 7).all() and (lse[10:30] == 7).all()
    # bounds
    out, _, _ = call(good, torch.tensor([0, 10, 5, 35], dtype=torch.int32), parents)
    assert torch.equal(out[:5], want[:5])
    out, _, _ = call(good, torch.tensor([0, 10, 30, 36], dtype=torch.int32), parents)
    assert torch.equal(out[:30], want[:30]) and (out[30:] == 7).all()
    # parents that are not before their node count as the cached tokens
    bad, fixed = parents.clone(), parents.clone()
    bad[10 + 4], bad[10 + 7], bad[10 + 9] = 4, -2, 1 << 30
    fixed[10 + 4] = fixed[10 + 7] = fixed[10 + 9] = -1
    assert torch.equal(call(good, starts, bad)[0], call(good, starts, fixed, False)[0])
    # a page outside the cache: in the middle of the cached tokens, and where the nodes go
    c = dict(good, table=good["table"].clone())
    c["table"][1, 2] = c["k"].shape[0]
    out, lse, g = call(c, starts, parents)
    assert all(torch.equal(out[at], want[at]) for at in rest)
    sees = torch.cat([torch.ones(20, 90, dtype=torch.bool), ref.ancestors(torch, parents[10:30].tolist())], 1)
    sees[:, 32:48] = False
    k, v = (torch.cat([kvref.rows_of(good, good[x], 1, 90).transpose(0, 1), new[10:30].double()]) for x, new in (("k", kn), ("v", vn)))
    ref.check(torch, ref.attend(torch, q[10:30], k, v, sees), out[10:30], lse[10:30], "bf16")
    c["table"][1, 2], c["table"][1, 6] = good["table"][1, 2], -1  # slots 96 to 111: nodes 6 to 19
    out, lse, g = call(c, starts, parents)
    sees[:, 32:48], sees[:, 96:] = True, False
    ref.check(torch, ref.attend(torch, q[10:30], k, v, sees), out[10:30], lse[10:30], "bf16")
    for j in range(96):
        p, o = int(good["table"][1, j // page]), j % page
        if j >= 90:
            assert torch.equal(g["k"][p, :, o].cpu(), kn[10 + j - 90])
    # nothing to see at all
    c = dict(good, lens=torch.tensor([50, 0, 20], dtype=torch.int32), table=good["table"].clone())
    c["table"][1, :] = -1
    out, lse, _ = call(c, starts, parents)
    assert (out[10:30] == 0).all() and (lse[10:30] == -math.inf).all() and all(torch.equal(out[at], want[at]) for at in rest)


# ------------------------------------------------------------------ pages

def run_assign(torch, pbd, state, page, lens, n_new, most, n_pages, ws):
    table, held, free, per = state["table"], state["held"], state["free"], state["per"]
    pool = state["pool"]
    before = [pool.page_table.clone(), pool.held.clone(), pool.free.clone(), pool.n_free.clone()]
    slots, pos = ref.assign(table, held, free, lens, n_new, page)
    got = pbd.pbd_op_assign_pages(pool, i32(torch, lens), i32(torch, n_new), most, workspace=ws)
    assert got.starts.tolist() == ref.starts_of(torch, n_new).tolist()
    assert got.slots.tolist() == slots + [-1] * (most - len(slots))
    assert got.positions.tolist() == pos + [0] * (most - len(pos))
    assert pool.held.tolist() == held and pool.n_free.tolist() == [len(free)]
    assert pool.free.tolist()[:len(free)] == free and torch.equal(pool.free[len(free):], before[2][len(free):])
    rows = pool.page_table.tolist()
    for b, h in enumerate(held):
        assert rows[b][:h] == table[b][:h]
        if h <= int(before[1][b]):
            assert rows[b][h:] == before[0][b].tolist()[h:]
    # every page is somewhere, once
    assert sorted(free + [x for b, h in enumerate(held) for x in table[b][:h]]) == list(range(n_pages))


@pytest.mark.parametrize("B,page,top", [(1, 16, 100), (1, 1, 40), (8, 16, 2000), (33, 5, 100), (1024, 16, 60), (257, 64, 3000), (64, 8, 1)])
def test_pages_follow_lengths(env, B, page, top):
    """A pool over many steps: sequences grow, are cut back, end and begin."""
    torch, pbd = env
    g = torch.Generator().manual_seed(B * 7 + page)
    per = (2 * top + 70) // page + 1
    n_pages = B * per
    table = torch.full((B, per), -5, dtype=torch.int32, device="cuda")
    state = dict(table=[[-5] * per for _ in range(B)], held=[0] * B, free=list(range(n_pages - 1, -1, -1)), per=per,
                 pool=pbd.PagePool(table, page, n_pages))
    ws = pbd.op_workspace(pbd.assign_pages_workspace_bytes(B))
    lens = [0] * B
    for step in range(6):
        r = torch.rand(B, 3, generator=g).tolist()
        new = [0 if x < 0.2 else 1 if x < 0.5 else int(y * top) for x, y, _ in r]
        most = sum(new) + (0, 1, 9000)[step % 3]
        run_assign(torch, pbd, state, page, lens, new, most, n_pages, ws)
        lens = [0 if z < 0.25 else (n + m) // 2 if z < 0.5 else min(n + m, top) for n, m, (_, _, z) in zip(lens, new, r)]


def test_many_packed_rows_and_the_last_page(env):
    torch, pbd = env
    for lens, new, page in (([0] * 3, [100000, 0, 70001], 16), ([5, 0], [123456, 1], 1)):
        need = [-(-(n + m) // page) for n, m in zip(lens, new)]
        n_pages, per = sum(need), max(need)
        held = [-(-n // page) for n in lens]
        perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).tolist()
        table = [[0] * per for _ in lens]
        for b, h in enumerate(held):
            for i in range(h):
                table[b][i] = perm.pop()
        free = list(perm)
        pool = pbd.PagePool(i32(torch, table), page, n_pages, held=i32(torch, held), free=i32(torch, free + [9] * (n_pages - len(free))),
                            n_free=i32(torch, [len(free)]))
        state = dict(table=table, held=held, free=free, per=per, pool=pool)
        run_assign(torch, pbd, state, page, lens, new, sum(new) + 7, n_pages, None)  # all pages are taken
        run_assign(torch, pbd, state, page, [0] * len(lens), [0] * len(lens), 0, n_pages, None)  # and given back


def test_what_cannot_be_assigned_changes_nothing(env):
    torch, pbd = env
    page, n_pages = 4, 6
    # status of each: 5 a length, 7 a page, 8 not enough
    good = dict(table=[[3, 5, 0], [1, 0, 0]], held=[2, 1], free=[0, 2, 4, 9, 9, 9], n_free=3, lens=[7, 3], new=[1, 4], most=8)
    cases = [dict(lens=[-1, 3]), dict(new=[1, -1]), dict(lens=[12, 3]), dict(new=[1, 10]), dict(new=[1 << 30, 4]), dict(most=4),
             dict(held=[2, -1]), dict(held=[2, 4]), dict(n_free=-1), dict(n_free=7), dict(n_free=4), dict(held=[3, 1], n_free=3),
             dict(free=[0, 2, 6, 9, 9, 9]), dict(free=[0, 2, -1, 9, 9, 9]), dict(table=[[3, 6, 0], [1, 0, 0]], lens=[0, 3], new=[0, 4]),
             dict(lens=[12, 12], new=[0, 0], n_free=2), dict(lens=[7, 3], new=[5, 9], n_free=2), dict(lens=[7, 3], new=[5, 9], n_free=2, most=14)]
    for kw in cases:
        for pad in (0, 9000):  # by one kernel and by two
            c = dict(good, **kw)
            pool = pbd.PagePool(i32(torch, c["table"]), page, n_pages, held=i32(torch, c["held"]), free=i32(torch, c["free"]), n_free=i32(torch, [c["n_free"]]))
            out = pbd.AssignedPages(torch.full((3,), 5, dtype=torch.int32, device="cuda"),
                                    torch.full((c["most"] + pad,), 5, dtype=torch.int64, device="cuda"),
                                    torch.full((c["most"] + pad,), 5, dtype=torch.int32, device="cuda"))
            if kw == dict(most=4) and pad:
                continue
            with pytest.raises(pbd.PbdError, match="PBD_ERR_DEVICE"):
                pbd.pbd_op_assign_pages(pool, i32(torch, c["lens"]), i32(torch, c["new"]), c["most"] + pad, out=out)
            assert pool.page_table.tolist() == c["table"] and pool.held.tolist() == c["held"], kw
            assert pool.free.tolist() == c["free"] and pool.n_free.tolist() == [c["n_free"]], kw
            assert (out.starts == 0).all() and (out.slots == -1).all() and (out.positions == 0).all(), kw
    # (with one more the first of the shortages above is none: 3 held and 3 free pages are the 6 of 24 tokens)
    pool = pbd.PagePool(i32(torch, good["table"]), page, n_pages, held=i32(torch, [2, 1]), free=i32(torch, good["free"]), n_free=i32(torch, [3]))
    pbd.pbd_op_assign_pages(pool, i32(torch, [12, 12]), i32(torch, [0, 0]), 8)
    assert pool.page_table.tolist() == [[3, 5, 4], [1, 2, 0]] and pool.n_free.tolist() == [0] and pool.held.tolist() == [3, 3]
    # a page held before that lies outside: its rows get no slot
    pool = pbd.PagePool(i32(torch, [[3, 6, 0], [1, 0, 0]]), page, n_pages, held=i32(torch, [2, 1]), free=i32(torch, good["free"]), n_free=i32(torch, [3]))
    ws = pbd.op_workspace(1024)
    got = pbd.pbd_op_assign_pages(pool, i32(torch, [6, 3]), i32(torch, [4, 1]), 6, workspace=ws, sync=False)
    with pytest.raises(pbd.PbdError, match="PBD_ERR_DEVICE"):
        pbd.pbd_op_status(ws)
    assert got.slots.tolist() == [-1, -1, 16, 17, 7, -1] and got.positions.tolist() == [6, 7, 8, 9, 3, 0]


# ------------------------------------------------------------------ accepted paths

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,page,layout,hkv", [(128, 16, "heads", 8), (64, 5, "tokens", 3), (256, 64, "heads", 1), (64, 1, "heads", 2)])
def test_accepted_paths_move(env, D, page, layout, hkv, dtype):
    torch, pbd = env
    dt = getattr(torch, ref.DT[dtype])
    lens, g = [0, 100, 31, 16, 77, 5, 63], torch.Generator().manual_seed(D + page)
    nodes, most = [64, 64, 7, 1, 33, 0, 64], 64
    paths = [list(range(64)), list(range(1, 64, 2)), [6], [0], sorted(torch.randperm(33, generator=g)[:20].tolist()), [], list(range(8, 64))]
    c = kvref.make_cache(torch, [n + m for n, m in zip(lens, nodes)], hkv, D, page, dt, layout, extra=0)
    c["lens"] = torch.tensor(lens, dtype=torch.int32)
    gpu = to_gpu(torch, c)
    kv = pbd.PagedKV(gpu["k"], gpu["v"], gpu["table"], gpu["lens"], weights=gpu["weights"], positions=gpu["positions"])
    path = i32(torch, [p + [-7] * (most - len(p)) for p in paths])
    pbd.pbd_op_commit_path(kv, path, i32(torch, [len(p) for p in paths]))
    old = {n: c[n].clone() for n in ("k", "v", "weights", "positions")}
    for b, p in enumerate(paths):
        for i, x in enumerate(p):
            s, d = lens[b] + x, lens[b] + i
            for n in ("k", "v"):
                c[n][int(c["table"][b, d // page]), :, d % page] = old[n][int(c["table"][b, s // page]), :, s % page]
            for n in ("weights", "positions"):
                c[n][b, :, d] = old[n][b, :, s]
    assert same_bits(torch, gpu["k"], c["k"]) and same_bits(torch, gpu["v"], c["v"])
    assert torch.equal(gpu["weights"].cpu(), c["weights"]) and torch.equal(gpu["positions"].cpu(), c["positions"])


def test_bad_paths_leave_their_sequence(env):
    torch, pbd = env
    lens, page, hkv, D = [20, 30], 8, 2, 64
    c = kvref.make_cache(torch, [40, 50], hkv, D, page, torch.bfloat16, extra=0)
    c["lens"] = torch.tensor(lens, dtype=torch.int32)

    def call(path, n, lens=lens, table=None):
        gpu = to_gpu(torch, dict(c, lens=torch.tensor(lens, dtype=torch.int32), table=c["table"] if table is None else table))
        kv = pbd.PagedKV(gpu["k"], gpu["v"], gpu["table"], gpu["lens"], weights=gpu["weights"], positions=gpu["positions"])
        ws = pbd.op_workspace(1024)
        pbd.pbd_op_commit_path(kv, i32(torch, path), i32(torch, n), workspace=ws, sync=False)
        return gpu, ws
    want, ws = call([[2, 5, 9], [1, 2, 3]], [3, 0])
    pbd.pbd_op_status(ws)
    for path, n, ln in (([[2, 5, 9], [3, 3, 4]], [3, 3], lens), ([[2, 5, 9], [3, 2, 4]], [3, 2], lens), ([[2, 5, 9], [-1, 2, 4]], [3, 2], lens),
                        ([[2, 5, 9], [1, 2, 64]], [3, 3], lens), ([[2, 5, 9], [1, 2, 3]], [3, 4], lens), ([[2, 5, 9], [1, 2, 3]], [3, -1], lens),
                        ([[2, 5, 9], [1, 2, 3]], [3, 3], [20, -1]), ([[2, 5, 9], [1, 2, 3]], [3, 3], [20, 57]), ([[2, 5, 9], [1, 2, 27]], [3, 3], lens)):
        got, ws = call(path, n, ln)
        with pytest.raises(pbd.PbdError, match="PBD_ERR_DEVICE"):
            pbd.pbd_op_status(ws)
        for x in ("k", "v", "weights", "positions"):
            assert torch.equal(torch.nan_to_num(got[x].float()), torch.nan_to_num(want[x].float())), (path, n, ln)
    # a bad page: its moves are left out (slots 32 to 39 of the second sequence: nodes 2 to 9)
    table = c["table"].clone()
    table[1, 4] = 1 << 30
    got, ws = call([[2, 5, 9], [1, 5, 12]], [3, 3], table=table)
    with pytest.raises(pbd.PbdError, match="PBD_ERR_DEVICE"):
        pbd.pbd_op_status(ws)
    for x in ("k", "v"):
        y = want[x].cpu().clone()
        s, d = 31, 30
        y[int(c["table"][1, d // page]), :, d % page] = c[x][int(c["table"][1, s // page]), :, s % page]
        assert same_bits(torch, got[x], y)


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype,D,group,page", [("bf16", 128, 2, 16), ("fp16", 64, 3, 8)])
def test_prompts_trees_and_paths_as_one_loop(env, dtype, D, group, page):
    """Prompts into a pool's pages, three verified trees each, then one plain step; a sequence ends and another takes its place.
    Every step against the tokens that each sequence holds by then."""
    torch, pbd = env
    dt, hkv, B, per, n_pages = getattr(torch, ref.DT[dtype]), 2, 4, 40, 90
    hq, gen = hkv * group, torch.Generator().manual_seed(5)
    table = torch.zeros(B, per, dtype=torch.int32, device="cuda")
    pool = pbd.PagePool(table, page, n_pages)
    k, v = (torch.full((n_pages, hkv, page, D), math.nan, dtype=dt, device="cuda") for _ in range(2))
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    positions = torch.zeros(B, hkv, per * page, dtype=torch.int32, device="cuda")
    kv = pbd.PagedKV(k, v, table, lens, positions=positions)
    T = 256
    need = max(pbd.assign_pages_workspace_bytes(B), pbd.prompt_attention_workspace_bytes(T, B, hq, hkv, D),
               pbd.tree_attention_workspace_bytes(kv, T, hq), pbd.commit_path_workspace_bytes(kv, 64),
               pbd.decode_attention_workspace_bytes(kv, hq))
    ws = pbd.op_workspace(need)
    held = [[torch.zeros(0, hkv, D, dtype=dt)] * 2 for _ in range(B)]  # K and V of the tokens of each sequence

    def new_rows(n):
        q, a, b = ref.rows(torch, T, hq, hkv, D, dt, False, [n], seed=int(torch.randint(1 << 30, (1,), generator=gen)))
        return q, a, b

    def prompts(counts):
        got = pbd.pbd_op_assign_pages(pool, lens, i32(torch, counts), T, workspace=ws)
        q, a, b = new_rows(sum(counts))
        out, lse = pbd.pbd_op_prompt_attention(q.cuda(), a.cuda(), b.cuda(), got.starts, kv=kv, slots=got.slots, want_lse=True, workspace=ws)
        s = got.starts.tolist()
        for i, n in enumerate(counts):
            if n:
                at = slice(s[i], s[i + 1])
                ref.check(torch, ref.attend(torch, q[at], a[at], b[at], ref.causal(torch, n)), out[at], lse[at], dtype)
                held[i] = [a[at], b[at]]
        lens.add_(i32(torch, counts))

    prompts([33, 70, 1, 0])
    for rnd in range(3):
        nodes = [[17, 40, 64, 0], [1, 64, 5, 0], [30, 2, 64, 16]][rnd]
        if rnd == 2:  # the second has ended and makes room for another's prompt
            lens[1] = 0
            held[1] = [torch.zeros(0, hkv, D, dtype=dt)] * 2
            pbd.pbd_op_assign_pages(pool, lens, i32(torch, [0] * 4), 0, workspace=ws)
            before = lens.clone()
            lens.zero_()  # (prompts of the others' call are empty)
            lens.copy_(before)
            got = pbd.pbd_op_assign_pages(pool, lens, i32(torch, [0, 55, 0, 21]), T, workspace=ws)
            q, a, b = new_rows(76)
            pbd.pbd_op_prompt_attention(q.cuda(), a.cuda(), b.cuda(), got.starts, kv=kv, slots=got.slots, workspace=ws)
            held[1], held[3] = [a[:55], b[:55]], [a[55:76], b[55:76]]
            lens.add_(i32(torch, [0, 55, 0, 21]))
        got = pbd.pbd_op_assign_pages(pool, lens, i32(torch, nodes), T, workspace=ws)
        q, a, b = new_rows(sum(nodes))
        parents = ref.trees(torch, nodes, seed=rnd)
        gp = torch.full((T,), -1, dtype=torch.int32)
        gp[:sum(nodes)] = parents
        out, lse = pbd.pbd_op_tree_attention(q.cuda(), kv, a.cuda(), b.cuda(), got.starts, gp.cuda(), new_positions=got.positions,
                                             want_lse=True, workspace=ws)
        s = got.starts.tolist()
        path, count = [[0] * 64 for _ in range(B)], [0] * B
        for i, m in enumerate(nodes):
            if not m:
                continue
            at = slice(s[i], s[i + 1])
            sees = ref.ancestors(torch, parents[at].tolist())
            n = held[i][0].shape[0]
            both = [torch.cat([x, y]) for x, y in zip(held[i], (a[at], b[at]))]
            want = ref.attend(torch, q[at], both[0], both[1], torch.cat([torch.ones(m, n, dtype=torch.bool), sees], 1))
            ref.check(torch, want, out[at], lse[at], dtype)
            leaf = int(torch.randint(m, (1,), generator=gen))
            took = sees[leaf].nonzero()[:, 0].tolist()
            path[i][:len(took)], count[i] = took, len(took)
            held[i] = [torch.cat([x, y[took]]) for x, y in zip(held[i], (a[at], b[at]))]
        pbd.pbd_op_commit_path(kv, i32(torch, path), i32(torch, count), workspace=ws)
        lens.add_(i32(torch, count))
        assert lens.tolist() == [h[0].shape[0] for h in held]
    pbd.pbd_op_assign_pages(pool, lens, i32(torch, [1] * B), B, workspace=ws)
    q, a, b = (x[:B].contiguous() for x in new_rows(B))
    out, lse = pbd.pbd_op_decode_attention(q.cuda(), kv, a.cuda(), b.cuda(), want_lse=True, workspace=ws)
    for i in range(B):
        both = [torch.cat([x, y]) for x, y in zip(held[i], (a[i:i + 1], b[i:i + 1]))]
        n = both[0].shape[0]
        ref.check(torch, ref.attend(torch, q[i:i + 1], both[0], both[1], torch.ones(1, n, dtype=torch.bool)), out[i:i + 1], lse[i:i + 1], dtype)
    assert pool.held.tolist() == [-(-(n + 1) // page) for n in lens.tolist()]


def test_a_step_captured_and_replayed(env):
    """Pages, trees and paths in one graph on a stream of its own, replayed as lengths move on; eager calls on another workspace
    in between."""
    torch, pbd = env
    hkv, group, D, page, B, per = 2, 2, 128, 16, 3, 30
    hq, T = hkv * group, 3 * 20
    n_pages = B * per
    gen = torch.Generator(device="cuda").manual_seed(3)

    def state():
        torch.manual_seed(1)
        k, v = (torch.randn(n_pages, hkv, page, D, device="cuda").bfloat16() for _ in range(2))
        pool = pbd.PagePool(torch.zeros(B, per, dtype=torch.int32, device="cuda"), page, n_pages)
        lens = i32(torch, [0, 0, 0])
        kv = pbd.PagedKV(k, v, pool.page_table, lens)
        pbd.pbd_op_assign_pages(pool, lens, i32(torch, [100, 3, 250]), 400)
        lens.copy_(i32(torch, [100, 3, 250]))
        need = max(1024, pbd.tree_attention_workspace_bytes(kv, T, hq))
        s = dict(kv=kv, pool=pool, lens=lens, ws=pbd.op_workspace(need), q=torch.zeros(T, hq, D, dtype=torch.bfloat16, device="cuda"),
                 kn=torch.zeros(T, hkv, D, dtype=torch.bfloat16, device="cuda"), vn=torch.zeros(T, hkv, D, dtype=torch.bfloat16, device="cuda"),
                 nodes=i32(torch, [20, 20, 20]), parents=torch.full((T,), -1, dtype=torch.int32, device="cuda"),
                 path=torch.zeros(B, 4, dtype=torch.int32, device="cuda"), took=i32(torch, [0] * 3),
                 out=torch.zeros(T, hq, D, dtype=torch.bfloat16, device="cuda"), lse=torch.zeros(T, hq, device="cuda"),
                 packed=pbd.AssignedPages(i32(torch, [0] * 4), torch.zeros(T, dtype=torch.int64, device="cuda"), i32(torch, [0] * T)))
        return s

    def step(s):
        pbd.pbd_op_assign_pages(s["pool"], s["lens"], s["nodes"], T, out=s["packed"], workspace=s["ws"], sync=False)
        pbd.pbd_op_tree_attention(s["q"], s["kv"], s["kn"], s["vn"], s["packed"].starts, s["parents"], out=s["out"], lse=s["lse"],
                                  workspace=s["ws"], sync=False)
        pbd.pbd_op_commit_path(s["kv"], s["path"], s["took"], workspace=s["ws"], sync=False)
        s["lens"].add_(s["took"])

    a, b = state(), state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(a)
    for i in range(5):
        nodes = [[20, 20, 20], [1, 0, 20], [7, 20, 0], [20, 5, 5], [2, 2, 2]][i]
        for s in (a, b):
            g2 = torch.Generator(device="cuda").manual_seed(i)
            for n in ("q", "kn", "vn"):
                s[n].normal_(generator=g2)
            s["nodes"].copy_(i32(torch, nodes))
            s["parents"][:sum(nodes)] = ref.trees(torch, nodes, seed=i).cuda()
            s["path"].copy_(i32(torch, [[0, 1, 3, 4], [0, 2, 3, 9], [1, 2, 3, 4]]))
            s["took"].copy_(i32(torch, [min(n, 2) // 2 * (1 + i % 2) if n < 5 else 4 for n in nodes]))
        graph.replay()
        step(b)
        n = sum(nodes)
        assert torch.equal(a["out"][:n], b["out"][:n]) and torch.equal(a["lse"][:n], b["lse"][:n])
        assert torch.equal(a["lens"], b["lens"]) and torch.equal(a["packed"].slots, b["packed"].slots)
        assert torch.equal(a["pool"].page_table, b["pool"].page_table)
        assert torch.equal(a["kv"].k, b["kv"].k) and torch.equal(a["kv"].v, b["kv"].v)
        pbd.pbd_op_status(a["ws"])


def test_prompts_on_two_streams_and_in_a_graph(env):
    torch, pbd = env
    lens, hkv, group, D = [300, 0, 77, 140], 2, 4, 128
    T = sum(lens)
    sets = [[x.cuda() for x in ref.rows(torch, T, hkv * group, hkv, D, torch.bfloat16, False, seed=i)] for i in range(4)]
    starts = ref.starts_of(torch, lens).cuda()
    want = [pbd.pbd_op_prompt_attention(*s, starts)[0] for s in sets]
    streams, got = [torch.cuda.Stream() for _ in range(4)], []
    for st, s in zip(streams, sets):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            got.append(pbd.pbd_op_prompt_attention(*s, starts, sync=False)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    q, k, v = (x.clone() for x in sets[0])
    out, ws, n = torch.zeros_like(q), pbd.op_workspace(pbd.prompt_attention_workspace_bytes(T, 4, hkv * group, hkv, D)), starts.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pbd.pbd_op_prompt_attention(q, k, v, n, out=out, workspace=ws, sync=False)
    for s, w in zip(sets, want):
        for x, y in zip((q, k, v), s):
            x.copy_(y)
        graph.replay()
        assert torch.equal(out, w)
    n.copy_(i32(torch, [0, 100, 100, 300, 300]))  # other lengths
    out.fill_(7.0)
    graph.replay()
    other = pbd.pbd_op_prompt_attention(q, k, v, n)[0]
    assert torch.equal(out[:300], other[:300]) and (out[300:] == 7).all()
    pbd.pbd_op_status(ws)
