"""Timed and compared cases of the operators that bring prompts and drafted trees into a paged key-value cache: pages and slot
maps from request lengths, attention over packed prompts whose K and V go into the cache, attention of drafted trees over
the cache, and the move of an accepted path's rows.

Sizes are those of the package's own shapes and workloads (16 query over 8 KV heads of 128, pages of 16 tokens, verify
blocks of 17 rows, its batch of eight ragged prompts) and of generic neighbours: other groups, head sizes, page lengths,
odd lengths.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
BATCH8 = "1757,725,451,791,997,1715,1065,420"
NODES = 64  # of a tree at most


def _ints(text):
    return [int(x) for x in text.split(",")]


def _text(values):
    return ",".join(str(v) for v in values)


# ------------------------------------------------------------------ the cases

def listed():
    ragged = _text([0, 1, 2, 15, 16, 17, 33, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 300, 391, 450, 511, 512,
                    513, 640, 777, 901, 1000, 1023, 1024, 1025, 1300])
    cached = _text([0, 1, 15, 16, 17, 33, 64, 100, 127, 128, 129, 200, 255, 257, 300, 391, 450, 511, 512, 513, 640, 777,
                    800, 901, 1000, 1023, 1024, 1025, 1100, 1200, 1300, 1377, 1500, 1600, 1733, 1800, 1999, 2047, 2048, 2049,
                    2200, 2300, 2500, 2700, 2900, 3001, 3300, 3500, 3777, 4000, 4095, 4096, 4097, 4500, 4800, 5000, 5333,
                    5600, 6000, 6400, 6661, 7000, 7500, 8000])
    return [
        # pages for a verify block of the batch of eight, and for the next one after some were accepted: the smallest call
        dict(name="pages-batch8", kind="pages", lens=BATCH8, new=_text([17] * 8), lens2=_text(n + 60 for n in _ints(BATCH8)),
             new2=_text([17] * 8), page=16, spare=64, pad=0),
        # a large server between two steps: prompts arrive, others end and give their pages back, most decode on; packed
        # rows padded to a captured step's size
        dict(name="pages-512-turnover", kind="pages", lens=_text(0 if i % 4 == 0 else 37 * i for i in range(512)),
             new=_text(997 + i if i % 4 == 0 else 1 + i % 17 for i in range(512)),
             lens2=_text(0 if i % 5 == 0 else 37 * i + 20 for i in range(512)),
             new2=_text(0 if i % 10 == 0 else (1311 - i if i % 5 == 0 else 1) for i in range(512)), page=16, spare=500, pad=4096),
        # a 512-token prompt: the smallest, latency counts
        dict(name="prompt-512", kind="prompt", lens="512", hkv=8, group=2, D=128, page=16, dtype="bf16", layout="heads",
             store=True, fused=False, pad=0),
        # the batch of eight ragged prompts, q, k and v cut out of one projection's rows
        dict(name="prompt-batch8", kind="prompt", lens=BATCH8, hkv=8, group=2, D=128, page=16, dtype="bf16", layout="heads",
             store=True, fused=True, pad=0),
        # one long prompt: the largest
        dict(name="prompt-16384", kind="prompt", lens="16384", hkv=8, group=2, D=128, page=16, dtype="bf16", layout="heads",
             store=True, fused=False, pad=0),
        # a serving batch from empty to long, seven query heads a KV head, packed rows padded behind the last sequence
        dict(name="prompt-32-ragged", kind="prompt", lens=ragged, hkv=4, group=7, D=64, page=32, dtype="fp16",
             layout="tokens", store=True, fused=True, pad=77),
        # a verify block (a chain) behind a 512-token prompt: the smallest, latency counts
        dict(name="tree-chain-17", kind="tree", lens="512", nodes="17", chain=True, hkv=8, group=2, D=128, page=16,
             dtype="bf16", layout="heads", pad=0),
        # trees of up to 64 drafted tokens for the batch of eight
        dict(name="tree-batch8", kind="tree", lens=BATCH8, nodes="64,64,33,1,0,47,64,17", chain=False, hkv=8, group=2, D=128,
             page=16, dtype="bf16", layout="heads", pad=0),
        # a tree behind one very long context: work split over its length and joined
        dict(name="tree-131071", kind="tree", lens="131071", nodes="64", chain=False, hkv=8, group=2, D=128, page=16,
             dtype="bf16", layout="heads", pad=0),
        # a serving batch from empty to long contexts, seven query heads a KV head, token-major pages, small trees
        dict(name="tree-64-ragged", kind="tree", lens=cached, nodes=_text(1 + (7 * i) % 26 for i in range(64)), chain=False,
             hkv=4, group=7, D=64, page=32, dtype="fp16", layout="tokens", pad=5),
        # the accepted paths of the batch of eight: the smallest
        dict(name="commit-batch8", kind="commit", lens=BATCH8, nodes="64,64,33,1,0,47,64,17", most=8, hkv=8, D=128, page=16,
             dtype="bf16", layout="heads"),
        # of a large batch, long paths
        dict(name="commit-512", kind="commit", lens=_text(11 + 3 * i for i in range(512)), nodes=_text(1 + i % 64 for i in range(512)),
             most=33, hkv=8, D=128, page=16, dtype="bf16", layout="tokens"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["pages", "prompt", "prompt", "tree", "tree", "commit"])
    page = rng.choice([1, 8, 16, 16, 24, 32, 64])
    if kind == "pages":
        B = _log(rng, 1, 1024)
        top = _log(rng, 8, min(30_000, 1_000_000 // B))
        lens = [rng.randint(0, top) for _ in range(B)]
        new = [rng.choice([0, 1, 1, 17, rng.randint(0, top)]) for _ in range(B)]
        lens2 = [rng.choice([0, n + m, n + m // 2]) for n, m in zip(lens, new)]
        new2 = [rng.choice([0, 1, 1, 17, rng.randint(0, top)]) for _ in range(B)]
        return dict(kind=kind, lens=_text(lens), new=_text(new), lens2=_text(lens2), new2=_text(new2), page=page,
                    spare=rng.choice([0, 3, 400]), pad=rng.choice([0, 0, 1, 300]))
    D = rng.choice([64, 128, 128, 256])
    hkv = rng.choice([1, 2, 4, 8, 8])
    common = dict(kind=kind, hkv=hkv, D=D, page=page, dtype=rng.choice(["bf16", "fp16"]), layout=rng.choice(["heads", "tokens"]))
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16])
    if kind == "prompt":
        B = _log(rng, 1, 32)
        # (padded to the longest, no more score values than the longest listed prompt's, nor more work)
        most = int(math.sqrt(16 * 16384 ** 2 * 128 / (B * hkv * group * max(D, 128))))
        top = _log(rng, 20, min(16384, most))
        lens = [_log(rng, max(1, top // 16), top) if b == 0 or rng.random() < 0.95 else rng.choice([0, 1]) for b in range(B)]
        return dict(common, lens=_text(lens), group=group, store=rng.random() < 0.7, fused=rng.random() < 0.5, pad=rng.choice([0, 0, 1, 150]))
    B = _log(rng, 1, 48)
    most = min(100_000, 130_000_000 // (B * hkv * max(D, 128)))
    top = _log(rng, 40, most)
    lens = [_log(rng, max(1, top // 8), top) if rng.random() < 0.95 else 0 for _ in range(B)]
    widest = rng.choice([1, 8, 17, 33, NODES])
    nodes = [rng.randint(1, widest) if b == 0 or rng.random() < 0.95 else 0 for b in range(B)]
    if kind == "tree":
        return dict(common, lens=_text(lens), nodes=_text(nodes), group=group, chain=rng.random() < 0.3, pad=rng.choice([0, 0, 3]))
    return dict(common, lens=_text(lens), nodes=_text(nodes), most=rng.choice([1, 4, 16, NODES]))


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 1000003 + 23)


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dtype)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _starts(counts):
    s = [0]
    for n in counts:
        s.append(s[-1] + n)
    return s


def _cache(case, g, lens, filled):
    """Pages in random order for `lens` slots a sequence, some of them nobody's; entries behind a sequence's last page are
    valid ones."""
    ps, hkv, D = case["page"], case["hkv"], case["D"]
    used = [max(1, -(-n // ps)) for n in lens]
    per, n_pages = max(used), sum(used) + 3
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    first, last = torch.tensor(_starts(used)[:-1], device=DEV), torch.tensor(used, device=DEV) - 1
    table = perm[first[:, None] + torch.minimum(torch.arange(per, device=DEV)[None], last[:, None])]
    shape = (n_pages, hkv, ps, D) if case["layout"] == "heads" else (n_pages, ps, hkv, D)
    dt = TYPES[case["dtype"]]
    k, v = (_normal(g, shape, dt) if filled else torch.zeros(shape, dtype=dt, device=DEV) for _ in range(2))
    if case["layout"] == "tokens":
        k, v = k.transpose(1, 2), v.transpose(1, 2)  # [page, head, slot, D] by strides
    return dict(k=k, v=v, table=table.contiguous(), cap=per * ps)


def _pages_inputs(case, g):
    """A pool in the middle of its life: pages held in no order, the free ones shuffled."""
    ps, lens, new, lens2, new2 = case["page"], *(_ints(case[n]) for n in ("lens", "new", "lens2", "new2"))
    B = len(lens)
    need = [[-(-(n + m) // ps) for n, m in zip(a, b)] for a, b in ((lens, new), (lens2, new2))]
    held = [-(-n // ps) for n in lens]
    n_pages = max(1, max(sum(need[0]), sum(need[1]), sum(held)) + case["spare"])
    per = max(1, max(need[0]), max(need[1]), max(held))
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    first, h = torch.tensor(_starts(held)[:-1], device=DEV), torch.tensor(held, device=DEV)
    at = first[:, None] + torch.arange(per, device=DEV)[None]
    inside = torch.arange(per, device=DEV)[None] < h[:, None]
    table = torch.where(inside, perm[at.clamp(max=n_pages - 1)], 0).to(torch.int32).contiguous()
    free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    n_free = n_pages - sum(held)
    free[:n_free] = perm[sum(held):]
    return dict(table=table, held=_i32(held), free=free, n_free=_i32([n_free]), B=B, n_pages=n_pages,
                calls=[(_i32(lens), _i32(new), sum(new) + case["pad"]), (_i32(lens2), _i32(new2), sum(new2) + case["pad"])])


def _prompt_inputs(case, g):
    lens, hkv, D, dt = _ints(case["lens"]), case["hkv"], case["D"], TYPES[case["dtype"]]
    starts, hq = _starts(lens), hkv * case["group"]
    T = max(1, starts[-1] + case["pad"])
    if case["fused"]:  # rows of one projection's output
        qkv = _normal(g, (T, hq + 2 * hkv, D), dt)
        q, kn, vn = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    else:
        q, kn, vn = _normal(g, (T, hq, D), dt), _normal(g, (T, hkv, D), dt), _normal(g, (T, hkv, D), dt)
    q.mul_(1.5)
    s = dict(q=q, kn=kn, vn=vn, starts=_i32(starts), out=torch.zeros(T, hq, D, dtype=dt, device=DEV),
             lse=torch.zeros(T, hq, dtype=torch.float32, device=DEV))
    if case["store"]:
        s.update(_cache(case, g, lens, False))
        s["slots"] = torch.full((T,), -1, dtype=torch.int64, device=DEV)
        s["lens"] = _i32([0] * len(lens))  # nothing cached yet
        if starts[-1]:
            b = torch.repeat_interleave(torch.arange(len(lens), device=DEV), torch.tensor(lens, device=DEV))
            i = torch.arange(starts[-1], device=DEV) - s["starts"].long()[b]
            s["slots"][:starts[-1]] = s["table"].long()[b, i // case["page"]] * case["page"] + i % case["page"]
    return s


def _parents(case, g, nodes):
    """Random trees: each drafted token hangs on one drafted before it, on a recent one more often than not."""
    parts = []
    for n in nodes:
        back = torch.rand(n, generator=g, device=DEV).pow(2) * torch.arange(n, device=DEV)
        parts.append(torch.arange(n, device=DEV) - 1 - back.long())
    return torch.cat(parts).clamp(min=-1).to(torch.int32)


def _tree_inputs(case, g):
    lens, nodes, hkv, D, dt = _ints(case["lens"]), _ints(case["nodes"]), case["hkv"], case["D"], TYPES[case["dtype"]]
    s = _cache(case, g, [n + m for n, m in zip(lens, nodes)], True)
    starts, hq = _starts(nodes), hkv * case["group"]
    T = max(1, starts[-1] + case["pad"])
    parents = torch.full((T,), -1, dtype=torch.int32, device=DEV)
    parents[:starts[-1]] = _parents(case, g, nodes)
    s.update(q=_normal(g, (T, hq, D), dt, 1.5), kn=_normal(g, (T, hkv, D), dt), vn=_normal(g, (T, hkv, D), dt), lens=_i32(lens),
             starts=_i32(starts), parents=None if case["chain"] else parents, out=torch.zeros(T, hq, D, dtype=dt, device=DEV),
             lse=torch.zeros(T, hq, dtype=torch.float32, device=DEV))
    return s


def _commit_inputs(case, g):
    lens, nodes = _ints(case["lens"]), _ints(case["nodes"])
    s = _cache(case, g, [n + m for n, m in zip(lens, nodes)], True)
    most, B = case["most"], len(lens)
    n = _i32(nodes)
    # some of each tree's nodes, in their order: those whose random keys are the smallest, as many as were accepted
    accepted = torch.minimum((torch.rand(B, generator=g, device=DEV) * (most + 1)).to(torch.int32), n)
    keys = torch.rand(B, NODES, generator=g, device=DEV).masked_fill(torch.arange(NODES, device=DEV) >= n[:, None], 2.0)
    taken = keys.argsort(-1).argsort(-1) < accepted[:, None]
    path = torch.where(taken, torch.arange(NODES, device=DEV), NODES).sort(-1).values[:, :most]
    s.update(lens=_i32(lens), nodes=n, path=path.to(torch.int32).contiguous(), accepted=accepted)
    s["positions"] = torch.arange(s["cap"], device=DEV, dtype=torch.int32).repeat(B, case["hkv"], 1)
    return s


def _inputs(case, seed):
    return dict(pages=_pages_inputs, prompt=_prompt_inputs, tree=_tree_inputs, commit=_commit_inputs)[case["kind"]](case, _gen(seed))


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own:
        from paper_2607_12422_gb300 import pbd
        s["pbd"] = pbd
        # the handles and the scratch, which a serving loop keeps
        if case["kind"] == "pages":
            s["pool"] = pbd.PagePool(s["table"], case["page"], s["n_pages"], held=s["held"], free=s["free"], n_free=s["n_free"])
            need = pbd.assign_pages_workspace_bytes(s["B"])
        elif case["kind"] == "prompt":
            s["kv"] = pbd.PagedKV(s["k"], s["v"], s["table"], s["lens"]) if case["store"] else None
            need = pbd.prompt_attention_workspace_bytes(s["q"].shape[0], len(_ints(case["lens"])), case["hkv"] * case["group"],
                                                        case["hkv"], case["D"])
        elif case["kind"] == "tree":
            s["kv"] = pbd.PagedKV(s["k"], s["v"], s["table"], s["lens"])
            need = pbd.tree_attention_workspace_bytes(s["kv"], s["q"].shape[0], case["hkv"] * case["group"])
        else:
            s["kv"] = pbd.PagedKV(s["k"], s["v"], s["table"], s["lens"], positions=s["positions"])
            need = pbd.commit_path_workspace_bytes(s["kv"], case["most"])
        s["ws"] = pbd.op_workspace(need, DEV)
    return s


# ------------------------------------------------------------------ one pass

def _own(s):
    case, pbd = s["case"], s["pbd"]
    if case["kind"] == "pages":
        got = [pbd.pbd_op_assign_pages(s["pool"], lens, new, most, workspace=s["ws"], sync=False) for lens, new, most in s["calls"]]
        return _pages_outputs(s, [(a.starts, a.slots, a.positions) for a in got])
    if case["kind"] == "prompt":
        pbd.pbd_op_prompt_attention(s["q"], s["kn"], s["vn"], s["starts"], kv=s["kv"], slots=s["slots"] if case["store"] else None,
                                    out=s["out"], lse=s["lse"], workspace=s["ws"], sync=False)
    elif case["kind"] == "tree":
        pbd.pbd_op_tree_attention(s["q"], s["kv"], s["kn"], s["vn"], s["starts"], parents=s["parents"], out=s["out"], lse=s["lse"],
                                  workspace=s["ws"], sync=False)
    else:
        pbd.pbd_op_commit_path(s["kv"], s["path"], s["accepted"], workspace=s["ws"], sync=False)
    return _outputs(s)


def _pages_outputs(s, packed):
    return dict(table=s["table"], held=s["held"], free=s["free"], n_free=s["n_free"], packed=packed)


def _outputs(s):
    return {n: s[n] for n in ("out", "lse", "k", "v", "positions") if n in s}


def _plain_assign(s, lens, new, most):
    ps, per = s["case"]["page"], s["table"].shape[1]
    lens, new, held, n_free = lens.long(), new.long(), s["held"].long(), s["n_free"].long()
    need = (lens + new + ps - 1) // ps
    i = torch.arange(per, device=DEV)[None]
    give, take = (i >= need[:, None]) & (i < held[:, None]), (i >= held[:, None]) & (i < need[:, None])
    # the stack with what is given back on top
    nth = give.flatten().cumsum(0).view_as(give)
    after = n_free + nth[-1, -1] - take.sum()
    place = torch.where(give, n_free + nth - 1, s["n_pages"])
    stack = torch.cat([s["free"], s["free"].new_zeros(1)]).scatter(0, place.flatten(), s["table"].flatten())
    top = n_free + nth[-1, -1] - take.flatten().cumsum(0).view_as(take)
    s["table"].copy_(torch.where(take, stack[torch.where(take, top, 0)], s["table"]))
    s["free"].copy_(torch.where(torch.arange(s["n_pages"], device=DEV) < after, stack[:-1], s["free"]))
    s["held"].copy_(need)
    s["n_free"].copy_(after)
    starts = torch.cat([new.new_zeros(1), new.cumsum(0)])
    t = torch.arange(most, device=DEV)
    b = torch.searchsorted(starts[1:].contiguous(), t, right=True).clamp(max=s["B"] - 1)
    pos, live = lens[b] + t - starts[b], t < starts[-1]
    slots = s["table"].long()[b, torch.where(live, pos // ps, 0)] * ps + pos % ps
    return (starts.to(torch.int32), torch.where(live, slots, -1), torch.where(live, pos, 0).to(torch.int32))


def _plain_pages(s):
    (lens, new, most), (lens2, new2, most2) = s["calls"]
    first = _plain_assign(s, lens, new, most)
    return _pages_outputs(s, [first, _plain_assign(s, lens2, new2, most2)])


def _softmax_av(sc, seen, vd):
    """Outputs and log sums of masked scores [B, KV heads, group, rows, keys] (written over)."""
    sc.masked_fill_(~seen, -math.inf)
    m = sc.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = sc.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), vd).view(*p.shape[:-1], vd.shape[-1])
    return o / torch.where(total == 0, torch.ones_like(total), total), (m + torch.log(total))[..., 0]


def _padded(rows, most):
    """[B, most] row numbers of packed rows (of a neighbour where a sequence has fewer), and which are its own."""
    i = torch.arange(most, device=DEV)[None]
    starts = rows["starts"].long()
    at = (starts[:-1, None] + i).clamp(max=rows["q"].shape[0] - 1)
    return at, i < (starts[1:] - starts[:-1])[:, None]


def _unpack(s, counts):
    """For each packed row its sequence and its place there."""
    b = torch.repeat_interleave(torch.arange(len(counts), device=DEV), s["starts"].long().diff(), output_size=sum(counts))
    return b, torch.arange(sum(counts), device=DEV) - s["starts"].long()[b]


def _plain_prompt(s):
    case, lens = s["case"], _ints(s["case"]["lens"])
    hkv, grp, D, ps, total, most = case["hkv"], case["group"], case["D"], case["page"], sum(lens), max(1, max(lens))
    if case["store"]:
        slots = s["slots"][:total]
        for_k = (slots // ps, slice(None), slots % ps)
        s["k"][for_k], s["v"][for_k] = s["kn"][:total], s["vn"][:total]
    at, own_rows = _padded(s, most)
    B = at.shape[0]
    q = s["q"][at].view(B, most, hkv, grp, D).permute(0, 2, 3, 1, 4).reshape(B, hkv, grp * most, D).float()
    kd, vd = (s[n][at].permute(0, 2, 1, 3).float() for n in ("kn", "vn"))
    sc = torch.matmul(q, kd.transpose(-1, -2)).mul_(1.0 / math.sqrt(D)).view(B, hkv, grp, most, most)
    i = torch.arange(most, device=DEV)
    seen = (i[None, :] <= i[:, None])[None, None, None] & own_rows[:, None, None, None, :]
    o, lse = _softmax_av(sc, seen, vd)
    b, j = _unpack(s, lens)
    s["out"][:total] = o.permute(0, 3, 1, 2, 4)[b, j].reshape(total, hkv * grp, D).to(s["out"].dtype)
    s["lse"][:total] = lse.permute(0, 3, 1, 2)[b, j].reshape(total, hkv * grp)
    return _outputs(s)


def _places(s):
    """Page, head and offset of every slot [B, hkv, cap] of the cache."""
    ps, hkv = s["case"]["page"], s["case"]["hkv"]
    slot = torch.arange(s["cap"], device=DEV)
    page = s["table"].long()[:, slot // ps][:, None].expand(-1, hkv, -1)
    head = torch.arange(hkv, device=DEV)[None, :, None].expand_as(page)
    return page, head, (slot % ps).expand_as(page)


def _plain_tree(s):
    case, nodes = s["case"], _ints(s["case"]["nodes"])
    hkv, grp, D, ps, total, N = case["hkv"], case["group"], case["D"], case["page"], sum(nodes), max(1, max(nodes))
    b, j = _unpack(s, nodes)
    lens = s["lens"].long()
    slot = lens[b] + j
    to = (s["table"].long()[b, slot // ps], slice(None), slot % ps)
    s["k"][to], s["v"][to] = s["kn"][:total], s["vn"][:total]
    at, _ = _padded(s, N)
    B = at.shape[0]
    # who is whose ancestor: paths of any length over the parents' edges
    i = torch.arange(N, device=DEV)
    up = i - 1 if case["chain"] else s["parents"].long()[at]
    edge = (up.expand(B, N)[:, :, None] == i[None, None, :]).float() + torch.eye(N, device=DEV)
    sees = torch.linalg.matrix_power(edge, N) > 0
    place = _places(s)
    kd, vd = s["k"][place].float(), s["v"][place].float()  # [B, hkv, cap, D]
    q = s["q"][at].view(B, N, hkv, grp, D).permute(0, 2, 3, 1, 4).reshape(B, hkv, grp * N, D).float()
    sc = torch.matmul(q, kd.transpose(-1, -2)).mul_(1.0 / math.sqrt(D)).view(B, hkv, grp, N, s["cap"])
    node = torch.arange(s["cap"], device=DEV)[None] - lens[:, None]
    drafted = torch.gather(sees, 2, node.clamp(0, N - 1)[:, None].expand(B, N, s["cap"])) & (node < N)[:, None]
    o, lse = _softmax_av(sc, ((node < 0)[:, None] | drafted)[:, None, None], vd)
    s["out"][:total] = o.permute(0, 3, 1, 2, 4)[b, j].reshape(total, hkv * grp, D).to(s["out"].dtype)
    s["lse"][:total] = lse.permute(0, 3, 1, 2)[b, j].reshape(total, hkv * grp)
    return _outputs(s)


def _plain_commit(s):
    ps, hkv, lens, (B, most) = s["case"]["page"], s["case"]["hkv"], s["lens"].long(), s["path"].shape
    i = torch.arange(most, device=DEV)[None]
    live = i < s["accepted"][:, None]
    # (what lies behind the path is written back over itself: the rows that follow, as far as the tree goes)
    last = (lens + s["nodes"] - 1).clamp(min=0)[:, None]
    to = torch.minimum(lens[:, None] + i, last)
    of = torch.where(live, lens[:, None] + s["path"].long(), to)
    rows, heads = torch.arange(B, device=DEV)[:, None], torch.arange(hkv, device=DEV)[None, :, None]
    page_of, page_to = (s["table"].long()[rows, x // ps][:, None].expand(B, hkv, most) for x in (of, to))
    for x in (s["k"], s["v"]):
        x[page_to, heads, (to % ps)[:, None]] = x[page_of, heads, (of % ps)[:, None]]
    of, to = (x[:, None].expand(B, hkv, most) for x in (of, to))
    s["positions"].scatter_(2, to, s["positions"].gather(2, of))
    return _outputs(s)


def run(state):
    if own:
        return _own(state)
    return dict(pages=_plain_pages, prompt=_plain_prompt, tree=_plain_tree, commit=_plain_commit)[state["case"]["kind"]](state)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["kind"] == "pages":
        B, ps = len(_ints(case["lens"])), case["page"]
        pages = [[-(-(n + m) // ps) for n, m in zip(_ints(case["lens" + x]), _ints(case["new" + x]))] for x in ("", "2")]
        b, before = 0, pages[1]  # (pass after pass, the second call's state is the first's)
        for x, now in (("", pages[0]), ("2", pages[1])):
            b += 4 * (5 * B + 3) + 12 * (sum(_ints(case["new" + x])) + case["pad"])
            b += 8 * sum(abs(n - m) for n, m in zip(now, before)) + 4 * sum(-(-m // ps) for m in _ints(case["new" + x]))
            before = now
        return dict(bytes=b, flops=0)
    hkv, D = case["hkv"], case["D"]
    row = 2 * 2 * D * hkv  # K and V of one slot
    if case["kind"] == "commit":
        moved = sum(min(n, case["most"]) for n in _ints(case["nodes"])) // 2  # half of what could be accepted, on average
        return dict(bytes=moved * 2 * (row + 4 * hkv) + 4 * moved + 8 * len(_ints(case["lens"])), flops=0)
    hq, lens = hkv * case["group"], _ints(case["lens"])
    if case["kind"] == "prompt":
        T = sum(lens)
        return dict(bytes=T * (4 * hq * D + row * (2 if case["store"] else 1) + 4 * hq + (8 if case["store"] else 0)) + 4 * len(lens),
                    flops=sum(2 * D * hq * n * (n + 1) for n in lens))
    nodes = _ints(case["nodes"])
    T = sum(nodes)
    read = sum(n for n, m in zip(lens, nodes) if m)
    return dict(bytes=read * row + T * (4 * hq * D + 2 * row + 4 * hq + 4) + 4 * sum(-(-n // case["page"]) for n in lens) + 12 * len(lens),
                flops=4 * D * hq * (sum(n * m for n, m in zip(lens, nodes)) + 4 * T))


# ------------------------------------------------------------------ the same in 64 bits

def _exact_rows(q, k, v, seen, scale):
    """One sequence: q [n, hkv, grp, D], k and v [m, hkv, D], seen(i0, i1) the rows' mask [i1 - i0, m]; [n, hq, D] and [n, hq]."""
    n, hkv, grp, D = q.shape
    outs, lses = [], []
    k, v = k.double().permute(1, 2, 0), v.double().transpose(0, 1)
    step = max(1, (1 << 27) // max(1, hkv * grp * k.shape[-1]))
    for i in range(0, n, step):
        e = min(n, i + step)
        sc = torch.matmul(q[i:e].double().permute(1, 2, 0, 3).reshape(hkv, -1, D), k).view(hkv, grp, e - i, -1) * scale
        sc = torch.where(seen(i, e), sc, -math.inf)
        lse = torch.logsumexp(sc, -1)
        o = torch.matmul(torch.exp(sc - lse[..., None]).view(hkv, grp * (e - i), -1), v).view(hkv, grp, e - i, D)
        outs.append(o.permute(2, 0, 1, 3).reshape(e - i, hkv * grp, D))
        lses.append(lse.permute(2, 0, 1).reshape(e - i, hkv * grp))
    return torch.cat(outs), torch.cat(lses)


def _exact_prompt(case, s):
    out, lse = s["out"].double(), s["lse"].double()
    ps, starts = case["page"], s["starts"].tolist()
    for b, n in enumerate(_ints(case["lens"])):
        if n == 0:
            continue
        at = slice(starts[b], starts[b] + n)
        q = s["q"][at].view(n, case["hkv"], case["group"], case["D"])
        j = torch.arange(n, device=DEV)
        out[at], lse[at] = _exact_rows(q, s["kn"][at], s["vn"][at], lambda i, e: j[None, :] <= j[i:e, None], case["D"] ** -0.5)
        if case["store"]:
            for x, new in ((s["k"], s["kn"]), (s["v"], s["vn"])):
                x[s["table"][b].long()[j // ps], :, j % ps] = new[at]
    return dict(_outputs(s), out=out, lse=lse)


def _exact_tree(case, s):
    out, lse = s["out"].double(), s["lse"].double()
    ps, starts = case["page"], s["starts"].tolist()
    parents = None if case["chain"] else s["parents"].tolist()
    for b, (n, m) in enumerate(zip(_ints(case["lens"]), _ints(case["nodes"]))):
        if m == 0:
            continue
        at = slice(starts[b], starts[b] + m)
        sees = [[False] * m for _ in range(m)]
        for i in range(m):
            j = i
            while j >= 0:
                sees[i][j] = True
                j = j - 1 if parents is None else parents[starts[b] + j]
        slot = torch.arange(n + m, device=DEV)
        where = (s["table"][b].long()[slot // ps], slice(None), slot % ps)
        for x, new in ((s["k"], s["kn"]), (s["v"], s["vn"])):
            x[where[0][n:], :, where[2][n:]] = new[at]
        mask = torch.cat([torch.ones(m, n, dtype=torch.bool, device=DEV), torch.tensor(sees, device=DEV)], 1)
        q = s["q"][at].view(m, case["hkv"], case["group"], case["D"])
        out[at], lse[at] = _exact_rows(q, s["k"][where], s["v"][where], lambda i, e: mask[i:e], case["D"] ** -0.5)
    return dict(_outputs(s), out=out, lse=lse)


def _exact_commit(case, s):
    ps, k, v = case["page"], s["k"].clone(), s["v"].clone()
    pos, table, path = s["positions"].clone(), s["table"].tolist(), s["path"].tolist()
    for b, (n, took) in enumerate(zip(_ints(case["lens"]), s["accepted"].tolist())):
        of, to = [n + path[b][i] for i in range(took)], list(range(n, n + took))
        src, dst = ([[table[b][x // ps], x % ps] for x in slots] for slots in (of, to))
        if took:
            src, dst = torch.tensor(src, device=DEV).T, torch.tensor(dst, device=DEV).T
            k[dst[0], :, dst[1]], v[dst[0], :, dst[1]] = s["k"][src[0], :, src[1]], s["v"][src[0], :, src[1]]
            pos[b, :, n:n + took] = s["positions"][b][:, torch.tensor(of, device=DEV)]
    return dict(k=k, v=v, positions=pos)


def exact(case, seed):
    if case["kind"] == "pages":
        return None  # whole numbers
    s = _inputs(case, seed)
    return dict(prompt=_exact_prompt, tree=_exact_tree, commit=_exact_commit)[case["kind"]](case, s)
