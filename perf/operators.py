"""Timed and compared cases of the single-token serving operators: attention of one new token over a
paged key-value cache, eviction from such a cache by accumulated attention weight, and log
probabilities of given tokens with entropy and top alternatives.

Sizes are those of the package's own shapes and workloads (16 query over 8 KV heads of 128, pages of
16 tokens, a vocabulary of 151936, verify blocks of 17 rows, its batch of eight ragged prompts) and
of generic neighbours: other groups, head sizes, page lengths, odd lengths and vocabularies.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BATCH8 = "1757,725,451,791,997,1715,1065,420"


# ------------------------------------------------------------------ the cases

def listed():
    ragged = ",".join(str(n) for n in (
        0, 1, 15, 16, 17, 33, 64, 100, 127, 128, 129, 200, 255, 257, 300, 391, 450, 511, 512, 513, 640, 777, 800, 901,
        1000, 1023, 1024, 1025, 1100, 1200, 1300, 1377, 1500, 1600, 1733, 1800, 1999, 2047, 2048, 2049, 2200, 2300, 2500,
        2700, 2900, 3001, 3300, 3500, 3777, 4000, 4095, 4096, 4097, 4500, 4800, 5000, 5333, 5600, 6000, 6400, 6661, 7000,
        7500, 8000))
    return [
        # one layer's attention of the next token behind a 512-token prompt: the smallest call, latency counts
        dict(name="attn-512", kind="attn", lens="512", hkv=8, group=2, D=128, page=16, dtype="bf16", layout="heads",
             append=True, accumulate=False),
        # the batch of eight ragged sequences, the weights kept for a later eviction
        dict(name="attn-batch8-weights", kind="attn", lens=BATCH8, hkv=8, group=2, D=128, page=16, dtype="bf16",
             layout="heads", append=True, accumulate=True),
        # one sequence with a very long context: work split over its length and joined
        dict(name="attn-131071-weights", kind="attn", lens="131071", hkv=8, group=2, D=128, page=16, dtype="bf16",
             layout="heads", append=True, accumulate=True),
        # a serving batch from empty to long, seven query heads a KV head, token-major pages
        dict(name="attn-64-ragged", kind="attn", lens=ragged, hkv=4, group=7, D=64, page=32, dtype="fp16",
             layout="tokens", append=False, accumulate=False),
        # a step of a bounded cache: the token that came over the budget goes
        dict(name="evict-step", kind="evict", lens=",".join(["1025"] * 8), keep=1024, recent=256, sink=4, hkv=8, D=128,
             page=16, dtype="bf16", layout="heads", ordered=False),
        # after long prompts: an eighth of the tokens stays
        dict(name="evict-prompts", kind="evict", lens="32768,30001,17,32767", keep=4096, recent=512, sink=4, hkv=8, D=128,
             page=16, dtype="bf16", layout="heads", ordered=True),
        # ragged lengths around the budget, half precision, token-major pages
        dict(name="evict-ragged", kind="evict", lens=",".join(str(500 + 173 * i) for i in range(32)), keep=1500,
             recent=100, sink=0, hkv=4, D=64, page=32, dtype="fp16", layout="tokens", ordered=False),
        # a decoded token's log probability and alternatives: the smallest read-out
        dict(name="logprobs-1", kind="logp", M=1, V=151936, dtype="fp32", k=20, T=1.0),
        # the rows of one verify block
        dict(name="logprobs-17", kind="logp", M=17, V=151936, dtype="fp32", k=5, T=1.0),
        # the rows of eight verify blocks, logits kept in 16 bits (ties), sampled at a temperature
        dict(name="logprobs-136-bf16", kind="logp", M=136, V=151936, dtype="bf16", k=20, T=0.7),
        # scoring of a whole text: the largest read-out
        dict(name="logprobs-2048", kind="logp", M=2048, V=151936, dtype="fp32", k=8, T=1.0),
        # an odd vocabulary, whose rows start at odd addresses, no alternatives asked for
        dict(name="logprobs-odd-fp16", kind="logp", M=333, V=32003, dtype="fp16", k=0, T=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "evict", "logp"])
    if kind == "logp":
        V = rng.choice([_log(rng, 100, 160000), _log(rng, 20000, 160000), 151936])
        return dict(kind=kind, M=_log(rng, 1, min(4096, 300_000_000 // V)), V=V, dtype=rng.choice(["fp32", "bf16", "fp16"]),
                    k=rng.choice([0, 1, 5, 20, 32]), T=rng.choice([1.0, 0.7, 1.3]))
    D = rng.choice([64, 128, 128, 256])
    hkv = rng.choice([1, 2, 4, 8, 8])
    common = dict(kind=kind, hkv=hkv, D=D, page=rng.choice([8, 16, 16, 32, 64]), dtype=rng.choice(["bf16", "fp16"]),
                  layout=rng.choice(["heads", "tokens"]))
    B = _log(rng, 1, 48)
    most = min(100_000, 130_000_000 // (B * hkv * D))
    top = _log(rng, 40, most)
    if kind == "attn":
        lens = [_log(rng, max(1, top // 8), top) if rng.random() < 0.95 else 0 for _ in range(B)]
        return dict(common, lens=",".join(map(str, lens)), group=rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16]),
                    append=rng.random() < 0.7, accumulate=rng.random() < 0.5)
    lens = [_log(rng, max(1, top // 8), top) for _ in range(B)]
    keep = max(8, int(top * rng.uniform(0.05, 0.95)))
    recent = int(keep * rng.choice([0, 0.1, 0.5]))
    return dict(common, lens=",".join(map(str, lens)), keep=keep, recent=recent, sink=rng.choice([0, 4]),
                ordered=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 1000003 + 11)


def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dtype)


def _cache(case, g):
    """Pages in random order, some of them nobody's; the table's entries behind a sequence's last page are valid ones."""
    lens, ps, hkv, D = _lens(case), case["page"], case["hkv"], case["D"]
    B = len(lens)
    per = (max(lens) + 1 + ps - 1) // ps
    used = [(n + 1 + ps - 1) // ps for n in lens]
    n_pages = sum(used) + 3
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    first = torch.tensor([sum(used[:b]) for b in range(B)], device=DEV)
    last = torch.tensor(used, device=DEV) - 1
    table = perm[(first[:, None] + torch.minimum(torch.arange(per, device=DEV)[None], last[:, None]))]
    shape = (n_pages, hkv, ps, D) if case["layout"] == "heads" else (n_pages, ps, hkv, D)
    k, v = (_normal(g, shape, TYPES[case["dtype"]]) for _ in range(2))
    if case["layout"] == "tokens":
        k, v = k.transpose(1, 2), v.transpose(1, 2)  # [page, head, slot, D] by strides
    return dict(k=k, v=v, table=table.contiguous(), lens=torch.tensor(lens, dtype=torch.int32, device=DEV), cap=per * ps)


def _inputs(case, seed):
    g = _gen(seed)
    if case["kind"] == "logp":
        # a few tokens stand out of a wide field, as a language model's logits do
        x = torch.randn(case["M"], case["V"], generator=g, device=DEV, dtype=torch.float32)
        x = (x * 2.0 + 0.1 * x.abs() ** 3).to(TYPES[case["dtype"]])
        tokens = torch.randint(0, case["V"], (case["M"],), generator=g, device=DEV, dtype=torch.int32)
        return dict(x=x, tokens=tokens)
    s = _cache(case, g)
    B, hkv, D, cap = len(_lens(case)), case["hkv"], case["D"], s["cap"]
    dt = TYPES[case["dtype"]]
    # what earlier tokens paid to each slot: few slots hold most of it
    s["weights"] = torch.rand(B, hkv, cap, generator=g, device=DEV).pow(6) * 3.0
    if case["kind"] == "attn":
        s["q"] = _normal(g, (B, hkv * case["group"], D), dt)
        s["k_new"], s["v_new"] = (_normal(g, (B, hkv, D), dt) if case["append"] else None for _ in range(2))
        s["next"] = s["lens"] + 100  # a hundred tokens have been evicted before
        s["positions"] = torch.arange(cap, device=DEV, dtype=torch.int32).repeat(B, hkv, 1)
        return s
    # slots in the order of their tokens, or in any order, as earlier evictions leave them
    order = torch.arange(cap, device=DEV).expand(B, hkv, cap)
    if not case["ordered"]:
        keys = torch.rand(B, hkv, cap, generator=g, device=DEV)
        keys = torch.where(torch.arange(cap, device=DEV) < s["lens"][:, None, None], keys, 2.0)
        order = keys.argsort(-1).argsort(-1)
    # (after the first four, fifty tokens have been evicted before)
    s["positions"] = torch.where(order < 4, order, order + 50).to(torch.int32)
    s["next"] = s["lens"] + 50
    s["new_weights"], s["new_positions"] = torch.zeros_like(s["weights"]), torch.zeros_like(s["positions"])
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own:
        from paper_2607_12422_gb300 import pbd
        s["pbd"] = pbd
        if case["kind"] == "logp":
            s["ws"] = pbd.op_workspace(pbd.token_logprobs_workspace_bytes(case["M"], case["V"], case["k"]), DEV)
        else:
            # the handle of a cache and the scratch, which a serving loop keeps
            kv = s["kv"] = pbd.PagedKV(s["k"], s["v"], s["table"], s["lens"], weights=s["weights"], positions=s["positions"])
            if case["kind"] == "attn":
                need = pbd.decode_attention_workspace_bytes(kv, case["hkv"] * case["group"], case["accumulate"])
            else:
                need = pbd.evict_workspace_bytes(kv, case["keep"])
            s["ws"] = pbd.op_workspace(need, DEV)
    return s


# ------------------------------------------------------------------ one pass

def _own(s):
    case, pbd = s["case"], s["pbd"]
    if case["kind"] == "logp":
        r = pbd.pbd_op_token_logprobs(s["x"], s["tokens"], k=case["k"], temperature=case["T"], workspace=s["ws"], sync=False)
        return dict(logprob=r.logprob, entropy=r.entropy, top_ids=r.top_ids, top_logprobs=r.top_logprobs)
    if case["kind"] == "attn":
        out, lse = pbd.pbd_op_decode_attention(s["q"], s["kv"], s["k_new"], s["v_new"],
                                               s["next"] if case["append"] else None, accumulate=case["accumulate"],
                                               want_lse=True, workspace=s["ws"], sync=False)
        return _attn_outputs(s, out, lse)
    pbd.pbd_op_evict(s["kv"], case["keep"], n_recent=case["recent"], n_sink=case["sink"], next_positions=s["next"],
                     out_weights=s["new_weights"], out_positions=s["new_positions"], workspace=s["ws"], sync=False)
    return _evict_outputs(s)


def _attn_outputs(s, out, lse):
    r = dict(out=out, lse=lse)
    if s["case"]["append"]:
        r.update(k=s["k"], v=s["v"], positions=s["positions"])
    if s["case"]["accumulate"]:
        r["weights"] = s["weights"]
    return r


def _evict_outputs(s):
    return dict(k=s["k"], v=s["v"], weights=s["new_weights"], positions=s["new_positions"])


def _places(s):
    """Page, head and offset of every slot [B, hkv, cap] of the cache."""
    ps, hkv = s["case"]["page"], s["case"]["hkv"]
    slot = torch.arange(s["cap"], device=DEV)
    page = s["table"].long()[:, slot // ps][:, None].expand(-1, hkv, -1)
    head = torch.arange(hkv, device=DEV)[None, :, None].expand_as(page)
    return page, head, (slot % ps).expand_as(page)


def _plain_attn(s):
    case = s["case"]
    lens, k, v = s["lens"].long(), s["k"], s["v"]
    B, hkv, grp, D, ps = lens.numel(), case["hkv"], case["group"], case["D"], case["page"]
    n = lens
    if case["append"]:
        b, h = torch.arange(B, device=DEV), torch.arange(hkv, device=DEV)
        page = s["table"].long()[b, lens // ps]
        at = (page[:, None].expand(B, hkv), h[None].expand(B, hkv), (lens % ps)[:, None].expand(B, hkv))
        k[at], v[at] = s["k_new"], s["v_new"]
        s["positions"][b[:, None], h[None], lens[:, None]] = s["next"][:, None].expand(B, hkv)
        n = lens + 1
    place = _places(s)
    kd, vd = k[place].float(), v[place].float()  # [B, hkv, cap, D]
    q = s["q"].view(B, hkv, grp, D).float()
    seen = (torch.arange(s["cap"], device=DEV) < n[:, None])[:, None, None]
    sc = (torch.matmul(q, kd.transpose(-1, -2)) * (1.0 / math.sqrt(D))).masked_fill(~seen, -math.inf)
    m = sc.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(sc - m)
    total = p.sum(-1, keepdim=True)
    lse = (m + torch.log(total)).reshape(B, hkv * grp)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    out = torch.matmul(p, vd).reshape(B, hkv * grp, D).to(s["q"].dtype)
    if case["accumulate"]:
        w = s["weights"]
        if case["append"]:  # the new token's slot starts from nothing
            w.masked_fill_((torch.arange(s["cap"], device=DEV) == lens[:, None])[:, None], 0.0)
        w += p.sum(2)
    return _attn_outputs(s, out, lse)


def _plain_evict(s):
    case, cap = s["case"], s["cap"]
    w, pos, lens = s["weights"], s["positions"], s["lens"].long()
    slot = torch.arange(cap, device=DEV)
    kept_n = lens.clamp(max=case["keep"])[:, None, None]
    safe = (pos < case["sink"]) | (pos >= (s["next"] - case["recent"])[:, None, None])
    rank = torch.where(safe, math.inf, w).masked_fill(slot >= lens[:, None, None], -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(safe).scatter_(-1, order, (slot < kept_n).expand_as(order))
    hole, tail = (slot < kept_n) & ~kept, (slot >= kept_n) & kept
    # the i-th hole in front takes the i-th kept slot behind
    nth = (tail.cumsum(-1) - 1).masked_fill(~tail, cap)
    tails = torch.zeros(*w.shape[:2], cap + 1, dtype=torch.long, device=DEV).scatter_(-1, nth, slot.expand_as(nth))
    src = torch.where(hole, tails.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), slot)
    front = (slot < kept_n).expand_as(src)
    s["new_weights"].copy_(torch.where(front, w.gather(-1, src), s["new_weights"]))
    s["new_positions"].copy_(torch.where(front, pos.gather(-1, src), s["new_positions"]))
    page, head, off = _places(s)
    top = min(cap, case["keep"])
    to = (page[..., :top], head[..., :top], off[..., :top])
    of = (page.gather(-1, src)[..., :top], head[..., :top], off.gather(-1, src)[..., :top])
    # (a table's entries behind the last page name that page again: what is not in front is written back unread)
    live = front[..., :top, None]
    for x in (s["k"], s["v"]):
        x.index_put_(to, torch.where(live, x[of], x[to]))
    return _evict_outputs(s)


def _plain_logp(s):
    case = s["case"]
    x = s["x"].float() / case["T"]
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    logprob = ((x.gather(-1, s["tokens"].long()[:, None]) - m) - torch.log(total))[:, 0]
    entropy = torch.log(total)[:, 0] + (e * (m - x)).sum(-1) / total[:, 0]
    r = dict(logprob=logprob, entropy=entropy, top_ids=None, top_logprobs=None)
    if case["k"]:
        ids = s["x"].sort(dim=-1, descending=True, stable=True).indices[:, : case["k"]].contiguous()
        r.update(top_ids=ids.to(torch.int32), top_logprobs=x.gather(-1, ids) - lse)
    return r


def run(state):
    if own:
        return _own(state)
    return dict(attn=_plain_attn, evict=_plain_evict, logp=_plain_logp)[state["case"]["kind"]](state)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["kind"] == "logp":
        M, V, k = case["M"], case["V"], case["k"]
        return dict(bytes=M * V * (4 if case["dtype"] == "fp32" else 2) + M * (12 + 8 * k), flops=4 * M * V)
    lens, hkv, D, ps = _lens(case), case["hkv"], case["D"], case["page"]
    row = 2 * 2 * D  # K and V of one slot and head
    if case["kind"] == "attn":
        new = 1 if case["append"] else 0
        n, B, hq = sum(lens) + new * len(lens), len(lens), hkv * case["group"]
        b = sum(lens) * hkv * row + 2 * B * hq * 2 * D + 4 * B * hq + 4 * sum(-(-x // ps) for x in lens) + 4 * B
        b += new * B * hkv * (2 * row + 4)
        b += 8 * n * hkv if case["accumulate"] else 0
        return dict(bytes=b, flops=4 * n * hq * D)
    b = 0
    for n in lens:
        keep = min(n, case["keep"])
        b += hkv * 8 * ((n if n > keep else 0) + keep)  # weights and positions in and out
        if n > keep:  # rows that are kept and lie behind the budget, if no slot is likelier kept than another
            last = min(case["recent"], n - keep) if case["ordered"] else 0
            free = case["recent"] + case["sink"] if case["ordered"] else 0
            b += hkv * 2 * row * (last + (keep - free) * (n - keep - last) / max(1, n - free))
    return dict(bytes=int(b), flops=sum(lens) * hkv)


# ------------------------------------------------------------------ the same in 64 bits

def _exact_attn(case, s):
    lens, grp, ps = _lens(case), case["group"], case["page"]
    k, v, w, pos = (s[n].clone() for n in ("k", "v", "weights", "positions"))
    w = w.double()
    outs, lses = [], []
    for b, n in enumerate(lens):
        pages = s["table"][b].tolist()
        if case["append"]:
            p, o = pages[n // ps], n % ps
            k[p, :, o], v[p, :, o] = s["k_new"][b], s["v_new"][b]
            pos[b, :, n], w[b, :, n] = s["next"][b], 0.0
            n += 1
        if n == 0:
            outs.append(torch.zeros(case["hkv"] * grp, case["D"], dtype=torch.float64, device=DEV))
            lses.append(torch.full((case["hkv"] * grp,), -math.inf, dtype=torch.float64, device=DEV))
            continue
        at = torch.tensor(pages[: -(-n // ps)], device=DEV)
        kb, vb = (x[at].transpose(0, 1).reshape(case["hkv"], -1, case["D"])[:, :n].double() for x in (k, v))
        q = s["q"][b].view(case["hkv"], grp, case["D"]).double()
        sc = torch.einsum("hgd,hnd->hgn", q, kb) / math.sqrt(case["D"])
        lse = torch.logsumexp(sc, -1)
        prob = torch.exp(sc - lse[..., None])
        outs.append(torch.einsum("hgn,hnd->hgd", prob, vb).reshape(-1, case["D"]))
        lses.append(lse.reshape(-1))
        w[b, :, :n] += prob.sum(1)
    r = dict(out=torch.stack(outs), lse=torch.stack(lses))
    if case["append"]:
        r.update(k=k, v=v, positions=pos)
    if case["accumulate"]:
        r["weights"] = w
    return r


def _exact_evict(case, s):
    ps = case["page"]
    k, v, neww, newp = (s[n].clone() for n in ("k", "v", "new_weights", "new_positions"))
    W, P, table, nxt = s["weights"].cpu().tolist(), s["positions"].cpu().tolist(), s["table"].tolist(), s["next"].tolist()
    for b, n in enumerate(_lens(case)):
        keep = min(n, case["keep"])
        for h in range(case["hkv"]):
            w, p = W[b][h], P[b][h]
            free = [j for j in range(n) if not (p[j] < case["sink"] or p[j] >= nxt[b] - case["recent"])]
            out = set(sorted(free, key=lambda j: (w[j], -j))[: n - keep])
            holes = [j for j in range(keep) if j in out]
            tails = [j for j in range(keep, n) if j not in out]
            src = list(range(keep))
            for i, j in zip(holes, tails):
                src[i] = j
            at = torch.tensor(src, device=DEV, dtype=torch.long)
            neww[b, h, :keep], newp[b, h, :keep] = s["weights"][b, h][at], s["positions"][b, h][at]
            to, of = ([(table[b][j // ps], j % ps) for j in js] for js in (holes, tails))
            if to:
                to, of = torch.tensor(to, device=DEV), torch.tensor(of, device=DEV)
                k[to[:, 0], h, to[:, 1]], v[to[:, 0], h, to[:, 1]] = k[of[:, 0], h, of[:, 1]], v[of[:, 0], h, of[:, 1]]
    return dict(k=k, v=v, weights=neww, positions=newp)


def _exact_logp(case, s):
    rows = max(1, (1 << 25) // case["V"])
    parts = []
    for i in range(0, case["M"], rows):
        x = s["x"][i:i + rows].double() / case["T"]
        lp = x - torch.logsumexp(x, -1, keepdim=True)
        parts.append((lp.gather(-1, s["tokens"][i:i + rows].long()[:, None])[:, 0], -(lp.exp() * lp).sum(-1),
                      lp.topk(case["k"]).values if case["k"] else None))
    return dict(logprob=torch.cat([p[0] for p in parts]), entropy=torch.cat([p[1] for p in parts]), top_ids=None,
                top_logprobs=torch.cat([p[2] for p in parts]) if case["k"] else None)


def exact(case, seed):
    s = _inputs(case, seed)
    return dict(attn=_exact_attn, evict=_exact_evict, logp=_exact_logp)[case["kind"]](case, s)
