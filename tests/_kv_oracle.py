"""The cache operators and token log probabilities in 64 bits, sequence by sequence, on the CPU; and the inputs of their
tests."""
import math

import numpy as np


def make_cache(torch, lens, hkv, D, page, dtype, layout="heads", extra=1, poison=True, seed=0):
    """A cache whose pages lie in random order, with NaN in every slot that no sequence holds (and in nobody's pages)
    when poisoned; table entries that no sequence uses lie outside the cache.  `extra`: slots a sequence can grow by."""
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    used = [(n + extra + page - 1) // page for n in lens]
    per = max(max(used), 1)
    n_pages = sum(used) + 2
    perm = torch.randperm(n_pages, generator=g)
    table = torch.full((B, per), 1 << 30, dtype=torch.int32)
    at = 0
    for b in range(B):
        table[b, :used[b]] = perm[at:at + used[b]].int()
        at += used[b]
    shape = (n_pages, hkv, page, D) if layout == "heads" else (n_pages, page, hkv, D)
    k, v = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
    if layout != "heads":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    if poison:
        held = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(n):
                held[int(table[b, j // page]), j % page] = True
        for x in (k, v):
            x[~held[:, None, :].expand(n_pages, hkv, page)] = math.nan
    weights = torch.rand(B, hkv, per * page, generator=g).pow(4)
    positions = torch.arange(per * page, dtype=torch.int32).repeat(B, hkv, 1)
    return dict(k=k, v=v, table=table, lens=torch.tensor(lens, dtype=torch.int32), weights=weights, positions=positions,
                page=page, cap=per * page)


def rows_of(c, x, b, n):
    """x's slots [0, n) of sequence b: [hkv, n, D] float64."""
    idx = [(int(c["table"][b, j // c["page"]]), j % c["page"]) for j in range(n)]
    if not idx:
        return x[:1, :, :0].double()[0]
    p, o = (np.array(z) for z in zip(*idx))
    return x[p, :, o].double().transpose(0, 1)


def attention(torch, c, q, k_new=None, v_new=None, scale=None):
    """Per sequence (out [hq, D], lse [hq], p [hq, n], and what the bounds of the comparison need): sum p |v| and the largest
    scale * sum |q k|."""
    B, hq, D = q.shape
    hkv = c["k"].shape[1]
    res = []
    for b in range(B):
        n = int(c["lens"][b])
        k, v = rows_of(c, c["k"], b, n), rows_of(c, c["v"], b, n)
        if k_new is not None:
            k, v = torch.cat([k, k_new[b].double()[:, None]], 1), torch.cat([v, v_new[b].double()[:, None]], 1)
        k, v = (x.repeat_interleave(hq // hkv, 0) for x in (k, v))
        qq = q[b].double()
        if k.shape[1] == 0:
            z = torch.zeros(hq, D, dtype=torch.float64)
            res.append(dict(out=z, lse=torch.full((hq,), -math.inf, dtype=torch.float64), p=z[:, :0], pv=z, mag=z[:, 0]))
            continue
        s = torch.einsum("hd,hnd->hn", qq, k) * (scale or D ** -0.5)
        lse = torch.logsumexp(s, -1)
        p = torch.exp(s - lse[:, None])
        mag = torch.einsum("hd,hnd->hn", qq.abs(), k.abs()).amax(-1) * (scale or D ** -0.5)
        res.append(dict(out=torch.einsum("hn,hnd->hd", p, v), lse=lse, p=p, pv=torch.einsum("hn,hnd->hd", p, v.abs()), mag=mag))
    return res


def evict_row(w, pos, n, n_keep, next_pos, n_recent, n_sink):
    """(slots whose contents slots [0, keep) hold afterwards) of one sequence and head, by sorting."""
    keep = min(n, n_keep)

    def order(j):
        safe = pos[j] < n_sink or pos[j] >= next_pos - n_recent
        return (0 if safe else 1, 1 if math.isnan(w[j]) and not safe else 0, 0 if safe or math.isnan(w[j]) else -w[j], j)

    kept = set(sorted(range(n), key=order)[:keep])
    src = list(range(keep))
    tails = [j for j in range(keep, n) if j in kept]
    for hole, tail in zip([j for j in range(keep) if j not in kept], tails):
        src[hole] = tail
    return src


def logprobs(torch, x, tokens, k, T):
    """(logprob, entropy, ids, top) of rows x (any type) in 64 bits; ids by value, equal ones by the lower id."""
    z = x.double() / T
    m = z.amax(-1, keepdim=True)
    empty = (m == -math.inf)[:, 0]
    z = z - torch.where(m == -math.inf, torch.zeros_like(m), m)  # (a sum of a type's lowest value and ln S would be off)
    e = torch.exp(z)
    lp = torch.where(empty[:, None], torch.full_like(z, -math.inf), z - torch.log(e.sum(-1, keepdim=True)))
    ent = torch.where(e > 0, -lp.exp() * lp, torch.zeros_like(z)).sum(-1)
    ent = torch.where(empty, torch.zeros_like(ent), ent)
    ids = torch.from_numpy(np.argsort(-x.double().numpy(), axis=-1, kind="stable")[:, :k].copy())
    t = tokens.long()
    chosen = torch.where(t < 0, torch.zeros_like(ent), lp.gather(-1, t.clamp(min=0)[:, None])[:, 0])
    return chosen, ent, ids, lp.gather(-1, ids)
