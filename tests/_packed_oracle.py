"""The operators on packed rows in 64 bits and plain Python, sequence by sequence, on the CPU; and the inputs of their tests."""
import math

import _kv_oracle as kvref

HALF = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
DT = {"bf16": "bfloat16", "fp16": "float16"}


def starts_of(torch, counts):
    return torch.tensor([0] + list(counts)).cumsum(0).to(torch.int32)


def rows(torch, T, hq, hkv, D, dt, fused, counts=None, seed=1):
    """q, k, v [T, heads, D]; with `fused` parts of one buffer's rows.  Rows behind the sequences hold NaN."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, hq + 2 * hkv, D, generator=g)
    x[:, :hq] *= 1.5
    x = x.to(dt)
    if counts is not None:
        x[sum(counts):] = math.nan
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    return (q, k, v) if fused else (q.contiguous(), k.contiguous(), v.contiguous())


def fused_to_gpu(torch, q, k, v):
    """The same three on the GPU, parts of one buffer if they are here."""
    if q.is_contiguous() and k.is_contiguous():
        return q.cuda(), k.cuda(), v.cuda()
    hq, hkv = q.shape[1], k.shape[1]
    x = torch.cat([q, k, v], 1).cuda()
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def attend(torch, q, k, v, sees, scale=None):
    """q [n, hq, D], k and v [m, hkv, D], sees [n, m]: out, lse and what the bounds of the comparison need.  What a row does not
    see takes no part, whatever it holds."""
    n, hq, D = q.shape
    grp = hq // k.shape[1]
    scale = scale or D ** -0.5
    q, k, v = q.double(), k.double().repeat_interleave(grp, 1), v.double().repeat_interleave(grp, 1)
    s = torch.einsum("ihd,jhd->hij", q, k) * scale
    s = torch.where(sees, s, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.where(sees, torch.exp(s - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[..., None]), 0.0)
    clean = torch.nan_to_num(v, 0.0, 0.0, 0.0)
    out, pv = torch.einsum("hij,jhd->ihd", p, clean), torch.einsum("hij,jhd->ihd", p, clean.abs())
    # a value that is not finite reaches the rows that see it, in its dimension
    odd = torch.einsum("ij,jhd->ihd", sees.double(), (~torch.isfinite(v)).double()) > 0
    mag = torch.einsum("ihd,jhd->hij", q.abs(), k.abs())
    mag = torch.where(sees, mag, 0.0).amax(-1).T * scale if k.shape[0] else torch.zeros(n, hq, dtype=torch.float64)
    return dict(out=out, odd=odd, lse=lse.T, pv=pv, mag=mag, seen=sees.sum(-1), vmax=float(clean.abs().max()) if clean.numel() else 0.0)


def check(torch, want, out, lse, kind):
    """Errors that the call may have, u being half a step of the type.  Scores: D products summed in fp32, each of at most D
    partial sums off by 2^-23 of their magnitude, so exponents are off by e = 2 D 2^-23 mag at most (the factor to base 2 and
    its product included), and p, whose sum carries the same error, by 2 e.  p's rounding: u; in fp16 p is held with a factor
    of 2^6 at least below the largest, and off by 2^-25 of a step of that where it is smallest, so by 2^-31 of the largest.  exp2:
    2^-22.  Sums over n keys: at most n / 2 + 32 additions in a row, 2^-23 each and for numerator and denominator.  Then the
    output's own rounding; fp16 has a smallest step of 2^-24."""
    D, u = out.shape[-1], HALF[kind]
    n = want["seen"].double()[:, None]
    e = 2 * D * 2.0 ** -23 * want["mag"]
    sums = (n / 2 + 32) * 2.0 ** -23
    rel = 2 * e + u + 2.0 ** -21 + 2 * sums
    tol = want["out"].abs() * u + want["pv"] * rel[..., None] * (1 + u) + 2.0 ** -25
    if kind == "fp16":
        tol = tol + (n * 2.0 ** -31 * want["vmax"])[..., None]
    got = out.cpu().double()
    assert torch.equal(want["odd"], ~torch.isfinite(got)), "values that are not finite in other places"
    err = torch.where(want["odd"], torch.zeros_like(got), (got - want["out"]).abs())
    assert (err <= tol).all(), (float((err / tol).max()), float(err.max()))
    if lse is not None:
        tol = e + sums + 2.0 ** -21 + want["lse"].abs() * 2.0 ** -22
        got = lse.cpu().double()
        err = (got - want["lse"]).abs()
        assert ((got == want["lse"]) | (err <= tol)).all(), float((err / tol).nan_to_num().max())


def causal(torch, n):
    i = torch.arange(n)
    return i[None, :] <= i[:, None]


def trees(torch, counts, seed=3):
    """Random parents, node by node before it, deep and wide ones."""
    g = torch.Generator().manual_seed(seed)
    parts = []
    for n in counts:
        i = torch.arange(n)
        back = (torch.rand(n, generator=g) ** 2 * i).long()
        parts.append((i - 1 - back).clamp(min=-1))
    return torch.cat(parts + [torch.zeros(0, dtype=torch.long)]).to(torch.int32)


def ancestors(torch, parents):
    """[n, n]: whether node i descends from node j or is it."""
    n = len(parents)
    sees = torch.eye(n, dtype=torch.bool)
    for i, p in enumerate(parents):
        if p >= 0:
            sees[i] |= sees[p]
    return sees


def tree_case(torch, lens, nodes, hkv, D, page, dt, layout, seed=0):
    """A cache with room for the nodes; what no sequence holds yet is NaN."""
    c = kvref.make_cache(torch, lens, hkv, D, page, dt, layout, extra=0, seed=seed)
    room = kvref.make_cache(torch, [n + m for n, m in zip(lens, nodes)], hkv, D, page, dt, layout, extra=0, seed=seed)
    # (the larger cache, with the slots of the nodes emptied)
    for b, (n, m) in enumerate(zip(lens, nodes)):
        for j in range(n, n + m):
            p, o = int(room["table"][b, j // page]), j % page
            room["k"][p, :, o], room["v"][p, :, o] = math.nan, math.nan
    room["lens"] = c["lens"]
    return room


def tree_attention(torch, c, b, q, kn, vn, parents, scale=None):
    """One sequence: its nodes' rows q, kn, vn; parents of them (None: a chain)."""
    n, m = int(c["lens"][b]), q.shape[0]
    sees = causal(torch, m) if parents is None else ancestors(torch, parents.tolist())
    k, v = (torch.cat([kvref.rows_of(c, c[x], b, n).transpose(0, 1) if n else new[:0].double(), new.double()]) for x, new in (("k", kn), ("v", vn)))
    return attend(torch, q, k, v, torch.cat([torch.ones(m, n, dtype=torch.bool), sees], 1), scale)


def assign(table, held, free, lens, n_new, page):
    """The pool after a call: table rows, held, the free stack; and the slots and positions of the packed rows."""
    need = [-(-(n + m) // page) for n, m in zip(lens, n_new)]
    for b, row in enumerate(table):
        free.extend(row[need[b]:held[b]])
    for b, row in enumerate(table):
        for i in range(held[b], need[b]):
            row[i] = free.pop()
        held[b] = need[b]
    at = [(b, n + i) for b, (n, m) in enumerate(zip(lens, n_new)) for i in range(m)]
    return [table[b][x // page] * page + x % page for b, x in at], [x for _, x in at]
