"""Attention of one new token over a paged cache and eviction from it, against the same in 64 bits."""
import ctypes as C
import math

import pytest

import _kv_oracle as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_12422_gb300 import pbd
    pbd.load()
    return torch, pbd


DT = {"bf16": "bfloat16", "fp16": "float16"}


def _to_gpu(torch, c):
    def move(x):
        y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
        return y.copy_(x)
    return {n: move(c[n]) for n in ("k", "v", "table", "lens", "weights", "positions")}


def _handle(pbd, g, **kw):
    return pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"], **kw)


def _check_attention(torch, want, out, lse, n, half_step):
    """Errors that the call may have.  Scores: D products summed in fp32, each of at most D partial sums off by 2^-23 of
    their magnitude, so exponents are off by e = 2 D 2^-23 mag at most (the factor to base 2 and its product included), and
    p, whose sum carries the same error, by 2 e.  P's two 16-bit halves: 2^-16.  exp2: 2^-22.  Sums over n slots: a step per 16
    slots and some more for the joins, 2^-23 each and for numerator and denominator.  Then the output's own rounding; fp16
    has a smallest step of 2^-24."""
    D = out.shape[-1]
    e = 2 * D * 2.0 ** -23 * want["mag"]
    sums = (n / 16 + 32) * 2.0 ** -23
    rel = 2 * e + 2.0 ** -16 + 2.0 ** -21 + 2 * sums
    tol = want["out"].abs() * half_step + want["pv"] * rel[:, None] * (1 + half_step) + 2.0 ** -25
    err = (out.cpu().double() - want["out"]).abs()
    assert (err <= tol).all(), (float((err / tol).max()), float(err.max()))
    if lse is not None:
        tol = e + sums + 2.0 ** -21 + want["lse"].abs() * 2.0 ** -22
        err = (lse.cpu().double() - want["lse"]).abs()
        assert ((lse.cpu().double() == want["lse"]) | (err <= tol)).all(), float((err / tol).nan_to_num().max())
    return rel


HALF = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}

SHAPES = [
    # lens, hkv, group, D, page, layout
    ([1], 1, 1, 64, 16, "heads"),
    ([5], 8, 2, 128, 16, "heads"),
    ([512], 8, 2, 128, 16, "heads"),
    ([0, 1, 15, 16, 17, 31, 33, 100], 2, 3, 128, 16, "heads"),
    ([700, 0, 0, 3, 1300], 2, 8, 64, 16, "tokens"),
    ([257, 90], 2, 7, 64, 24, "tokens"),
    ([129, 64, 1], 1, 16, 128, 8, "heads"),
    ([200, 31], 2, 9, 256, 32, "heads"),
    ([77, 300], 1, 40, 128, 64, "tokens"),
    ([45], 1, 33, 256, 1, "heads"),
    ([2500], 1, 4, 256, 16, "tokens"),
    ([20000], 1, 2, 128, 16, "heads"),
    ([37] * 150, 2, 2, 64, 16, "heads"),
    ([0, 1, 17, 300, 64] * 70, 1, 2, 64, 16, "heads"),  # more rows than CTAs run at once
    ([33, 0, 5, 150] * 26, 4, 5, 128, 16, "tokens"),
    ([200, 1, 90] * 60, 1, 12, 256, 16, "heads"),
    ([30000, 10, 500, 0], 2, 7, 64, 16, "tokens"),      # too long for clusters
    ([26000, 4000], 1, 3, 256, 32, "heads"),
]


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%dx%s-%s" % (len(s[0]), max(s[0]), "-".join(map(str, s[1:]))))
def test_attention_matches_64_bits(env, shape, dtype, append):
    """Every slot that no sequence holds is NaN, and table entries behind a sequence lie outside the cache."""
    torch, pbd = env
    lens, hkv, group, D, page, layout = shape
    dt = getattr(torch, DT[dtype])
    c = ref.make_cache(torch, lens, hkv, D, page, dt, layout, extra=1 if append else 0)
    gen = torch.Generator().manual_seed(7)
    B = len(lens)
    q = (torch.randn(B, hkv * group, D, generator=gen) * 1.5).to(dt)
    kn, vn = ((torch.randn(B, hkv, D, generator=gen)).to(dt) if append else None for _ in range(2))
    g = _to_gpu(torch, c)
    kv = _handle(pbd, g, weights=g["weights"], positions=g["positions"])
    pos = (torch.arange(B, dtype=torch.int32) + 100000).cuda() if append else None
    want = ref.attention(torch, c, q, kn, vn)
    args = (q.cuda(), kv, kn.cuda() if append else None, vn.cuda() if append else None, pos)
    out, lse = pbd.pbd_op_decode_attention(*args, want_lse=True)
    assert torch.equal(g["weights"].cpu(), c["weights"])  # without accumulate nothing is written there
    out2, lse2 = pbd.pbd_op_decode_attention(*args, accumulate=True, want_lse=True)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)  # the same bits on every call
    for b in range(B):
        n = lens[b] + append
        rel = _check_attention(torch, want[b], out[b], lse[b], n, HALF[dtype])
        got = g["weights"][b].cpu().double()
        w = c["weights"][b].double().clone()
        if append:
            w[:, lens[b]] = 0
        p = want[b]["p"].view(hkv, group, -1)
        w[:, :n] += p.sum(1)
        # one rounding of the sum, and of up to `group` terms
        tol = w * (group + 1) * 2.0 ** -23 + 1e-30
        tol[:, :n] += (p * rel.view(hkv, group, 1)).sum(1)
        assert ((got - w).abs() <= tol).all(), float(((got - w).abs() / tol).max())
        # the cache: the new row in its slot, everything else as it was
        for x, y, new in ((g["k"], c["k"], kn), (g["v"], c["v"], vn)):
            if append:
                p_, o_ = int(c["table"][b, lens[b] // page]), lens[b] % page
                y[p_, :, o_] = new[b]
    for x, y in ((g["k"], c["k"]), (g["v"], c["v"])):
        assert torch.equal(x.cpu().contiguous().view(torch.int16), y.contiguous().view(torch.int16))
    if append:
        want_pos = c["positions"].clone()
        want_pos[torch.arange(B), :, c["lens"].long()] = pos.cpu()[:, None]
        assert torch.equal(g["positions"].cpu(), want_pos)


def test_attention_of_large_scores_and_equal_keys(env):
    """Scores of several hundred (a softmax without the running maximum overflows), and a softmax over n equal keys, which
    is the mean of the values."""
    torch, pbd = env
    c = ref.make_cache(torch, [300, 300], 2, 128, 16, torch.bfloat16, poison=False)
    c["k"] *= 20
    q = torch.randn(2, 4, 128).bfloat16() * 4
    q[1] = 0
    g = _to_gpu(torch, c)
    out, lse = pbd.pbd_op_decode_attention(q.cuda(), _handle(pbd, g), want_lse=True)
    for b, want in enumerate(ref.attention(torch, c, q)):
        _check_attention(torch, want, out[b], lse[b], 300, HALF["bf16"])
    assert (lse[1].cpu() - math.log(300)).abs().max() < 1e-5


def test_attention_far_below_the_maximum_in_half_precision(env):
    """20000 keys a factor 2^-22 below one: together half a percent, which weights rounded to fp16's 2^-24 would lose."""
    torch, pbd = env
    c = ref.make_cache(torch, [20000], 1, 64, 16, torch.float16, poison=False)
    c["k"].zero_()
    p, o = int(c["table"][0, 0]), 3
    c["k"][p, 0, o, 0] = 22 * math.log(2) * 8
    c["v"][:] = 1.0
    c["v"][p, 0, o] = 0.0
    q = torch.zeros(1, 1, 64, dtype=torch.float16)
    q[0, 0, 0] = 1.0
    g = _to_gpu(torch, c)
    out, lse = pbd.pbd_op_decode_attention(q.cuda(), _handle(pbd, g), want_lse=True)
    want = ref.attention(torch, c, q)[0]
    assert 0.003 < float(want["out"].min()) < 0.006
    _check_attention(torch, want, out[0], lse[0], 20000, HALF["fp16"])


def test_attention_takes_rows_of_a_fused_projection(env):
    """q, k_new and v_new as slices of one [batch, (hq + 2 hkv) D] buffer, the output in the caller's tensor."""
    torch, pbd = env
    hq, hkv, D, lens = 6, 2, 64, [40, 9]
    c = ref.make_cache(torch, lens, hkv, D, 16, torch.bfloat16)
    qkv = torch.randn(2, (hq + 2 * hkv) * D).bfloat16()
    cut = [x.view(2, -1, D) for x in qkv.split([hq * D, hkv * D, hkv * D], 1)]
    dev = [x.view(2, -1, D) for x in qkv.cuda().split([hq * D, hkv * D, hkv * D], 1)]
    g = _to_gpu(torch, c)
    out = torch.empty(2, hq, D, dtype=torch.bfloat16, device="cuda")
    got, lse = pbd.pbd_op_decode_attention(dev[0], _handle(pbd, g), dev[1], dev[2], scale=0.2, out=out)
    assert got is out and lse is None
    for b, want in enumerate(ref.attention(torch, c, *cut, scale=0.2)):
        _check_attention(torch, want, out[b], None, lens[b] + 1, HALF["bf16"])


def test_offsets_beyond_32_bits(env):
    """Pages that lie more than 2^32 values apart: the attention reads and the eviction moves the right ones."""
    torch, pbd = env
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB of free device memory")
    stride = (1 << 32) + 64
    D, page, n = 64, 16, 40
    k, v = (torch.empty(2 * stride + page * D, dtype=torch.bfloat16, device="cuda").as_strided(
        (3, 1, page, D), (stride, page * D, D, 1)) for _ in range(2))
    small = ref.make_cache(torch, [n], 1, D, page, torch.bfloat16, extra=0, poison=False)
    perm = torch.tensor([[2, 0, 1]], dtype=torch.int32)
    small["table"] = perm
    small["k"], small["v"] = small["k"][:3], small["v"][:3]
    k.copy_(small["k"])
    v.copy_(small["v"])
    q = torch.randn(1, 2, D).bfloat16()
    w, pos = small["weights"].cuda(), small["positions"].cuda()
    kv = pbd.PagedKV(k, v, perm.cuda(), small["lens"].cuda(), weights=w, positions=pos)
    out, lse = pbd.pbd_op_decode_attention(q.cuda(), kv, want_lse=True)
    _check_attention(torch, ref.attention(torch, small, q)[0], out[0], lse[0], n, HALF["bf16"])
    pbd.pbd_op_evict(kv, 10, torch.tensor([n], dtype=torch.int32, device="cuda"))
    src = ref.evict_row(small["weights"][0, 0].tolist(), small["positions"][0, 0].tolist(), n, 10, n, 0, 0)
    want = ref.rows_of(small, small["k"], 0, n)[:, src]
    small["k"], small["v"] = k.cpu(), v.cpu()
    assert torch.equal(ref.rows_of(small, small["k"], 0, 10), want)


EVICT = [
    # lens, n_keep, n_recent, n_sink, hkv, D, page, layout
    ([17], 16, 4, 2, 8, 128, 16, "heads"),
    ([1, 0, 16, 17, 40], 16, 0, 0, 2, 64, 16, "heads"),
    ([100, 300, 299, 64], 64, 32, 32, 2, 64, 24, "tokens"),
    ([1000, 50], 1, 1, 0, 1, 256, 8, "heads"),
    ([1000, 50], 0, 0, 0, 1, 64, 8, "heads"),
    ([5000, 4097], 4096, 512, 4, 2, 64, 16, "heads"),
    ([3000], 100, 10, 4, 1, 128, 16, "tokens"),
    ([9000, 20011], 2500, 0, 4, 1, 64, 32, "heads"),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["random", "few", "special"])
@pytest.mark.parametrize("shape", EVICT, ids=lambda s: "%dx%d-%s" % (len(s[0]), max(s[0]), "-".join(map(str, s[1:]))))
def test_evict_matches_sorting(env, shape, kind, in_place):
    """Weights all different, of few values (ties go to the lower slot), and with NaN, infinities, zeros of both signs and
    negative ones among them.  Slots hold tokens in any order."""
    torch, pbd = env
    lens, n_keep, n_recent, n_sink, hkv, D, page, layout = shape
    c = ref.make_cache(torch, lens, hkv, D, page, torch.bfloat16 if D != 64 else torch.float16, layout, extra=0)
    gen = torch.Generator().manual_seed(3)
    w = c["weights"]
    if kind == "few":
        w.copy_(torch.randint(0, 4, w.shape, generator=gen).float())
    elif kind == "special":
        table = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-42, -1.0, 3.0])
        w.copy_(table[torch.randint(0, 8, w.shape, generator=gen)])
    for b, n in enumerate(lens):
        for h in range(hkv):
            c["positions"][b, h, :n] = torch.randperm(n, generator=gen).int()
            c["positions"][b, h, n:] = 0  # (a slot behind the sequence, though its position says "sink")
    g = _to_gpu(torch, c)
    kv = _handle(pbd, g, weights=g["weights"], positions=g["positions"])
    new_w, new_p = torch.full_like(g["weights"], 7.0), torch.full_like(g["positions"], 7)
    nxt = c["lens"].cuda()
    outs = {} if in_place else dict(out_weights=new_w, out_positions=new_p)
    got_w, got_p = pbd.pbd_op_evict(kv, n_keep, nxt, n_recent=n_recent, n_sink=n_sink, **outs)
    if in_place:
        assert got_w is g["weights"] and got_p is g["positions"]
    want_w = c["weights"].clone() if in_place else torch.full_like(c["weights"], 7.0)
    want_p = c["positions"].clone() if in_place else torch.full_like(c["positions"], 7)
    want_k, want_v = c["k"].clone(), c["v"].clone()
    for b, n in enumerate(lens):
        keep = min(n, n_keep)
        for h in range(hkv):
            src = ref.evict_row(c["weights"][b, h].tolist(), c["positions"][b, h].tolist(), n, n_keep, n, n_recent, n_sink)
            want_w[b, h, :keep], want_p[b, h, :keep] = c["weights"][b, h][src], c["positions"][b, h][src]
            for i, j in enumerate(src):
                if i != j:
                    a, d = (int(c["table"][b, z // page]) for z in (i, j))
                    want_k[a, h, i % page] = c["k"][d, h, j % page]
                    want_v[a, h, i % page] = c["v"][d, h, j % page]
    assert torch.equal(got_p.cpu(), want_p)
    assert torch.equal(got_w.cpu().view(torch.int32), want_w.view(torch.int32))
    for x, y in ((g["k"], want_k), (g["v"], want_v)):
        assert torch.equal(x.cpu().contiguous().view(torch.int16), y.contiguous().view(torch.int16))
    if not in_place:  # the cache's own arrays are as they were
        assert torch.equal(g["positions"].cpu(), c["positions"])


def test_evict_of_a_very_long_sequence(env):
    """More slots than the cluster's shared memory holds keys of."""
    torch, pbd = env
    n, keep, D = 450_000, 1000, 64
    gen = torch.Generator().manual_seed(5)
    k = torch.randn(n // 16 + 1, 1, 16, D, generator=gen).half().cuda()
    table = torch.randperm(n // 16 + 1, generator=gen).int()[None]
    w = torch.rand(1, 1, table.shape[1] * 16, generator=gen)
    pos = torch.arange(w.shape[2], dtype=torch.int32)[None, None].contiguous()
    v = k.clone()
    kv = pbd.PagedKV(k, v, table.cuda(), torch.tensor([n], dtype=torch.int32).cuda(), weights=w.cuda(), positions=pos.cuda())
    before = k.cpu()
    gw, gp = pbd.pbd_op_evict(kv, keep, torch.tensor([n], dtype=torch.int32).cuda(), n_recent=100, n_sink=4)
    src = ref.evict_row(w[0, 0].tolist(), range(n), n, keep, n, 100, 4)
    assert gp[0, 0, :keep].cpu().tolist() == src and torch.equal(gw[0, 0, :keep].cpu(), w[0, 0][src])
    page, off = table[0][torch.arange(keep) // 16].long(), torch.arange(keep) % 16
    spage, soff = table[0][torch.tensor(src) // 16].long(), torch.tensor(src) % 16
    for x in (k, v):
        assert torch.equal(x.cpu()[page, 0, off], before[spage, 0, soff])


def test_a_bounded_decode_loop(env):
    """Thirty steps of a bounded cache as a program runs them: attention appends the token and gathers weights, lengths
    grow, what is over the budget goes.  Against the same loop in 64 bits over lists of tokens; a step's eviction is
    checked only by the kept positions, which the weights separate by far more than their error."""
    torch, pbd = env
    B, hkv, group, D, page, budget = 2, 2, 2, 64, 16, 24
    lens = [20, 5]
    c = ref.make_cache(torch, lens, hkv, D, page, torch.bfloat16, extra=40)
    c["weights"].zero_()
    g = _to_gpu(torch, c)
    kv = _handle(pbd, g, weights=g["weights"], positions=g["positions"])
    ws = pbd.op_workspace(max(pbd.decode_attention_workspace_bytes(kv, hkv * group, True), pbd.evict_workspace_bytes(kv, budget)))
    seen = g["lens"].clone()
    gen = torch.Generator().manual_seed(11)
    held = [[[(j, ref.rows_of(c, c["k"], b, n)[h, j], ref.rows_of(c, c["v"], b, n)[h, j], 0.0) for j in range(n)]
             for h in range(hkv)] for b, n in enumerate(lens)]
    for step in range(30):
        q, kn, vn = (torch.randn(B, m, D, generator=gen).bfloat16() for m in (hkv * group, hkv, hkv))
        out, _ = pbd.pbd_op_decode_attention(q.cuda(), kv, kn.cuda(), vn.cuda(), seen, accumulate=True, workspace=ws, sync=False)
        kv.lens += 1
        seen += 1
        pbd.pbd_op_evict(kv, budget, seen, n_recent=6, n_sink=2, workspace=ws, sync=False)
        kv.lens.clamp_(max=budget)
        pbd.pbd_op_status(ws)
        for b in range(B):
            now = lens[b] + step + 1
            for h in range(hkv):
                row = held[b][h] + [(now - 1, kn[b, h].double(), vn[b, h].double(), 0.0)]
                kk, vv = torch.stack([r[1] for r in row]), torch.stack([r[2] for r in row])
                qq = q[b, h * group:(h + 1) * group].double()
                p = torch.softmax(qq @ kk.T / D ** 0.5, -1)
                got = out[b, h * group:(h + 1) * group].cpu().double()
                want = p @ vv
                assert ((got - want).abs() <= want.abs() * 2.0 ** -8 + (p @ vv.abs()) * 1e-4).all()
                row = [(r[0], r[1], r[2], r[3] + float(x)) for r, x in zip(row, p.sum(0))]
                n_now = int(kv.lens[b])
                slots = g["positions"][b, h, :n_now].tolist()
                if len(row) > budget:
                    ranked = sorted(row, key=lambda r: (r[0] < 2 or r[0] >= now - 6, r[3]), reverse=True)
                    assert ranked[budget - 1][3] - ranked[budget][3] > 1e-4 or ranked[budget - 1][0] >= now - 6
                    row = ranked[:budget]
                assert sorted(slots) == sorted(r[0] for r in row)
                held[b][h] = row


def test_graphs_streams_and_a_shared_workspace(env):
    """The calls captured into two graphs that share a workspace, replayed in turn on a side stream with other contents;
    and plain calls on another stream than the tensors' own."""
    torch, pbd = env
    c = ref.make_cache(torch, [100, 333], 2, 128, 16, torch.bfloat16, extra=0, poison=False)
    g = _to_gpu(torch, c)
    kv = _handle(pbd, g, weights=g["weights"], positions=g["positions"])
    q = torch.randn(2, 4, 128, device="cuda").bfloat16()
    logits = torch.randn(2, 5000, device="cuda")
    ws = pbd.op_workspace(max(pbd.decode_attention_workspace_bytes(kv, 4, True), pbd.token_logprobs_workspace_bytes(2, 5000, 4),
                              pbd.evict_workspace_bytes(kv, 64)))
    nw, npos = torch.zeros_like(g["weights"]), torch.zeros_like(g["positions"])
    nxt = g["lens"].clone()

    def first():
        return pbd.pbd_op_decode_attention(q, kv, workspace=ws, sync=False, want_lse=True)

    def second():
        return pbd.pbd_op_token_logprobs(logits, k=4, workspace=ws, sync=False)

    def third():
        return pbd.pbd_op_evict(kv, 64, nxt, 8, 2, nw, npos, workspace=ws, sync=False)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(side):
        for f in (first, second, third):
            f()
        side.synchronize()
        kv.k.copy_(c["k"])
        kv.v.copy_(c["v"])
        for f in (first, second, third):
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr, stream=side):
                outs.append(f())
            graphs.append(gr)
        for turn in range(3):
            q.copy_(torch.randn(2, 4, 128, generator=torch.Generator().manual_seed(turn)).bfloat16())
            logits.copy_(torch.randn(2, 5000, generator=torch.Generator().manual_seed(turn)))
            for gr in graphs[:2]:
                gr.replay()
            side.synchronize()
            for b, want in enumerate(ref.attention(torch, c, q.cpu())):
                _check_attention(torch, want, outs[0][0][b], outs[0][1][b], int(c["lens"][b]), HALF["bf16"])
            ids = ref.logprobs(torch, logits.cpu(), torch.zeros(2), 4, 1.0)[2]
            assert torch.equal(outs[1].top_ids.cpu().long(), ids)
        graphs[2].replay()
        side.synchronize()
        for b, n in enumerate(c["lens"].tolist()):
            src = ref.evict_row(c["weights"][b, 0].tolist(), c["positions"][b, 0].tolist(), n, 64, n, 8, 2)
            assert npos[b, 0, :64].cpu().tolist() == src
        pbd.pbd_op_status(ws)
    torch.cuda.current_stream().wait_stream(side)


@pytest.mark.parametrize("what", ["page", "negative page", "length", "negative length", "full"])
def test_bad_pages_and_lengths_are_reported(env, what):
    """What the host cannot see is read as nothing, and reported: kernels check it before they use it."""
    torch, pbd = env
    c = ref.make_cache(torch, [40, 40], 2, 64, 16, torch.bfloat16, extra=0, poison=False)
    if "page" in what:
        c["table"][1, 1] = -3 if "negative" in what else c["k"].shape[0]
    elif what != "full":
        c["lens"][1] = -1 if "negative" in what else c["cap"] + 1
    else:  # no slot left for the new token
        c["lens"][1] = c["cap"]
    g = _to_gpu(torch, c)
    kv = _handle(pbd, g, weights=g["weights"], positions=g["positions"])
    q, new = torch.randn(2, 4, 64, device="cuda").bfloat16(), torch.randn(2, 2, 64, device="cuda").bfloat16()
    args = (q, kv, new, new) if what == "full" else (q, kv)
    with pytest.raises(pbd.PbdError) as e:
        pbd.pbd_op_decode_attention(*args)
    assert e.value.status == 6 and ("page" in str(e.value) or "position" in str(e.value))
    # nothing was stored for the sequence
    page = int(c["table"][1, 2])
    assert torch.equal(g["k"].cpu()[page], c["k"][page]) and torch.equal(g["v"].cpu()[page], c["v"][page])
    if what == "full":
        pbd.pbd_op_decode_attention(q, kv)  # (a full sequence can be read)
        return
    # the other sequence's output is what it is
    out, _ = pbd.pbd_op_decode_attention(q, kv, workspace=pbd.op_workspace(1 << 25), sync=False)
    one = dict(c, table=c["table"][:1], lens=c["lens"][:1])
    _check_attention(torch, ref.attention(torch, one, q[:1].cpu())[0], out[0], None, 40, HALF["bf16"])
    g["weights"][1, :, 16:32] = 9  # slots of the bad page are kept and would move
    with pytest.raises(pbd.PbdError) as e:
        pbd.pbd_op_evict(kv, 20, g["lens"].clamp(0, 40))
    assert e.value.status == 6
    # the status word is the last call's own
    c["table"][1, 1], c["lens"][1] = 0, 40
    g["table"].copy_(c["table"])
    g["lens"].copy_(c["lens"])
    pbd.pbd_op_decode_attention(q, kv)


def test_two_devices_or_the_current_one(env):
    """A call for tensors of a device that is not the current one; with one GPU, of the current one by its index."""
    torch, pbd = env
    dev = torch.device("cuda", torch.cuda.device_count() - 1)
    c = ref.make_cache(torch, [50], 1, 64, 16, torch.bfloat16, extra=0)
    g = {n: x.to(dev) for n, x in _to_gpu(torch, c).items()}
    q = torch.randn(1, 1, 64).bfloat16()
    out, _ = pbd.pbd_op_decode_attention(q.to(dev), _handle(pbd, g))
    assert out.device == dev
    _check_attention(torch, ref.attention(torch, c, q)[0], out[0], None, 50, HALF["bf16"])


def test_refusals_of_the_binding(env):
    torch, pbd = env
    c = ref.make_cache(torch, [40, 40], 2, 64, 16, torch.bfloat16, poison=False)
    g = _to_gpu(torch, c)
    kv = _handle(pbd, g)
    q, new = torch.randn(2, 4, 64, device="cuda").bfloat16(), torch.randn(2, 2, 64, device="cuda").bfloat16()
    nxt = g["lens"]
    calls = [
        lambda: pbd.PagedKV(g["k"], g["v"][:-1], g["table"], g["lens"]),
        lambda: pbd.PagedKV(g["k"], g["v"].half(), g["table"], g["lens"]),
        lambda: pbd.PagedKV(g["k"].float(), g["v"].float(), g["table"], g["lens"]),
        lambda: pbd.PagedKV(g["k"], g["v"], g["table"].long(), g["lens"]),
        lambda: pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"][:1]),
        lambda: pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"].cpu()),
        lambda: pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"], weights=g["weights"][:, :1]),
        lambda: pbd.PagedKV(g["k"].transpose(2, 3), g["v"].transpose(2, 3), g["table"], g["lens"]),
        lambda: pbd.pbd_op_decode_attention(q[:1], kv),
        lambda: pbd.pbd_op_decode_attention(q[:, :3], kv),
        lambda: pbd.pbd_op_decode_attention(q.half(), kv),
        lambda: pbd.pbd_op_decode_attention(q, kv, new),
        lambda: pbd.pbd_op_decode_attention(q, kv, new, new[:, :1]),
        lambda: pbd.pbd_op_decode_attention(q, kv, None, None, nxt),
        lambda: pbd.pbd_op_decode_attention(q, kv, scale=0.0),
        lambda: pbd.pbd_op_decode_attention(q, kv, scale=math.inf),
        lambda: pbd.pbd_op_decode_attention(q, kv, accumulate=True),  # no weights
        lambda: pbd.pbd_op_decode_attention(q, kv, out=torch.empty(2, 4, 64, device="cuda")),
        lambda: pbd.pbd_op_decode_attention(q, kv, out=q),
        lambda: setattr(kv, "lens", g["lens"] + 1),
        lambda: pbd.pbd_op_decode_attention(q, kv, workspace=pbd.op_workspace(4096)),
        lambda: pbd.pbd_op_evict(kv, 8, nxt),
        lambda: pbd.pbd_op_evict(_handle(pbd, g, weights=g["weights"], positions=g["positions"]), 8, nxt, n_recent=6, n_sink=3),
        lambda: pbd.pbd_op_evict(_handle(pbd, g, weights=g["weights"], positions=g["positions"]), -1, nxt),
        lambda: pbd.pbd_op_evict(_handle(pbd, g, weights=g["weights"], positions=g["positions"]), 8, nxt.long()),
        lambda: pbd.op_workspace(0),
    ]
    before = g["k"].clone()
    for i, f in enumerate(calls):
        with pytest.raises(pbd.PbdError) as e:
            f()
        assert e.value.status in (1, 2), i
    torch.cuda.synchronize()
    assert torch.equal(before, g["k"])
