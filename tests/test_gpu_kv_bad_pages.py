"""Tables that name pages outside the cache: what is reported leaves the cache's slots as they were."""
import math

import pytest

import _kv_oracle as ref
from test_gpu_kv_ops import _handle, _to_gpu, env  # noqa: F401

pytestmark = pytest.mark.gpu


def _bits(x):
    import torch
    return x.cpu().contiguous().view({2: torch.int16, 4: torch.int32}[x.element_size()])


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lens,n_keep", [([100, 70], 40), ([5000, 300], 200)])  # a CTA a row; clusters and the moves' kernel
def test_evict_moves_nothing_from_or_to_a_bad_page(env, lens, n_keep, in_place):  # noqa: F811
    """Every other page of the first sequence is outside the cache, in front of the kept slots' end and behind it: rows,
    weights and positions move together or not at all.  The second sequence is evicted as ever."""
    torch, pbd = env
    hkv, D, page = 2, 64, 8
    c = ref.make_cache(torch, lens, hkv, D, page, torch.bfloat16, extra=0, poison=False, seed=4)
    gen = torch.Generator().manual_seed(9)
    for b, n in enumerate(lens):
        for h in range(hkv):
            c["positions"][b, h, :n] = torch.randperm(n, generator=gen).int()
    bad = torch.arange(c["table"].shape[1]) % 2 == 1
    table = c["table"].clone()
    table[0, bad] = torch.where(torch.arange(int(bad.sum())) % 4 < 2, torch.tensor(c["k"].shape[0]), torch.tensor(-1)).int()
    g = _to_gpu(torch, dict(c, table=table))
    kv = _handle(pbd, g, weights=g["weights"], positions=g["positions"])
    new_w, new_p = torch.full_like(g["weights"], 7.0), torch.full_like(g["positions"], 7)
    outs = {} if in_place else dict(out_weights=new_w, out_positions=new_p)
    with pytest.raises(pbd.PbdError) as e:
        pbd.pbd_op_evict(kv, n_keep, g["lens"].clone(), n_recent=5, n_sink=3, **outs)
    assert e.value.status == 6 and "page" in str(e.value)
    want_w, want_p = (c["weights"].clone(), c["positions"].clone()) if in_place else (new_w.cpu() * 0 + 7, new_p.cpu() * 0 + 7)
    want_k, want_v = c["k"].clone(), c["v"].clone()
    left_out = 0
    for b, n in enumerate(lens):
        for h in range(hkv):
            src = ref.evict_row(c["weights"][b, h].tolist(), c["positions"][b, h].tolist(), n, n_keep, n, 5, 3)
            for i, j in enumerate(src):
                if b == 0 and i != j and (bad[i // page] or bad[j // page]):
                    left_out += 1
                    j = i
                want_w[b, h, i], want_p[b, h, i] = c["weights"][b, h, j], c["positions"][b, h, j]
                if i != j:
                    a, d = (int(c["table"][b, z // page]) for z in (i, j))
                    want_k[a, h, i % page] = c["k"][d, h, j % page]
                    want_v[a, h, i % page] = c["v"][d, h, j % page]
    assert left_out > 0
    got_w, got_p = (g["weights"], g["positions"]) if in_place else (new_w, new_p)
    assert torch.equal(_bits(got_w), _bits(want_w)) and torch.equal(got_p.cpu(), want_p)
    assert torch.equal(_bits(g["k"]), _bits(want_k)) and torch.equal(_bits(g["v"]), _bits(want_v))


# (small calls; the list of tiles with rows joined by CTAs, by warps, and with chunks of a group)
WAYS = [([40, 70, 33, 50], 2, 2, 64, 16), ([20000, 70, 33, 4000], 1, 3, 128, 16), ([40, 70, 33, 50] * 40, 2, 4, 64, 8),
        ([77, 130, 41, 300], 1, 40, 128, 24)]


def _with_bad_pages(torch, shape, dtype, seed=1):
    """A cache whose sequences of each four have a bad page in their middle, for the new token's slot, everywhere and
    nowhere."""
    lens, hkv, group, D, page = shape
    c = ref.make_cache(torch, lens, hkv, D, page, dtype, extra=1, seed=seed)
    table = c["table"].clone()
    far = c["k"].shape[0]
    for b, n in enumerate(lens):
        if b % 4 == 0:
            table[b, n // page // 2] = far
        elif b % 4 == 1:
            table[b, n // page] = -5
        elif b % 4 == 2:
            table[b] = far + 7
    gen = torch.Generator().manual_seed(seed)
    B = len(lens)
    q = (torch.randn(B, hkv * group, D, generator=gen) * 1.5).to(dtype)
    kn, vn = (torch.randn(B, hkv, D, generator=gen).to(dtype) for _ in range(2))
    ok = [[0 <= int(table[b, j // page]) < far for j in range(n + 1)] for b, n in enumerate(lens)]
    return c, table, q, kn, vn, ok


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("shape", WAYS, ids=lambda s: "%dx%d-g%d" % (len(s[0]), max(s[0]), s[2]))
def test_a_new_token_without_a_page_leaves_its_position_alone(env, shape, dtype):  # noqa: F811
    torch, pbd = env
    lens, hkv, page = shape[0], shape[1], shape[4]
    c, table, q, kn, vn, ok = _with_bad_pages(torch, shape, getattr(torch, dtype))
    g = _to_gpu(torch, dict(c, table=table))
    kv = _handle(pbd, g, positions=g["positions"])
    pos = (torch.arange(len(lens), dtype=torch.int32) + 100000).cuda()
    with pytest.raises(pbd.PbdError) as e:
        pbd.pbd_op_decode_attention(q.cuda(), kv, kn.cuda(), vn.cuda(), pos)
    assert e.value.status == 6 and "page" in str(e.value)
    want = c["positions"].clone()
    for b, n in enumerate(lens):
        if ok[b][n]:
            want[b, :, n] = 100000 + b
            p, o = int(table[b, n // page]), n % page
            c["k"][p, :, o], c["v"][p, :, o] = kn[b], vn[b]
    assert torch.equal(g["positions"].cpu(), want)
    assert torch.equal(_bits(g["k"]), _bits(c["k"])) and torch.equal(_bits(g["v"]), _bits(c["v"]))


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("shape", WAYS, ids=lambda s: "%dx%d-g%d" % (len(s[0]), max(s[0]), s[2]))
def test_slots_of_bad_pages_take_no_part(env, shape, dtype, append):  # noqa: F811
    """A softmax over the slots whose pages exist; the weights of all others keep their bits."""
    from test_gpu_kv_ops import HALF, _check_attention
    torch, pbd = env
    lens, hkv, group, D, page = shape
    c, table, q, kn, vn, ok = _with_bad_pages(torch, shape, getattr(torch, dtype))
    g = _to_gpu(torch, dict(c, table=table))
    kv = _handle(pbd, g, weights=g["weights"], positions=g["positions"])
    new = (kn.cuda(), vn.cuda()) if append else ()
    with pytest.raises(pbd.PbdError) as e:
        pbd.pbd_op_decode_attention(q.cuda(), kv, *new, accumulate=True)
    assert e.value.status == 6 and "page" in str(e.value)
    g2 = _to_gpu(torch, dict(c, table=table))
    kv2 = _handle(pbd, g2, weights=g2["weights"], positions=g2["positions"])
    ws = pbd.op_workspace(pbd.decode_attention_workspace_bytes(kv2, hkv * group, True))
    out, lse = pbd.pbd_op_decode_attention(q.cuda(), kv2, *new, accumulate=True, want_lse=True, workspace=ws, sync=False)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        m = n + append
        live = torch.tensor(ok[b][:m], dtype=torch.bool)
        idx = live.nonzero()[:, 0]
        one = dict(c, table=c["table"][b:b + 1])  # (the table as it would be without the fault)
        k, v = ref.rows_of(one, c["k"], 0, n), ref.rows_of(one, c["v"], 0, n)
        if append:
            k, v = torch.cat([k, kn[b].double()[:, None]], 1), torch.cat([v, vn[b].double()[:, None]], 1)
        k, v = (x[:, idx].repeat_interleave(group, 0) for x in (k, v))
        w = c["weights"][b].double().clone()
        if append and live[n]:
            w[:, n] = 0
        tol = w * (group + 1) * 2.0 ** -23 + 1e-30
        if len(idx) == 0:
            assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
        else:
            s = torch.einsum("hd,hnd->hn", q[b].double(), k) * D ** -0.5
            l64 = torch.logsumexp(s, -1)
            p = torch.exp(s - l64[:, None])
            mag = torch.einsum("hd,hnd->hn", q[b].double().abs(), k.abs()).amax(-1) * D ** -0.5
            want = dict(out=torch.einsum("hn,hnd->hd", p, v), lse=l64, p=p, pv=torch.einsum("hn,hnd->hd", p, v.abs()), mag=mag)
            rel = _check_attention(torch, want, out[b], lse[b], m, HALF["bf16" if dtype == "bfloat16" else "fp16"])
            pw = p.view(hkv, group, -1)
            w[:, idx] += pw.sum(1)
            tol[:, idx] = w[:, idx] * (group + 1) * 2.0 ** -23 + 1e-30 + (pw * rel.view(hkv, group, 1)).sum(1)
        got = g["weights"][b].cpu()
        assert ((got.double() - w).abs() <= tol).all()
        dead = torch.ones(c["cap"], dtype=torch.bool)
        dead[idx] = False
        assert torch.equal(_bits(got[:, dead]), _bits(c["weights"][b][:, dead]))
