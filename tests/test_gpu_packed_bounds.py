"""Packed rows whose bounds descend: a sequence that begins below a bound in front of its own is left out, so that no row is
two sequences'."""
import pytest

import _packed_oracle as ref
from test_gpu_packed import env, i32, to_gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def taken(starts, T, most):
    """The sequences that take part, by the header's words."""
    return [b for b in range(len(starts) - 1)
            if 0 <= starts[b] <= starts[b + 1] <= T and starts[b + 1] - starts[b] <= most and all(s <= starts[b] for s in starts[:b])]


T = 60
BOUNDS = [
    [0, 20, 10, 60],          # the third would lie over the first
    [0, 60, 0, 60],
    [0, 20, 10, 30, 40, 60],  # what begins behind all bounds again takes part
    [5, 5, 4, 50, 50, 60],
    [0, 70, 30, 60],
    [-3, 20, -5, 10, 20, 41],
    [10, 0, 10, 10, 60],
    [0] + [1 + i // 2 for i in range(40)] + [7, 33, 33, 60],   # more than 32 sequences
    [0] * 700 + [30, 29, 31] + [31] * 200 + [60],              # more than a CTA's threads, the descent behind them
    [9, 3] + [i // 20 for i in range(1000)] + [60],            # and in front
]


@pytest.mark.parametrize("D,group", [(128, 2), (64, 7), (256, 1)])
@pytest.mark.parametrize("starts", BOUNDS, ids=lambda s: "%d-%s" % (len(s) - 1, "-".join(map(str, s[:3]))))
def test_prompts(env, starts, D, group):  # noqa: F811
    torch, pbd = env
    hkv, page = 2, 16
    hq, dt = hkv * group, torch.bfloat16
    q, k, v = ref.rows(torch, T, hq, hkv, D, dt, False)
    ck, cv = (torch.full((4, hkv, page, D), 7.0, dtype=dt, device="cuda") for _ in range(2))
    B = len(starts) - 1
    kv = pbd.PagedKV(ck, cv, i32(torch, [[0]] * B), i32(torch, [0] * B))
    slots = torch.arange(T, device="cuda").flip(0).contiguous()
    out, lse = torch.full((T, hq, D), 7.0, dtype=dt, device="cuda"), torch.full((T, hq), 7.0, device="cuda")
    with pytest.raises(pbd.PbdError, match="PBD_ERR_DEVICE"):
        pbd.pbd_op_prompt_attention(q.cuda(), k.cuda(), v.cuda(), i32(torch, starts), kv=kv, slots=slots, out=out, lse=lse)
    rest = torch.ones(T, dtype=torch.bool)
    for b in taken(starts, T, T):
        at = slice(starts[b], starts[b + 1])
        if at.start < at.stop:
            assert rest[at].all()
            rest[at] = False
            ref.check(torch, ref.attend(torch, q[at], k[at], v[at], ref.causal(torch, at.stop - at.start)), out[at], lse[at], "bf16")
    assert (out[rest.cuda()] == 7).all() and (lse[rest.cuda()] == 7).all()
    for x, new in ((ck, k), (cv, v)):
        rows = x.transpose(1, 2).reshape(4 * page, hkv, D)[:T].flip(0).cpu()
        assert torch.equal(rows[~rest], new[~rest]) and (rows[rest] == 7).all()


@pytest.mark.parametrize("D,group", [(128, 2), (64, 7), (256, 1)])
@pytest.mark.parametrize("starts", BOUNDS, ids=lambda s: "%d-%s" % (len(s) - 1, "-".join(map(str, s[:3]))))
def test_trees(env, starts, D, group):  # noqa: F811
    torch, pbd = env
    hkv, page, dt = 2, 16, torch.bfloat16
    hq, B = hkv * group, len(starts) - 1
    lens = [(37 * b) % 50 for b in range(B)]
    c = ref.tree_case(torch, lens, [64] * B, hkv, D, page, dt, "heads")
    g = to_gpu(torch, c)
    q, kn, vn = ref.rows(torch, T, hq, hkv, D, dt, False)
    parents = torch.full((T,), -1, dtype=torch.int32)
    out, lse = torch.full((T, hq, D), 7.0, dtype=dt, device="cuda"), torch.full((T, hq), 7.0, device="cuda")
    with pytest.raises(pbd.PbdError, match="PBD_ERR_DEVICE"):
        pbd.pbd_op_tree_attention(q.cuda(), pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"]), kn.cuda(), vn.cuda(), i32(torch, starts), parents.cuda(),
                                  out=out, lse=lse)
    rest, filled = torch.ones(T, dtype=torch.bool), {n: c[n].clone() for n in ("k", "v")}
    for b in taken(starts, T, 64):
        at = slice(starts[b], starts[b + 1])
        if at.start == at.stop:
            continue
        assert rest[at].all()
        rest[at] = False
        ref.check(torch, ref.tree_attention(torch, c, b, q[at], kn[at], vn[at], parents[at]), out[at], lse[at], "bf16")
        for i in range(at.stop - at.start):
            p, o = int(c["table"][b, (lens[b] + i) // page]), (lens[b] + i) % page
            filled["k"][p, :, o], filled["v"][p, :, o] = kn[at][i], vn[at][i]
    assert (out[rest.cuda()] == 7).all() and (lse[rest.cuda()] == 7).all()
    for n in ("k", "v"):
        assert torch.equal(g[n].cpu().view(torch.int16), filled[n].view(torch.int16))
