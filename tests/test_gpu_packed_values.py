"""Attention over packed rows with the largest values of V that the header allows: 2^123 by the number of keys in bf16, the type's
largest in fp16."""
import math

import pytest

import _kv_oracle as kvref
import _packed_oracle as ref
from test_gpu_packed import env, to_gpu  # noqa: F401

pytestmark = pytest.mark.gpu

# K of a score that is 2^3.9 times as large as 1 at q = 1 and scale 1: within what the running maximum is not moved for, so that sums are
# taken of p up to 2^3.9 where the keys in front have scores of 0
HIGH = 2.703125


def largest(torch, dtype, n):
    """The largest value of the type that is no larger than 2^123 / n."""
    if dtype == "fp16":
        return 65504.0
    x = torch.tensor(2.0 ** 123 / n, dtype=torch.float64)
    y = x.to(torch.bfloat16)
    return float(y if y.double() <= x else torch.nextafter(y, torch.zeros_like(y)))


def signs(torch, shape):
    """Dimensions of one sign each, so that sums grow with every key; every seventh key of theirs is 0."""
    s = torch.ones(shape)
    s[..., 1::2] = -1
    s[::7] = 0
    return s


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,group", [(64, 3), (128, 2), (256, 1)])
def test_prompts(env, D, group, dtype):  # noqa: F811
    torch, pbd = env
    lens, hkv, dt = [700, 133], 2, getattr(torch, ref.DT[dtype])
    T = sum(lens)
    q, k, v = torch.zeros(T, hkv * group, D), torch.zeros(T, hkv, D), signs(torch, (T, hkv, D)) * largest(torch, dtype, T)
    q[..., 0] = 1
    starts = ref.starts_of(torch, lens)
    for s in starts[:-1].tolist():
        k[s + 128:, :, 0] = HIGH
    q, k, v = q.to(dt), k.to(dt), v.to(dt)
    out, lse = pbd.pbd_op_prompt_attention(q.cuda(), k.cuda(), v.cuda(), starts.cuda(), scale=1.0, want_lse=True)
    for b, n in enumerate(lens):
        at = slice(int(starts[b]), int(starts[b + 1]))
        want = ref.attend(torch, q[at], k[at], v[at], ref.causal(torch, n), 1.0)
        assert not want["odd"].any()
        ref.check(torch, want, out[at], lse[at], dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,group,lens,nodes", [
    (128, 2, [40000], [17]),                       # parts of many CTAs, joined
    (64, 7, [20000, 3], [5, 64]),
    (256, 1, [9000], [33]),
    (128, 2, [900, 0, 517, 128] * 12, [17, 64, 1, 9] * 12),  # whole units of a CTA
    (64, 7, [300, 129] * 20, [26, 3] * 20),
])
def test_trees(env, D, group, lens, nodes, dtype):  # noqa: F811
    torch, pbd = env
    hkv, page, dt = 2, 16, getattr(torch, ref.DT[dtype])
    c = ref.tree_case(torch, lens, nodes, hkv, D, page, dt, "heads")
    for b, (n, m) in enumerate(zip(lens, nodes)):
        at = torch.arange(n)
        p, o = c["table"][b].long()[at // page], at % page
        row = torch.zeros(n, hkv, D)
        row[128:, :, 0] = HIGH
        c["k"][p, :, o] = row.to(dt)
        c["v"][p, :, o] = (signs(torch, (n, hkv, D)) * largest(torch, dtype, n + m)).to(dt)
    T, starts = sum(nodes), ref.starts_of(torch, nodes)
    q, kn, vn = torch.zeros(T, hkv * group, D), torch.zeros(T, hkv, D), signs(torch, (T, hkv, D))
    q[..., 0], kn[..., 0] = 1, HIGH
    for b, (n, m) in enumerate(zip(lens, nodes)):
        vn[int(starts[b]):int(starts[b + 1])] *= largest(torch, dtype, n + m)
    q, kn, vn = q.to(dt), kn.to(dt), vn.to(dt)
    parents = ref.trees(torch, nodes)
    g = to_gpu(torch, c)
    out, lse = pbd.pbd_op_tree_attention(q.cuda(), pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"]), kn.cuda(), vn.cuda(), starts.cuda(), parents.cuda(),
                                         scale=1.0, want_lse=True)
    assert math.isfinite(float(out.float().abs().max()))
    for b, m in enumerate(nodes):
        at = slice(int(starts[b]), int(starts[b + 1]))
        n = lens[b]
        k, v = (torch.cat([kvref.rows_of(c, c[x], b, n).transpose(0, 1) if n else new[:0].double(), new[at].double()]) for x, new in (("k", kn), ("v", vn)))
        sees = torch.cat([torch.ones(m, n, dtype=torch.bool), ref.ancestors(torch, parents[at].tolist())], 1)
        ref.check(torch, ref.attend(torch, q[at], k, v, sees, 1.0), out[at], lse[at], dtype)
