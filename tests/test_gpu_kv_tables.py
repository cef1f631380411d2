"""Page tables with room for far more pages than the sequences hold."""
import pytest

import _kv_oracle as ref
from test_gpu_kv_ops import env  # noqa: F401

pytestmark = pytest.mark.gpu


def _call(torch, pbd, B, max_pages, page, lens, hkv=1, D=64, seed=2):
    """A cache whose tables name pages outside it behind every sequence's last one."""
    used = [-(-n // page) for n in lens]
    table = torch.full((B, max_pages), 1 << 30, dtype=torch.int32)
    perm = torch.randperm(sum(used), generator=torch.Generator().manual_seed(seed)).int()
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = perm[at:at + u]
        at += u
    k, v = (torch.randn(max(1, sum(used)), hkv, page, D).bfloat16() for _ in range(2))
    c = dict(k=k, v=v, table=table, lens=torch.tensor(lens, dtype=torch.int32), page=page, cap=max_pages * page,
             weights=torch.rand(B, hkv, max_pages * page), positions=torch.arange(max_pages * page, dtype=torch.int32).repeat(B, hkv, 1))
    g = {n: c[n].cuda() for n in ("k", "v", "table", "lens", "weights", "positions")}
    return c, g, pbd.PagedKV(g["k"], g["v"], g["table"], g["lens"], weights=g["weights"], positions=g["positions"])


SHAPES = [(64, 2048, 8, 300), (1000, 300, 8, 40), (3, 30000, 1, 20000), (2, 9000, 1, 700), (1, 5, 16, 77), (20, 4000, 1, 33)]


@pytest.mark.parametrize("B,max_pages,page,most", SHAPES)
def test_pages_in_use_are_checked_and_no_others(env, B, max_pages, page, most):  # noqa: F811
    torch, pbd = env
    lens = [max(1, most - 7 * b % most) if b % 9 != 4 else 0 for b in range(B)]
    c, g, kv = _call(torch, pbd, B, max_pages, page, lens)
    keep = 20
    new_w, new_p = torch.zeros_like(g["weights"]), torch.zeros_like(g["positions"])
    q = torch.randn(B, 2, 64, device="cuda").bfloat16()

    def evict():
        pbd.pbd_op_evict(kv, keep, g["lens"], n_recent=4, n_sink=2, out_weights=new_w, out_positions=new_p)

    pbd.pbd_op_decode_attention(q, kv)
    evict()
    for b in {0, B // 2, B - 1}:
        if lens[b] == 0:
            continue
        src = ref.evict_row(c["weights"][b, 0].tolist(), range(lens[b]), lens[b], keep, lens[b], 4, 2)
        assert new_p[b, 0, :len(src)].tolist() == src
    for b in sorted({0, B // 3, B - 1}):
        last = -(-lens[b] // page) - 1
        for at in sorted({0, last // 2, last}):
            if last < 0:
                continue
            good = int(g["table"][b, at])
            for bad in (int(c["k"].shape[0]), -1):
                g["table"][b, at] = bad
                with pytest.raises(pbd.PbdError) as e:
                    pbd.pbd_op_decode_attention(q, kv)
                assert e.value.status == 6 and "page" in str(e.value)
                if lens[b] > keep:
                    with pytest.raises(pbd.PbdError) as e:
                        evict()
                    assert e.value.status == 6 and "page" in str(e.value)
                else:
                    evict()  # (a sequence that keeps all moves nothing)
            g["table"][b, at] = good
    pbd.pbd_op_decode_attention(q, kv)
    evict()


def test_room_in_a_table_costs_nothing(env):  # noqa: F811
    """64 sequences of 300 slots in tables of 64 and of 8192 pages: entries of no sequence take no time (they were walked over
    one by one, which took 14 times as long as all the rest)."""
    torch, pbd = env

    def us(max_pages):
        _, g, kv = _call(torch, pbd, 64, max_pages, 8, [300] * 64)
        new_w, new_p = torch.zeros_like(g["weights"]), torch.zeros_like(g["positions"])
        ws = pbd.op_workspace(pbd.evict_workspace_bytes(kv, 256))
        times = []
        for _ in range(12):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            pbd.pbd_op_evict(kv, 256, g["lens"], out_weights=new_w, out_positions=new_p, workspace=ws, sync=False)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b) * 1e3)
        return min(times)

    assert us(8192) < 4 * us(64) + 20
