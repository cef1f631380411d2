"""Calls of the cache operators and the token log probabilities whose arrays reach too far or lie over one another are
refused before they touch a GPU."""
import pytest

from paper_2607_12422_gb300 import pbd
from test_kv_ops_args import A, attention, cache, evict, lib  # noqa: F401

G = 1 << 30  # distance of arrays that lie apart


def apart(**kw):
    """A cache whose arrays lie apart from one another and from what the calls below pass."""
    return cache(**dict(dict(d_k=A + G, d_v=A + 2 * G, d_page_table=A + 3 * G, d_lens=A + 4 * G, d_weights=A + 5 * G,
                             d_positions=A + 6 * G), **kw))


def attend(lib, kv=None, **kw):  # noqa: F811
    return attention(lib, kv or apart(), **dict(dict(q=A, kn=A + 7 * G, vn=A + 8 * G, pos=A + 9 * G, acc=1, out=A + 10 * G,
                                                     lse=A + 11 * G, ws=A + 12 * G), **kw))


def drop(lib, kv=None, **kw):  # noqa: F811
    return evict(lib, kv or apart(), **dict(dict(nxt=A + 9 * G, ow=A + 10 * G, op=A + 11 * G, ws=A + 12 * G), **kw))


def score(lib, M=2, V=100, dt=pbd.PBD_FP32, x=A, ld=100, tok=A + G, k=4, lp=A + 2 * G, ent=A + 3 * G, ids=A + 4 * G, top=A + 5 * G,  # noqa: F811
          ws=A + 6 * G):
    return lib.pbd_op_token_logprobs(M, V, dt, x, ld, 1.0, tok, k, lp, ent, ids, top, ws, 1 << 40, None)


@pytest.mark.parametrize("bad", [dict(stride_page=1 << 61), dict(stride_head=1 << 62), dict(stride_slot=1 << 58),
                                 dict(stride_page=(1 << 63) - 8)], ids=str)
def test_strides_that_wrap_are_refused(lib, bad):  # noqa: F811
    import ctypes as C
    kv = apart(**bad)
    assert attend(lib, kv, kn=None, vn=None, pos=None) == 1 and b"2^60" in lib.pbd_op_last_error()
    assert drop(lib, kv) == 1 and b"2^60" in lib.pbd_op_last_error()
    assert lib.pbd_op_decode_attention_workspace_bytes(C.byref(kv), 4, 1) == 0
    assert lib.pbd_op_evict_workspace_bytes(C.byref(kv), 16) == 0


def test_row_strides_that_wrap_are_refused(lib):  # noqa: F811
    for kw in (dict(qs=1 << 60), dict(ns=1 << 60), dict(qs=(1 << 63) - 8)):
        assert attend(lib, **kw) == 1 and b"2^60" in lib.pbd_op_last_error(), kw
    for kw in (dict(M=3, ld=1 << 60), dict(M=1 << 30, ld=1 << 31)):
        assert score(lib, **kw) == 1 and b"2^60" in lib.pbd_op_last_error(), kw


def accepted(status):
    """No argument was found wrong: the call got as far as the (absent) GPU."""
    return status not in (1, 2, 3)


def gpu():
    import torch
    return torch.cuda.is_available()


no_gpu = pytest.mark.skipif("gpu()", reason="addresses that are no memory must not reach a GPU")

PS, H, D = 16, 2, 128  # slots of a page, heads, their size in `cache`
# strides of pages, heads and slots whose rows lie over one another although each is a row or more
OVER = [(H * PS * D, D, D),               # head 1 of a slot is head 0 of the next
        (D, 9 * D, 20 * D),               # ten pages over the next head
        (PS * D, PS * D, D),              # a page's heads over the next page's
        (H * PS * D, PS * D - 8, D),      # the last slot's row over the next head's first
        (H * PS * D - 8, PS * D, D), (H * D, D, H * D),
        (10 * H * D, 7 * D, D + 8)]       # 16 slots reach over the next head's
# any order of the dimensions that keeps rows apart
APART = [(H * PS * D, PS * D, D), (H * PS * D, D, H * D), (D, 10 * PS * D, 10 * D), (H * D, D, 10 * H * D), (2 * H * PS * D, PS * D, D),
         (H * PS * (D + 8) + 64, PS * (D + 8), D + 8)]


@pytest.mark.parametrize("strides", OVER, ids=str)
def test_written_rows_that_lie_over_one_another_are_refused(lib, strides):  # noqa: F811
    kv = apart(**dict(zip(("stride_page", "stride_head", "stride_slot"), strides)))
    assert attend(lib, kv) == 1 and b"rows" in lib.pbd_op_last_error()
    assert drop(lib, kv) == 1 and b"rows" in lib.pbd_op_last_error()


@no_gpu
def test_other_strides_are_not(lib):  # noqa: F811
    for strides in APART:
        kv = apart(**dict(zip(("stride_page", "stride_head", "stride_slot"), strides)))
        assert accepted(attend(lib, kv)) and accepted(drop(lib, kv)), strides
    for strides in OVER:  # a cache that is only read
        kv = apart(**dict(zip(("stride_page", "stride_head", "stride_slot"), strides)))
        assert accepted(attend(lib, kv, kn=None, vn=None, pos=None)), strides
    # one page, one head or one slot: that stride does not matter
    assert accepted(drop(lib, apart(n_pages=1, stride_page=0)))
    assert accepted(drop(lib, apart(n_kv_heads=1, stride_head=0, stride_page=PS * D)))
    assert accepted(drop(lib, apart(page_size=1, stride_slot=0, stride_head=D, stride_page=H * D)))


def test_written_k_and_v_over_one_another_are_refused(lib):  # noqa: F811
    page = 2 * H * PS * D  # [page][K or V][head][slot][d]
    for off in (0, 1, PS, H * PS - 1, 2 * H * PS * 9 + 1, -1, -2 * H * PS):  # rows of V behind K
        kv = apart(stride_page=page, stride_head=PS * D, stride_slot=D, d_v=A + G + 2 * D * off)
        assert attend(lib, kv) == 1 and b"K and V" in lib.pbd_op_last_error(), off
        assert drop(lib, kv) == 1 and b"K and V" in lib.pbd_op_last_error(), off
    kv = apart(stride_page=page, stride_head=2 * PS * D, stride_slot=2 * D, d_v=A + G + 2 * (D - 8))  # the end of K's row
    assert attend(lib, kv) == 1 and drop(lib, kv) == 1


@no_gpu
def test_k_and_v_in_turns_are_not(lib):  # noqa: F811
    # [page][K or V][head][slot][d], [page][head][slot][K or V][d], [page][head][K or V][slot][d]; and a cache that is only read
    for strides, off in (((2 * H * PS * D, PS * D, D), H * PS), ((2 * H * PS * D, 2 * PS * D, 2 * D), 1),
                         ((2 * H * PS * D, 2 * PS * D, D), PS), ((2 * H * PS * D, PS * D, D), -H * PS),
                         ((2 * H * PS * D, PS * D, D), 2 * 10 * H * PS)):
        kv = apart(**dict(zip(("stride_page", "stride_head", "stride_slot"), strides), d_v=A + G + 2 * D * off))
        assert accepted(attend(lib, kv)) and accepted(drop(lib, kv)), (strides, off)
    assert accepted(attend(lib, apart(d_v=A + G), kn=None, vn=None, pos=None))


@no_gpu
def test_rows_over_one_another_by_counting(lib):  # noqa: F811
    """Random small caches: rows counted out one by one.  Strides that keep rows apart in no order of the dimensions may be
    refused as well."""
    import random
    r = random.Random(3)
    seen = [0, 0]
    for _ in range(3000):
        n, h, s = (r.randint(1, 3) for _ in range(3))
        st = [64 * r.choice([1, 2, 3, 4, 6, 8, 12]) + 8 * r.choice([0, 0, 1, -1]) for _ in range(3)]
        off = r.choice([0, 8, 64, 120, 128, 192, 256, 384, 512, 1024, 4096, -64, -128, -512]) + 8 * r.choice([0, 0, 1, -1])
        kv = apart(n_pages=n, n_kv_heads=h, page_size=s, head_dim=64, stride_page=st[0], stride_head=st[1], stride_slot=st[2], d_v=A + G + 2 * off)
        rows = sorted(p * st[0] + i * st[1] + j * st[2] for p in range(n) for i in range(h) for j in range(s))
        over = any(b - a < 64 for a, b in zip(rows, rows[1:]))
        meet = any(abs(a - b - off) < 64 for a in rows for b in rows)
        ok = accepted(drop(lib, kv))
        assert accepted(attention(lib, kv, hq=h, q=A, kn=A + 7 * G, vn=A + 8 * G, ns=h * 64, out=A + 10 * G, ws=A + 12 * G)) == ok
        seen[ok] += 1
        if over or meet:
            assert not ok, (n, h, s, st, off)
        else:
            assert ok or b"strides of a row" in lib.pbd_op_last_error() or b"the rows" in lib.pbd_op_last_error(), (n, h, s, st, off)
    assert min(seen) > 300


def overlays(at, written, read, sizes):
    """Every written array over the beginning and the end of every other one."""
    for w in written:
        for other in written + read:
            if other == w or {w, other} == {"d_k", "d_v"}:
                continue
            for to in (at[other], at[other] + (sizes[other] - 16) // 16 * 16):
                if w == "ws":
                    to = to // 1024 * 1024
                yield w, other, to


@no_gpu
def test_what_attention_writes_lies_over_nothing_else(lib):  # noqa: F811
    at = dict(q=A, d_k=A + G, d_v=A + 2 * G, d_page_table=A + 3 * G, d_lens=A + 4 * G, d_weights=A + 5 * G, d_positions=A + 6 * G, kn=A + 7 * G,
              vn=A + 8 * G, pos=A + 9 * G, out=A + 10 * G, lse=A + 11 * G, ws=A + 12 * G)
    B, hq, cap, table = 3, 4, 64, 4
    kv_bytes = 2 * 10 * H * PS * D
    sizes = dict(q=2 * B * hq * D, d_k=kv_bytes, d_v=kv_bytes, d_page_table=4 * B * table, d_lens=4 * B, d_weights=4 * B * H * cap,
                 d_positions=4 * B * H * cap, kn=2 * B * H * D, vn=2 * B * H * D, pos=4 * B, out=2 * B * hq * D, lse=4 * B * hq, ws=1024)

    def call(**moved):
        x = {**at, **moved}
        kv = cache(**{n: a for n, a in x.items() if n.startswith("d_")})
        return attention(lib, kv, acc=1, **{n: a for n, a in x.items() if not n.startswith("d_")})

    assert accepted(call())
    for w, other, to in overlays(at, ("out", "lse", "ws", "d_k", "d_v", "d_weights", "d_positions"), ("q", "kn", "vn", "pos", "d_page_table", "d_lens"), sizes):
        assert call(**{w: to}) == 1, (w, other)
        assert b"lies over" in lib.pbd_op_last_error() or b"lie over" in lib.pbd_op_last_error(), (w, other)
    # what is only read may lie anywhere, and without a new row or weights so may K, V, weights and positions
    assert accepted(call(kn=at["q"], vn=at["q"])) and accepted(call(pos=at["d_lens"]))
    kv = cache(d_k=A + G, d_v=A + G, d_weights=A + G, d_positions=A + G, d_page_table=A + 3 * G, d_lens=A + 3 * G)
    assert accepted(attention(lib, kv, q=A + G, out=at["out"], ws=at["ws"]))


@no_gpu
def test_what_eviction_writes_lies_over_nothing_else(lib):  # noqa: F811
    at = dict(d_k=A + G, d_v=A + 2 * G, d_page_table=A + 3 * G, d_lens=A + 4 * G, d_weights=A + 5 * G, d_positions=A + 6 * G, nxt=A + 9 * G,
              ow=A + 10 * G, op=A + 11 * G, ws=A + 12 * G)
    B, cap, table = 3, 64, 4
    kv_bytes = 2 * 10 * H * PS * D
    sizes = dict(d_k=kv_bytes, d_v=kv_bytes, d_page_table=4 * B * table, d_lens=4 * B, d_weights=4 * B * H * cap, d_positions=4 * B * H * cap,
                 nxt=4 * B, ow=4 * B * H * cap, op=4 * B * H * cap, ws=1024)

    def call(**moved):
        x = {**at, **moved}
        kv = cache(**{n: a for n, a in x.items() if n.startswith("d_")})
        return evict(lib, kv, **{n: a for n, a in x.items() if not n.startswith("d_")})

    assert accepted(call()) and accepted(call(ow=at["d_weights"], op=at["d_positions"]))
    written, read = ("d_k", "d_v", "ow", "op", "ws"), ("d_page_table", "d_lens", "d_weights", "d_positions", "nxt")
    for w, other, to in overlays(at, written, read, sizes):
        assert call(**{w: to}) == 1, (w, other)
    # in place, weights and positions are written
    for moved in (dict(d_weights=at["d_positions"], ow=at["d_positions"], op=at["d_positions"]), dict(d_weights=at["d_k"], ow=at["d_k"], op=at["d_positions"]),
                  dict(d_positions=at["nxt"], op=at["nxt"], ow=at["d_weights"]), dict(d_weights=at["d_lens"], ow=at["d_lens"], op=at["d_positions"])):
        assert call(**moved) == 1, moved


@no_gpu
def test_what_log_probabilities_write_lies_over_nothing_else(lib):  # noqa: F811
    at = dict(x=A, tok=A + G, lp=A + 2 * G, ent=A + 3 * G, ids=A + 4 * G, top=A + 5 * G, ws=A + 6 * G)
    M, V, ld, k = 40, 100, 120, 4
    sizes = dict(x=4 * ((M - 1) * ld + V), tok=4 * M, lp=4 * M, ent=4 * M, ids=4 * M * k, top=4 * M * k, ws=1024)

    def call(**moved):
        return score(lib, M=M, V=V, ld=ld, k=k, **{**at, **moved})

    assert accepted(call())
    for w, other, to in overlays(at, ("lp", "ent", "ids", "top", "ws"), ("x", "tok"), sizes):
        assert call(**{w: to}) == 1 and b"lies over" in lib.pbd_op_last_error(), (w, other)
    # what is read may lie anywhere, behind the last row is free, and what is not asked for is not looked at
    assert accepted(call(tok=at["x"])) and accepted(call(lp=at["x"] + sizes["x"])) and accepted(call(ent=None))
    assert accepted(score(lib, M=M, V=V, ld=ld, k=0, **{**at, "ids": at["x"], "top": at["lp"]}))
