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
