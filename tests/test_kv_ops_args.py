"""What the entry points of the cache operators and the token log probabilities refuse, before they touch a GPU."""
import ctypes as C
import os
import shutil

import pytest

from paper_2607_12422_gb300 import pbd

A = 0x100000  # an aligned address that no call here gets to use


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pbd.LIB_PATH):
        if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
            pytest.skip("nvcc unavailable and libpbd.so not built")
        from paper_2607_12422_gb300 import build
        build.build()
    return pbd.load()


def cache(**kw):
    c = pbd.pbd_kv_pages(A, A, pbd.PBD_BF16, 10, 16, 2, 128, 3, 4, 2 * 16 * 128, 16 * 128, 128, A, A, A, A)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD = [dict(dtype=pbd.PBD_FP32), dict(dtype=9), dict(batch=0), dict(batch=1025), dict(n_kv_heads=0), dict(n_kv_heads=257),
       dict(head_dim=96), dict(head_dim=0), dict(n_pages=0), dict(page_size=0), dict(max_pages=0), dict(page_size=1 << 20, max_pages=1 << 11),
       dict(stride_page=-8), dict(stride_head=4), dict(stride_slot=129)]
BAD_POINTERS = [dict(d_k=None), dict(d_v=None), dict(d_page_table=None), dict(d_lens=None), dict(d_k=A + 8), dict(d_v=A + 2),
                dict(d_lens=A + 2)]


def attention(lib, kv, hq=4, scale=1.0, q=A, qs=None, kn=None, vn=None, ns=256, pos=None, acc=0, out=A, lse=None, ws=A, n=1 << 40):
    return lib.pbd_op_decode_attention(C.byref(kv) if kv else None, hq, scale, q, qs or hq * 128, kn, vn, ns, pos, acc, out, lse,
                                       ws, n, None)


def evict(lib, kv, keep=16, recent=0, sink=0, nxt=A, ow=A, op=A, ws=A, n=1 << 40):
    return lib.pbd_op_evict(C.byref(kv) if kv else None, keep, recent, sink, nxt, ow, op, ws, n, None)


@pytest.mark.parametrize("bad", BAD + BAD_POINTERS, ids=str)
def test_caches_that_are_refused(lib, bad):
    kv = cache(**bad)
    assert attention(lib, kv) == 1 and b"pbd_op_decode_attention" in lib.pbd_op_last_error()
    assert evict(lib, kv) == 1 and b"pbd_op_evict" in lib.pbd_op_last_error()
    sizes = bad in BAD
    assert (lib.pbd_op_decode_attention_workspace_bytes(C.byref(kv), 4, 1) == 0) == sizes
    assert (lib.pbd_op_evict_workspace_bytes(C.byref(kv), 16) == 0) == sizes


def test_attention_arguments(lib):
    kv = cache()
    assert attention(lib, None) == 1
    for kw in (dict(hq=3), dict(hq=1), dict(hq=0), dict(hq=-2), dict(hq=8192), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(q=None), dict(out=None), dict(q=A + 8), dict(out=A + 4), dict(kn=A), dict(vn=A),
               dict(kn=A, vn=A + 8), dict(qs=511), dict(qs=516), dict(kn=A, vn=A, ns=128), dict(kn=A, vn=A, ns=260)):
        assert attention(lib, kv, **kw) == 1, kw
    # the output over q, the cache or the new rows
    for kw in (dict(out=A), dict(q=A + (1 << 30), qs=1 << 20, out=A + (1 << 30) + (2 << 20)), dict(out=A + 2 * 10 * 4096 - 16),
               dict(kn=A + (1 << 24), vn=A + (1 << 25), out=A + (1 << 25) + 1520)):
        kw = dict(dict(q=A + (1 << 28)), **kw)
        assert attention(lib, kv, **kw) == 1 and b"lies over" in lib.pbd_op_last_error(), kw
    # new rows into a cache whose rows lie over one another
    for bad in (dict(stride_slot=0), dict(stride_head=64), dict(stride_page=0)):
        assert attention(lib, cache(**bad), kn=A, vn=A, q=A + (1 << 28), out=A + (1 << 29)) == 1, bad
    kv = cache(d_k=A + (1 << 26), d_v=A + (1 << 27))
    assert attention(lib, cache(d_weights=None, d_k=A + (1 << 26), d_v=A + (1 << 27)), acc=1, out=A + (1 << 29)) == 1 and b"d_weights" in lib.pbd_op_last_error()
    need = lib.pbd_op_decode_attention_workspace_bytes(C.byref(kv), 4, 0)
    assert need and lib.pbd_op_decode_attention_workspace_bytes(C.byref(kv), 4, 1) > need
    for kw in (dict(ws=None), dict(ws=A + 16), dict(n=need - 1), dict(n=need, acc=1)):
        assert attention(lib, kv, out=A + (1 << 29), **kw) == 2, kw
    # more 16-slot tiles than 32 bits count
    big = cache(batch=1024, page_size=1 << 15, max_pages=1 << 15)
    assert attention(lib, big, out=A + (1 << 50)) == 3 and lib.pbd_op_decode_attention_workspace_bytes(C.byref(big), 4, 0) == 0


def test_evict_arguments(lib):
    kv = cache()
    assert evict(lib, None) == 1
    for kw in (dict(keep=-1), dict(recent=-1), dict(sink=-1), dict(keep=8, recent=5, sink=4), dict(keep=8, recent=2**31 - 1, sink=8),
               dict(nxt=None), dict(ow=None), dict(op=None),
               dict(ow=A, op=A + 4096),       # one of them the cache's own
               dict(ow=A + 64, op=A + 64)):   # over a part of them
        assert evict(lib, kv, **kw) == 1, kw
    for bad in (dict(stride_slot=0), dict(stride_head=64), dict(stride_page=0)):
        assert evict(lib, cache(**bad), ow=A + (1 << 20), op=A + (1 << 21)) == 1 and b"strides" in lib.pbd_op_last_error(), bad
    assert evict(lib, cache(d_weights=None)) == 1 and evict(lib, cache(d_positions=None)) == 1
    need = lib.pbd_op_evict_workspace_bytes(C.byref(kv), 16)
    for kw in (dict(ws=None), dict(ws=A + 16), dict(n=need - 1)):
        assert evict(lib, kv, **kw) == 2, kw
    assert lib.pbd_op_evict_workspace_bytes(C.byref(kv), -1) == 0
    assert lib.pbd_op_evict_workspace_bytes(C.byref(kv), 0) > 0


def test_logprob_arguments(lib):
    def call(M=2, V=100, dt=pbd.PBD_FP32, x=A, ld=100, T=1.0, tok=A, k=4, lp=A, ent=A, ids=A, top=A, ws=A, n=1 << 40):
        return lib.pbd_op_token_logprobs(M, V, dt, x, ld, T, tok, k, lp, ent, ids, top, ws, n, None)
    for kw in (dict(M=0), dict(V=0), dict(V=(1 << 30) + 1, ld=1 << 31), dict(k=-1), dict(k=33), dict(V=3, k=4), dict(dt=7), dict(x=None), dict(x=A + 2),
               dict(dt=pbd.PBD_BF16, x=A + 1), dict(ld=99), dict(T=0.0), dict(T=-1.0), dict(T=float("nan")), dict(T=float("inf")),
               dict(T=1e-45), dict(tok=None), dict(lp=None), dict(ids=None), dict(top=None)):
        assert call(**kw) == 1, kw
    need = lib.pbd_op_token_logprobs_workspace_bytes(2, 100, 4)
    for kw in (dict(ws=None), dict(ws=A + 512), dict(n=need - 1)):
        assert call(**kw) == 2, kw
    assert lib.pbd_op_token_logprobs_workspace_bytes(1, 100, 33) == 0


def test_calls_that_would_address_or_scale_out_of_range(lib):
    kv = cache(d_k=A + (1 << 26), d_v=A + (1 << 27))
    far = dict(out=A + (1 << 29))
    # a 32-bit array off its boundary
    for kw in (dict(lse=A + 2), dict(pos=A + 1)):
        assert attention(lib, kv, **far, **kw) == 1 and b"4-byte" in lib.pbd_op_last_error(), kw
    for kw in (dict(nxt=A + 2), dict(ow=A + (1 << 20) + 1, op=A + (1 << 21)), dict(ow=A + (1 << 20), op=A + (1 << 21) + 3)):
        assert evict(lib, kv, **kw) == 1 and b"4-byte" in lib.pbd_op_last_error(), kw
    # two outputs over one another
    assert evict(lib, kv, ow=A + (1 << 20), op=A + (1 << 20) + 64) == 1 and b"one another" in lib.pbd_op_last_error()

    def logprobs(M=2, T=1.0, tok=A, lp=A, ent=A, ids=A, top=A):
        return lib.pbd_op_token_logprobs(M, 100, pbd.PBD_FP32, A, 100, T, tok, 4, lp, ent, ids, top, A, 1 << 40, None)
    for name in ("tok", "lp", "ent", "ids", "top"):
        assert logprobs(**{name: A + 2}) == 1 and b"4-byte" in lib.pbd_op_last_error(), name
    # rows that 32 bits cannot count on from
    assert logprobs(M=2**31 - 1) == 1 and lib.pbd_op_token_logprobs_workspace_bytes((1 << 30) + 1, 100, 4) == 0
    # factors that log2 e takes over the largest number: 2.36e38 * 1.4427 = 3.405e38 > 3.4028e38
    assert logprobs(T=1 / 2.5e38) == 1
    assert attention(lib, kv, scale=2.5e38, **far) == 1
