"""Python binding of libpbd (include/pbd.h): argument marshalling only.

Every step of a pass runs in the library's CUDA kernels; PyTorch is used here only to
own device memory (weights, workspace, outputs) and the CUDA stream.  If the compiled
library is missing this module raises; there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
import re
from typing import Dict, List, NamedTuple, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "lib", "libpbd.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "pbd.h")

PBD_OK = 0
STATUS_NAMES = {0: "PBD_OK", 1: "PBD_ERR_INVALID_ARG", 2: "PBD_ERR_WORKSPACE", 3: "PBD_ERR_CAPACITY",
                4: "PBD_ERR_STATE", 5: "PBD_ERR_CUDA", 6: "PBD_ERR_DEVICE"}
LINEARS = ("q", "k", "v", "o", "gate", "up", "down")
TRACE_STAMPS = 16  # timestamps per work item of pbd_trace_pass


class PbdError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("%s: %s" % (STATUS_NAMES.get(status, status), msg))
        self.status = status


class pbd_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("hidden", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("intermediate", C.c_int32),
                ("vocab", C.c_int32), ("rms_eps", C.c_float), ("rope_theta", C.c_float),
                ("lora_rank", C.c_int32), ("lora_scale", C.c_float), ("block_D", C.c_int32),
                ("max_batch", C.c_int32), ("max_seq_len", C.c_int32), ("page_size", C.c_int32),
                ("draft_layers", C.c_int32), ("denoise_steps", C.c_int32), ("draft_unanchored", C.c_int32),
                ("draft_skip_mask", C.c_uint64), ("max_ctas", C.c_int32)]


class pbd_base_weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("final_norm", C.c_void_p), ("attn_norm", C.c_void_p),
                ("mlp_norm", C.c_void_p), ("q_norm", C.c_void_p), ("k_norm", C.c_void_p), ("w", C.c_void_p * 7)]


class pbd_adapter_weights(C.Structure):
    _fields_ = [("lora_a", C.c_void_p * 7), ("lora_b", C.c_void_p * 7), ("mask_embed", C.c_void_p)]


PBD_BF16, PBD_FP16, PBD_FP32 = 0, 1, 2  # pbd_dtype


class pbd_kv_pages(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("dtype", C.c_int32), ("n_pages", C.c_int32),
                ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("batch", C.c_int32),
                ("max_pages", C.c_int32), ("stride_page", C.c_int64), ("stride_head", C.c_int64),
                ("stride_slot", C.c_int64), ("d_page_table", C.c_void_p), ("d_lens", C.c_void_p),
                ("d_weights", C.c_void_p), ("d_positions", C.c_void_p)]


class pbd_stats(C.Structure):
    _fields_ = [("rounds", C.c_int64), ("accepted", C.c_int64), ("emitted", C.c_int64),
                ("draft_ms", C.c_double), ("verify_ms", C.c_double)]


_lib = None


def header_functions() -> List[str]:
    """Names of the functions include/pbd.h and include/pbd_ops.h declare."""
    names = set()
    for h in (HEADER, os.path.join(os.path.dirname(HEADER), "pbd_ops.h")):
        txt = re.sub(r"/\*.*?\*/", "", open(h).read(), flags=re.S)
        names.update(re.findall(r"\b(pbd_[a-z_]+)\s*\(", txt))
    return sorted(names)


def load(path: str = LIB_PATH) -> C.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError("libpbd.so is not built (%s); run __graft_entry__.build()" % path)
    L = C.CDLL(path)
    P = C.c_void_p
    I32 = C.c_int32
    L.pbd_workspace_bytes.restype = C.c_size_t
    L.pbd_workspace_bytes.argtypes = [C.POINTER(pbd_config)]
    L.pbd_create.argtypes = [C.POINTER(pbd_config), C.POINTER(pbd_base_weights), C.POINTER(pbd_adapter_weights),
                             P, C.c_size_t, P, C.POINTER(P)]
    L.pbd_destroy.argtypes = [P]
    L.pbd_prefill.argtypes = [P, I32, P, P, I32, P]
    L.pbd_draft_block.argtypes = [P, P, P]
    L.pbd_verify_block.argtypes = [P, P, P, P]
    L.pbd_accept_commit.argtypes = [P, P, P]
    L.pbd_decode_step.argtypes = [P, P, P]
    L.pbd_generate.argtypes = [P, I32, P, P, I32, I32, P, P, C.POINTER(pbd_stats)]
    L.pbd_get_state.argtypes = [P, P, P, P]
    L.pbd_get_tokens.argtypes = [P, P]
    L.pbd_read_kv.argtypes = [P, I32, I32, I32, P, P]
    L.pbd_sync.argtypes = [P]
    L.pbd_last_error.restype = C.c_char_p
    L.pbd_last_error.argtypes = [P]
    L.pbd_version.restype = C.c_char_p
    L.pbd_bench_rounds.argtypes = [P, I32, I32, I32, P, P, P]
    L.pbd_time_pass.argtypes = [P, I32, I32, P, P]
    L.pbd_trace_pass.argtypes = [P, I32, P, P, I32, P]
    L.pbd_trace_pass.restype = C.c_int
    L.pbd_bench_rounds.restype = C.c_int
    L.pbd_time_pass.restype = C.c_int
    L.pbd_check_stalled_pass.argtypes = [P, P]
    L.pbd_check_stalled_pass.restype = C.c_int
    L.pbd_plan_pass.argtypes = [C.POINTER(pbd_config), I32, I32, P, I32, I32, P, P, I32, P]
    L.pbd_plan_pass.restype = C.c_int
    L.pbd_op_linear_workspace_bytes.restype = C.c_size_t
    L.pbd_op_linear_workspace_bytes.argtypes = [I32, I32, I32, I32]
    L.pbd_op_linear.argtypes = [I32, I32, I32, I32, C.c_float, P, P, P, P, P, P, C.c_size_t, P]
    L.pbd_op_lm_head_workspace_bytes.restype = C.c_size_t
    L.pbd_op_lm_head_workspace_bytes.argtypes = [I32, I32, I32]
    L.pbd_op_lm_head_argmax.argtypes = [I32, I32, I32, P, P, P, P, P, C.c_size_t, P]
    L.pbd_op_last_error.restype = C.c_char_p
    L.pbd_op_linear_static.argtypes = [I32, I32, I32, I32, C.c_float, P, P, P, P, P, P]
    L.pbd_op_linear_static.restype = C.c_int
    L.pbd_op_status.argtypes = [P, P, P]
    L.pbd_op_status.restype = C.c_int
    L.pbd_op_linear_static_status.argtypes = [P, P]
    L.pbd_op_linear_static_status.restype = C.c_int
    I64, F, Z, KV = C.c_int64, C.c_float, C.c_size_t, C.POINTER(pbd_kv_pages)
    L.pbd_op_decode_attention_workspace_bytes.argtypes = [KV, I32, I32]
    L.pbd_op_decode_attention.argtypes = [KV, I32, F, P, I64, P, P, I64, P, I32, P, P, P, Z, P]
    L.pbd_op_evict_workspace_bytes.argtypes = [KV, I32]
    L.pbd_op_evict.argtypes = [KV, I32, I32, I32, P, P, P, P, Z, P]
    L.pbd_op_token_logprobs_workspace_bytes.argtypes = [I32, I32, I32]
    L.pbd_op_token_logprobs.argtypes = [I32, I32, I32, P, I64, F, P, I32, P, P, P, P, P, Z, P]
    for name in ("decode_attention", "evict", "token_logprobs"):
        getattr(L, "pbd_op_" + name).restype = C.c_int
        getattr(L, "pbd_op_%s_workspace_bytes" % name).restype = C.c_size_t
    for name in ("pbd_create", "pbd_destroy", "pbd_prefill", "pbd_draft_block", "pbd_verify_block",
                 "pbd_accept_commit", "pbd_decode_step", "pbd_generate", "pbd_get_state", "pbd_get_tokens",
                 "pbd_read_kv", "pbd_sync", "pbd_op_linear", "pbd_op_lm_head_argmax"):
        getattr(L, name).restype = C.c_int
    _lib = L
    return L


def _ws(torch, nbytes, device):
    """1024-byte-aligned view into a fresh uint8 device buffer."""
    buf = torch.empty(nbytes + 1024, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 1024
    return buf, buf.data_ptr() + off


def _raise_if(L, s):
    if s != PBD_OK:
        raise PbdError(s, L.pbd_op_last_error().decode())


def pbd_op_linear(x, W, A=None, B=None, scale: float = 2.0):
    """y = bf16(x W^T + scale * bf16(x A^T) B^T) on the GPU (torch bf16 device tensors in, out).
    Waits for the result and raises PbdError(PBD_ERR_DEVICE) if a kernel latched an error."""
    import torch
    L = load()
    M, K = x.shape
    N = W.shape[0]
    r = A.shape[0] if (A is not None and B is not None) else 0
    need = L.pbd_op_linear_workspace_bytes(M, K, N, r)
    if need == 0:
        raise PbdError(1, "pbd_op_linear: unsupported sizes")
    with torch.cuda.device(x.device):  # the library runs on the current device
        buf, ws = _ws(torch, need, x.device)
        y = torch.empty(M, N, dtype=torch.bfloat16, device=x.device)
        st = torch.cuda.current_stream(x.device).cuda_stream
        _raise_if(L, L.pbd_op_linear(M, K, N, r, scale, x.data_ptr(), W.data_ptr(), _ptr(A) if r else None,
                                     _ptr(B) if r else None, y.data_ptr(), ws, need, st))
        _raise_if(L, L.pbd_op_status(ws, st, None))
    del buf
    return y


def pbd_op_linear_static(x, W, A=None, B=None, scale: float = 2.0, y=None, sync: bool = True):
    """pbd_op_linear through the entry point that takes no workspace (the library's own static
    scratch); y [M, N] bf16 is the caller's output tensor (allocated here when not given).
    With sync, waits and raises PbdError(PBD_ERR_DEVICE) if the kernel latched an error; without
    it the caller asks pbd_op_linear_static_status before the next call."""
    import torch
    L = load()
    M, K = x.shape
    N = W.shape[0]
    r = A.shape[0] if (A is not None and B is not None) else 0
    with torch.cuda.device(x.device):  # the library picks its scratch by the current device
        if y is None:
            y = torch.empty(M, N, dtype=torch.bfloat16, device=x.device)
        st = torch.cuda.current_stream(x.device).cuda_stream
        _raise_if(L, L.pbd_op_linear_static(M, K, N, r, scale, x.data_ptr(), W.data_ptr(), _ptr(A) if r else None,
                                            _ptr(B) if r else None, y.data_ptr(), st))
        if sync:
            _raise_if(L, L.pbd_op_linear_static_status(st, None))
    return y


def pbd_op_linear_static_status(device=None) -> int:
    """Device code of the last pbd_op_linear_static call on `device` (0 = none); raises PbdError
    on PBD_ERR_DEVICE, PBD_ERR_STATE (no call yet) or PBD_ERR_CUDA."""
    import torch
    L = load()
    dev = torch.device(device) if device is not None else torch.device("cuda", torch.cuda.current_device())
    code = C.c_int32(0)
    with torch.cuda.device(dev):
        s = L.pbd_op_linear_static_status(torch.cuda.current_stream(dev).cuda_stream, C.byref(code))
    if s != PBD_OK:
        raise PbdError(s, L.pbd_op_last_error().decode())
    return code.value


def pbd_op_lm_head_argmax(x, E, want_logits: bool = False):
    """(argmax ids [M] int32, logits [M, V] fp32 or None) of x E^T on the GPU.
    Waits for the result and raises PbdError(PBD_ERR_DEVICE) if a kernel latched an error."""
    import torch
    L = load()
    M, H = x.shape
    V = E.shape[0]
    need = L.pbd_op_lm_head_workspace_bytes(M, H, V)
    if need == 0:
        raise PbdError(1, "pbd_op_lm_head_argmax: unsupported sizes")
    with torch.cuda.device(x.device):
        buf, ws = _ws(torch, need, x.device)
        ids = torch.empty(M, dtype=torch.int32, device=x.device)
        lg = torch.empty(M, V, dtype=torch.float32, device=x.device) if want_logits else None
        st = torch.cuda.current_stream(x.device).cuda_stream
        _raise_if(L, L.pbd_op_lm_head_argmax(M, H, V, x.data_ptr(), E.data_ptr(), ids.data_ptr(), _ptr(lg), ws,
                                             need, st))
        _raise_if(L, L.pbd_op_status(ws, st, None))
    del buf
    return ids, lg


# ------------------------------------------------------------------ a caller's paged cache, and logits


def _bad(who, what):
    raise PbdError(1, "%s: %s" % (who, what))


def _int32(*values):
    """Whether 32 bits hold the numbers (ctypes hands on the low ones of any)."""
    return all(-1 << 31 <= x < 1 << 31 for x in values)


_DTYPES = {"torch.bfloat16": PBD_BF16, "torch.float16": PBD_FP16, "torch.float32": PBD_FP32}


def _dtype(t, who):
    code = _DTYPES.get(str(t.dtype))
    if code is None:
        _bad(who, "unsupported type %s" % t.dtype)
    return code


def _check(who, name, t, like, shape, dtype=None, rows=False):
    """t lies on like's device, has this shape and type, and is contiguous (rows: each t[i] is)."""
    if t.shape == shape and t.dtype == (dtype or like.dtype) and t.device == like.device and t.is_contiguous():
        return  # (the usual case, in one line: a call checks up to five tensors)
    if t.device != like.device:
        _bad(who, "%s is not on the cache's or logits' device" % name)
    if t.shape != shape:
        _bad(who, "%s has shape %s, not %s" % (name, tuple(t.shape), tuple(shape)))
    if t.dtype != (dtype or like.dtype):
        _bad(who, "%s has type %s" % (name, t.dtype))
    if not t.is_contiguous() and not (rows and t[0].is_contiguous() and t.stride(0) >= t[0].numel()):
        _bad(who, "%s is not contiguous" % name)


def _stream(torch, device):
    """The current stream of a device as a cudaStream_t; without the Stream object, whose making takes longer (4 us
    of a call's 30) than the launch."""
    return torch._C._cuda_getCurrentRawStream(device.index)


class OpWorkspace:
    """Scratch for the calls that take one (op_workspace): calls that may overlap in time need one each."""

    def __init__(self, nbytes, device):
        import torch
        if nbytes <= 0:
            raise PbdError(1, "op_workspace: unsupported sizes")
        self.buf = torch.empty(nbytes + 1024, dtype=torch.uint8, device=device)
        self.device, self.nbytes = self.buf.device, nbytes
        self.ptr = self.buf.data_ptr() + (-self.buf.data_ptr()) % 1024


def op_workspace(nbytes: int, device="cuda") -> OpWorkspace:
    return OpWorkspace(nbytes, device)


def _scratch(who, workspace, need, device):
    """The workspace of a call that needs `need` bytes: the caller's, or a new one."""
    if need == 0:
        _bad(who, "unsupported sizes")
    if workspace is None:
        workspace = OpWorkspace(need, device)
    elif workspace.device != device:
        _bad(who, "the workspace is on another device")
    return workspace


class PagedKV:
    """A paged key-value cache of one layer (pbd_kv_pages): a handle that keeps the tensors it was given.

    k, v [n_pages, n_kv_heads, page_size, head_dim] bf16 or fp16, with the same strides, the last one 1 (token-major
    pages: a transposed view); page_table [batch, max_pages] int32, lens [batch] int32; weights and positions
    [batch, n_kv_heads, max_pages * page_size], fp32 and int32, where they are wanted.  The calls read the tensors' present
    contents; what lens and positions say is up to the program, which changes them in place (kv.lens += 1): the handle
    takes no other tensors."""

    _TENSORS = ("k", "v", "page_table", "lens", "weights", "positions")

    def __setattr__(self, name, value):
        if name in self._TENSORS and getattr(self, name, value) is not value:
            _bad("PagedKV", "%s is another tensor than the handle was made for" % name)
        object.__setattr__(self, name, value)

    def __init__(self, k, v, page_table, lens, weights=None, positions=None):
        import torch
        who = "PagedKV"
        if k.dim() != 4 or page_table.dim() != 2:
            _bad(who, "k is [n_pages, n_kv_heads, page_size, head_dim] and page_table [batch, max_pages]")
        if not k.is_cuda or _dtype(k, who) == PBD_FP32:
            _bad(who, "the cache is bf16 or fp16 on a GPU")
        if v.shape != k.shape or v.dtype != k.dtype or v.device != k.device or v.stride() != k.stride():
            _bad(who, "k and v differ in shape, type, device or strides")
        if k.stride(3) != 1:
            _bad(who, "the values of a head are not contiguous")
        B, max_pages = page_table.shape
        n_pages, hkv, ps, D = k.shape
        if not _int32(B, max_pages, n_pages, hkv, ps, D):
            _bad(who, "a size does not fit 32 bits")
        _check(who, "page_table", page_table, k, (B, max_pages), torch.int32)
        _check(who, "lens", lens, k, (B,), torch.int32)
        for name, t, dt in (("weights", weights, torch.float32), ("positions", positions, torch.int32)):
            if t is not None:
                _check(who, name, t, k, (B, hkv, max_pages * ps), dt)
        self.k, self.v, self.page_table, self.lens = k, v, page_table, lens
        self.weights, self.positions = weights, positions
        self.batch, self.n_kv_heads, self.head_dim, self.device, self.dtype = B, hkv, D, k.device, k.dtype
        self.c = pbd_kv_pages(k.data_ptr(), v.data_ptr(), _dtype(k, who), n_pages, ps, hkv, D, B, max_pages, k.stride(0),
                              k.stride(1), k.stride(2), page_table.data_ptr(), lens.data_ptr(), _ptr(weights),
                              _ptr(positions))
        self.ref = C.byref(self.c)
        self._need = {}


def decode_attention_workspace_bytes(kv: PagedKV, n_q_heads: int, accumulate: bool = False) -> int:
    return load().pbd_op_decode_attention_workspace_bytes(kv.ref, n_q_heads, int(accumulate)) if _int32(n_q_heads) else 0


def pbd_op_decode_attention(q, kv: PagedKV, k_new=None, v_new=None, new_positions=None, scale: Optional[float] = None,
                            accumulate: bool = False, out=None, want_lse: bool = False, workspace=None,
                            sync: bool = True):
    """(out [batch, n_q_heads, head_dim], lse [batch, n_q_heads] fp32 or None): attention of one new token a sequence over
    a paged cache; see include/pbd_ops.h.  q [batch, n_q_heads, head_dim]; k_new, v_new [batch, n_kv_heads, head_dim]: the
    token's own K and V, stored into the cache first, with new_positions [batch] int32 into its positions; scale is
    1/sqrt(head_dim) when not given; accumulate adds the attention weights to the cache's.  With sync, waits and raises
    PbdError(PBD_ERR_DEVICE) for a length or page outside the cache; without (as in a graph's capture), ask
    pbd_op_status(workspace)."""
    import torch
    who = "pbd_op_decode_attention"
    dev = kv.device
    if torch.cuda.current_device() != dev.index:  # the library runs on the current device
        with torch.cuda.device(dev):
            return pbd_op_decode_attention(q, kv, k_new, v_new, new_positions, scale, accumulate, out, want_lse, workspace, sync)
    L = load()
    B, D, hkv = kv.batch, kv.head_dim, kv.n_kv_heads
    if q.dim() != 3:
        _bad(who, "q is [batch, n_q_heads, head_dim]")
    hq = q.shape[1]
    _check(who, "q", q, kv, (B, hq, D), None, True)
    new_stride = 0
    if k_new is not None and v_new is not None:
        _check(who, "k_new", k_new, kv, (B, hkv, D), None, True)
        _check(who, "v_new", v_new, kv, (B, hkv, D), None, True)
        new_stride = k_new.stride(0) if B > 1 else hkv * D
        if B > 1 and v_new.stride(0) != new_stride:
            _bad(who, "rows of k_new and v_new lie differently far apart")
        if new_positions is not None:
            _check(who, "new_positions", new_positions, kv, (B,), torch.int32)
    elif k_new is not None or v_new is not None or new_positions is not None:
        _bad(who, "k_new and v_new come together, and new_positions with them")
    if out is None:
        out = torch.empty((B, hq, D), dtype=kv.dtype, device=dev)
    else:
        _check(who, "out", out, kv, (B, hq, D))
    need = kv._need.get((hq, accumulate))
    if need is None:  # (sizes of a handle do not change)
        need = kv._need[hq, accumulate] = decode_attention_workspace_bytes(kv, hq, accumulate)
    ws = _scratch(who, workspace, need, dev)
    lse = torch.empty((B, hq), dtype=torch.float32, device=dev) if want_lse else None
    st = _stream(torch, dev)
    s = L.pbd_op_decode_attention(kv.ref, hq, D ** -0.5 if scale is None else scale, q.data_ptr(),
                                  q.stride(0) if B > 1 else hq * D, _ptr(k_new), _ptr(v_new), new_stride,
                                  _ptr(new_positions), accumulate, out.data_ptr(), _ptr(lse), ws.ptr, ws.nbytes, st)
    _raise_if(L, s)
    if sync:
        _raise_if(L, L.pbd_op_status(ws.ptr, st, None))
    return out, lse


def evict_workspace_bytes(kv: PagedKV, n_keep: int) -> int:
    return load().pbd_op_evict_workspace_bytes(kv.ref, n_keep) if _int32(n_keep) else 0


def pbd_op_evict(kv: PagedKV, n_keep: int, next_positions, n_recent: int = 0, n_sink: int = 0, out_weights=None,
                 out_positions=None, workspace=None, sync: bool = True):
    """(weights, positions) of the kept slots: of each sequence and KV head the n_keep slots of largest accumulated weight
    stay, the tokens at positions below n_sink and from next_positions [batch] int32 - n_recent on among them; see
    include/pbd_ops.h.  K and V move in place; weights and positions go to out_weights and out_positions, the cache's own
    where they are not given.  The program lowers kv.lens to at most n_keep once all layers that share it are through."""
    import torch
    who = "pbd_op_evict"
    dev = kv.device
    if torch.cuda.current_device() != dev.index:  # the library runs on the current device
        with torch.cuda.device(dev):
            return pbd_op_evict(kv, n_keep, next_positions, n_recent, n_sink, out_weights, out_positions, workspace, sync)
    L = load()
    if kv.weights is None or kv.positions is None:
        _bad(who, "the cache has no weights or positions")
    if out_weights is None and out_positions is None:
        out_weights, out_positions = kv.weights, kv.positions
    elif out_weights is None or out_positions is None:
        _bad(who, "out_weights and out_positions come together")
    else:
        _check(who, "out_weights", out_weights, kv, kv.weights.shape, torch.float32)
        _check(who, "out_positions", out_positions, kv, kv.weights.shape, torch.int32)
    if not (-1 << 31 <= n_recent < 1 << 31 and -1 << 31 <= n_sink < 1 << 31):
        _bad(who, "n_recent or n_sink does not fit 32 bits")
    _check(who, "next_positions", next_positions, kv, (kv.batch,), torch.int32)
    need = kv._need.get(n_keep)
    if need is None:  # (sizes of a handle do not change)
        need = kv._need[n_keep] = evict_workspace_bytes(kv, n_keep) if n_keep >= 0 else 0
    ws = _scratch(who, workspace, need, dev)
    st = _stream(torch, dev)
    s = L.pbd_op_evict(kv.ref, n_keep, n_recent, n_sink, next_positions.data_ptr(), out_weights.data_ptr(),
                       out_positions.data_ptr(), ws.ptr, ws.nbytes, st)
    _raise_if(L, s)
    if sync:
        _raise_if(L, L.pbd_op_status(ws.ptr, st, None))
    return out_weights, out_positions


class TokenLogprobs(NamedTuple):
    logprob: object       # [M] fp32, or None without tokens
    entropy: object       # [M] fp32
    top_ids: object       # [M, k] int32, or None for k = 0
    top_logprobs: object  # [M, k] fp32, or None for k = 0


def token_logprobs_workspace_bytes(M: int, V: int, k: int = 0) -> int:
    return load().pbd_op_token_logprobs_workspace_bytes(M, V, k) if _int32(M, V, k) else 0


def pbd_op_token_logprobs(logits, tokens=None, k: int = 0, temperature: float = 1.0, workspace=None, sync: bool = True):
    """TokenLogprobs of logits [M, V] (fp32, bf16 or fp16; rows may lie apart): log probability of tokens [M] int32 (a
    negative one: none), entropy, and the k likeliest ids with theirs; see include/pbd_ops.h.  With sync, waits and raises
    PbdError(PBD_ERR_DEVICE) for a token at or above V; without, ask pbd_op_status(workspace)."""
    import torch
    who = "pbd_op_token_logprobs"
    dev = logits.device
    if logits.dim() != 2 or dev.type != "cuda":
        _bad(who, "logits are [M, V] on a GPU")
    if torch.cuda.current_device() != dev.index:  # the library runs on the current device
        with torch.cuda.device(dev):
            return pbd_op_token_logprobs(logits, tokens, k, temperature, workspace, sync)
    L = load()
    M, V = logits.shape
    if V > 1 and logits.stride(1) != 1:
        _bad(who, "the values of a row are not contiguous")
    dt = _dtype(logits, who)
    logprob = ids = top = None
    if tokens is not None:
        _check(who, "tokens", tokens, logits, (M,), torch.int32)
    if M >> 31 or V >> 31 or not -1 << 31 <= k < 1 << 31:  # (_int32, without its call)
        _bad(who, "a size does not fit 32 bits")
    ws = _scratch(who, workspace, L.pbd_op_token_logprobs_workspace_bytes(M, V, k), dev)
    entropy = torch.empty(M, dtype=torch.float32, device=dev)
    if tokens is not None:
        logprob = torch.empty(M, dtype=torch.float32, device=dev)
    if k:
        ids = torch.empty((M, k), dtype=torch.int32, device=dev)
        top = torch.empty((M, k), dtype=torch.float32, device=dev)
    st = _stream(torch, dev)
    s = L.pbd_op_token_logprobs(M, V, dt, logits.data_ptr(), logits.stride(0) if M > 1 else V, temperature, _ptr(tokens),
                                k, _ptr(logprob), entropy.data_ptr(), _ptr(ids), _ptr(top), ws.ptr, ws.nbytes, st)
    _raise_if(L, s)
    if sync:
        _raise_if(L, L.pbd_op_status(ws.ptr, st, None))
    return TokenLogprobs(logprob, entropy, ids, top)


def pbd_op_status(workspace: OpWorkspace) -> None:
    """Waits for the current stream and raises PbdError(PBD_ERR_DEVICE) if the last call that used the workspace latched an
    error."""
    import torch
    L = load()
    with torch.cuda.device(workspace.device):
        _raise_if(L, L.pbd_op_status(workspace.ptr, _stream(torch, workspace.device), None))


def make_config(shape, block_D: int, max_batch: int, max_seq_len: int, draft_layers: int = 0,
                denoise_steps: int = 1, anchored: bool = True, draft_skip: int = 0, max_ctas: int = 0) -> pbd_config:
    """pbd_config for a model shape; the draft variant defaults to the method of Section 3."""
    return pbd_config(shape.n_layers, shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                      shape.intermediate, shape.vocab, shape.rms_eps, shape.rope_theta, shape.lora_rank,
                      shape.lora_alpha / shape.lora_rank, block_D, max_batch, max_seq_len, 16,
                      draft_layers, denoise_steps, 0 if anchored else 1, draft_skip, max_ctas)


def pbd_plan_pass(cfg: pbd_config, kind: int, prompt_lens: Sequence[int], max_new: int, grid: int,
                  cap: int = 1 << 20):
    """(items [n, 8] int32, cta_off [grid + 1] int32) of one pass's schedule, host only: per item
    {op | lin << 8 | layer << 16, a, b, c, wait counter, wait target, release counters 0, 1}."""
    L = load()
    lens = np.ascontiguousarray(np.asarray(prompt_lens, dtype=np.int32))
    items = np.zeros((cap, 8), np.int32)
    off = np.zeros(grid + 1, np.int32)
    n = np.zeros(1, np.int32)
    s = L.pbd_plan_pass(C.byref(cfg), kind, len(lens), lens.ctypes.data, max_new, grid, items.ctypes.data,
                        off.ctypes.data, cap, n.ctypes.data)
    if s != PBD_OK:
        raise PbdError(s, (L.pbd_last_error(None) or b"").decode())
    return items[: int(n[0])].copy(), off


def _ptr(t) -> int:
    return t.data_ptr() if t is not None else None


class Engine:
    """One pbd context on one GPU: owns the workspace and a private CUDA stream."""

    def __init__(self, shape, base: Dict[str, np.ndarray], adapter: Dict[str, np.ndarray], block_D: int,
                 max_batch: int, max_seq_len: int, device: str = "cuda:0", keep_host_weights: bool = False,
                 draft_layers: int = 0, denoise_steps: int = 1, anchored: bool = True, draft_skip: int = 0,
                 max_ctas: int = 0):
        import torch
        self.torch = torch
        self.lib = load()
        self.shape = shape
        self.D = block_D
        self.device = torch.device(device)
        self.cfg = make_config(shape, block_D, max_batch, max_seq_len, draft_layers, denoise_steps, anchored,
                               draft_skip, max_ctas)
        need = self.lib.pbd_workspace_bytes(C.byref(self.cfg))
        if need == 0:
            raise PbdError(1, "configuration rejected by pbd_workspace_bytes")
        self.workspace = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        self.stream = torch.cuda.Stream(device=self.device)

        def dev(a):
            return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(self.device).view(torch.bfloat16)

        bw = pbd_base_weights()
        tmp = {}
        for k in ("embed", "final_norm", "attn_norm", "mlp_norm", "q_norm", "k_norm"):
            tmp[k] = dev(base[k])
            setattr(bw, k, _ptr(tmp[k]))
        for i, n in enumerate(LINEARS):
            tmp["w" + n] = dev(base["w" + n])
            bw.w[i] = _ptr(tmp["w" + n])
        aw = pbd_adapter_weights()
        for i, n in enumerate(LINEARS):
            tmp["a_" + n] = dev(adapter["a_" + n])
            tmp["b_" + n] = dev(adapter["b_" + n])
            aw.lora_a[i] = _ptr(tmp["a_" + n])
            aw.lora_b[i] = _ptr(tmp["b_" + n])
        tmp["mask_embed"] = dev(adapter["mask_embed"])
        aw.mask_embed = _ptr(tmp["mask_embed"])
        torch.cuda.synchronize(self.device)
        base_addr = self.workspace.data_ptr()
        aligned = (base_addr + 255) // 256 * 256
        ctx = C.c_void_p()
        self._check(self.lib.pbd_create(C.byref(self.cfg), C.byref(bw), C.byref(aw), aligned,
                                        need + 256 - (aligned - base_addr), self.stream.cuda_stream, C.byref(ctx)),
                    None)
        self.ctx = ctx
        if keep_host_weights:
            self._weights = tmp
        del tmp
        self.batch = 0
        self.max_new = 0

    # -- helpers
    def _call(self, fn, *args):
        """Run one library call on the engine's stream, ordered after and before torch's current stream."""
        cur = self.torch.cuda.current_stream(self.device)
        self.stream.wait_stream(cur)
        status = fn(self.ctx, *args)
        cur.wait_stream(self.stream)
        self._check(status)

    def _check(self, status: int, ctx=None):
        if status != PBD_OK:
            msg = self.lib.pbd_last_error(ctx if ctx is not None else getattr(self, "ctx", None))
            raise PbdError(status, (msg or b"").decode())

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.pbd_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _i32(self, n):
        return self.torch.empty(n, dtype=self.torch.int32, device=self.device)

    # -- C ABI calls, same names
    def pbd_prefill(self, prompts: Sequence[np.ndarray], max_new: int):
        torch = self.torch
        lens = np.array([len(p) for p in prompts], dtype=np.int32)
        packed = torch.from_numpy(np.concatenate([np.asarray(p, np.int32) for p in prompts])).to(self.device)
        first = self._i32(len(prompts))
        self._call(self.lib.pbd_prefill, len(prompts), packed.data_ptr(), lens.ctypes.data, max_new,
                   first.data_ptr())
        self.batch, self.max_new = len(prompts), max_new
        return first

    def pbd_draft_block(self, want_logits: bool = False):
        d = self._i32(self.batch * self.D)
        lg = (self.torch.empty(self.batch * self.D * self.shape.vocab, dtype=self.torch.float32, device=self.device)
              if want_logits else None)
        self._call(self.lib.pbd_draft_block, d.data_ptr(), _ptr(lg))
        return d.view(self.batch, self.D), (lg.view(self.batch, self.D, -1) if lg is not None else None)

    def pbd_verify_block(self, drafts=None, want_logits: bool = False):
        v = self._i32(self.batch * (self.D + 1))
        lg = (self.torch.empty(self.batch * (self.D + 1) * self.shape.vocab, dtype=self.torch.float32,
                               device=self.device) if want_logits else None)
        dp = None
        if drafts is not None:
            drafts = self.torch.as_tensor(drafts, dtype=self.torch.int32).to(self.device).contiguous()
            dp = drafts.data_ptr()
        self._call(self.lib.pbd_verify_block, dp, v.data_ptr(), _ptr(lg))
        return v.view(self.batch, self.D + 1), (lg.view(self.batch, self.D + 1, -1) if lg is not None else None)

    def pbd_accept_commit(self, forced_n=None):
        n = self._i32(self.batch)
        fp = None
        if forced_n is not None:
            forced_n = self.torch.as_tensor(forced_n, dtype=self.torch.int32).to(self.device).contiguous()
            fp = forced_n.data_ptr()
        self._call(self.lib.pbd_accept_commit, fp, n.data_ptr())
        return n

    def pbd_decode_step(self, want_logits: bool = False):
        t = self._i32(self.batch)
        lg = (self.torch.empty(self.batch * self.shape.vocab, dtype=self.torch.float32, device=self.device)
              if want_logits else None)
        self._call(self.lib.pbd_decode_step, t.data_ptr(), _ptr(lg))
        return t, (lg.view(self.batch, -1) if lg is not None else None)

    def pbd_generate(self, prompts: Sequence[np.ndarray], max_new: int, mode: int = 0, forced_n_seq=None):
        torch = self.torch
        lens = np.array([len(p) for p in prompts], dtype=np.int32)
        packed = torch.from_numpy(np.concatenate([np.asarray(p, np.int32) for p in prompts])).to(self.device)
        out = self._i32(len(prompts) * max_new)
        fp = None
        if forced_n_seq is not None:
            forced_n_seq = torch.as_tensor(forced_n_seq, dtype=torch.int32).to(self.device).contiguous()
            fp = forced_n_seq.data_ptr()
        st = pbd_stats()
        self._call(self.lib.pbd_generate, len(prompts), packed.data_ptr(), lens.ctypes.data, max_new,
                   mode, fp, out.data_ptr(), C.byref(st))
        self.batch, self.max_new = len(prompts), max_new
        return out.view(len(prompts), max_new), st

    def pbd_get_state(self):
        n = max(self.batch, 1)
        L = np.zeros(n, np.int32)
        p = np.zeros(n, np.int32)
        o = np.zeros(n, np.int32)
        self._call(self.lib.pbd_get_state, L.ctypes.data, p.ctypes.data, o.ctypes.data)
        return L, p, o

    def pbd_get_tokens(self):
        out = self._i32(self.batch * self.max_new)
        self._call(self.lib.pbd_get_tokens, out.data_ptr())
        self.pbd_sync()
        return out.view(self.batch, self.max_new)

    def pbd_read_kv(self, layer: int, seq: int, n: int):
        w = self.shape.n_kv_heads * self.shape.head_dim
        k = self.torch.empty(n * w, dtype=self.torch.bfloat16, device=self.device)
        v = self.torch.empty(n * w, dtype=self.torch.bfloat16, device=self.device)
        self._call(self.lib.pbd_read_kv, layer, seq, n, k.data_ptr(), v.data_ptr())
        self.pbd_sync()
        return k.view(n, w), v.view(n, w)

    def pbd_sync(self):
        self._call(self.lib.pbd_sync)

    def pbd_bench_rounds(self, mode: int, warmup: int, steps: int, forced_n_seq=None):
        """Returns (ms_draft, ms_verify_or_ar, ms_commit, ms_total, launches_per_round) summed over the steps."""
        ms = np.zeros(4, np.float64)
        launches = np.zeros(1, np.int32)
        fp = None
        if forced_n_seq is not None:
            forced_n_seq = self.torch.as_tensor(forced_n_seq, dtype=self.torch.int32).to(self.device).contiguous()
            fp = forced_n_seq.data_ptr()
        self._call(self.lib.pbd_bench_rounds, mode, warmup, steps, fp, ms.ctypes.data, launches.ctypes.data)
        return float(ms[0]), float(ms[1]), float(ms[2]), float(ms[3]), int(launches[0])

    def pbd_trace_pass(self, kind: int, cap: int = 400000):
        """(items [n, 4] int32 {op|lin<<8|layer<<16, a, b, c}, stamps [n, 16] uint64 ns) of one traced pass."""
        items = np.zeros(cap * 4, np.int32)
        tr = np.zeros(cap * TRACE_STAMPS, np.uint64)
        n = np.zeros(1, np.int32)
        self._call(self.lib.pbd_trace_pass, kind, items.ctypes.data, tr.ctypes.data, cap, n.ctypes.data)
        k = int(n[0])
        return items[: 4 * k].reshape(k, 4), tr[: TRACE_STAMPS * k].reshape(k, TRACE_STAMPS)

    def pbd_check_stalled_pass(self):
        """(status, device code) of passes made to wait in vain (see include/pbd.h)."""
        code = np.zeros(1, np.int32)
        status = self.lib.pbd_check_stalled_pass(self.ctx, code.ctypes.data)
        return int(status), int(code[0])

    def pbd_time_pass(self, kind: int, iters: int):
        """(ms per pass, algorithmic bytes per pass) of the decoder layers of one pass timed alone
        (kind 0 draft, 1 verify, 2 plain decoding)."""
        ms = np.zeros(1, np.float64)
        nb = np.zeros(1, np.float64)
        self._call(self.lib.pbd_time_pass, kind, iters, ms.ctypes.data, nb.ctypes.data)
        return float(ms[0]), float(nb[0])
