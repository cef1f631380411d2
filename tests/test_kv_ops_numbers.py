"""Numbers that 32 bits do not hold are refused by the binding, which would hand on what is left of them."""
import ctypes as C

import pytest

from paper_2607_12422_gb300 import pbd
from test_kv_ops_args import cache, lib  # noqa: F401


def test_workspace_sizes(lib):  # noqa: F811
    class Handle:
        c = cache()
        ref = C.byref(c)

    for big in (1 << 32, -(1 << 32)):
        for M, V, k in ((2 + big, 100, 4), (2, 100 + big, 4), (2, 100, 4 + big)):
            assert pbd.token_logprobs_workspace_bytes(M, V, k) == 0, (M, V, k)
        assert pbd.evict_workspace_bytes(Handle, 16 + big) == 0
        assert pbd.decode_attention_workspace_bytes(Handle, 4 + big) == 0
    assert pbd.token_logprobs_workspace_bytes(2, 100, 4) > 0 and pbd.evict_workspace_bytes(Handle, 16) > 0
    assert pbd.decode_attention_workspace_bytes(Handle, 4) > 0


@pytest.mark.gpu
def test_calls():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import _kv_oracle as ref
    from test_gpu_kv_ops import _handle, _to_gpu
    c = ref.make_cache(torch, [40, 40], 2, 64, 16, torch.bfloat16, poison=False)
    g = _to_gpu(torch, c)
    kv = _handle(pbd, g, weights=g["weights"], positions=g["positions"])
    big = 1 << 32
    x = torch.randn(3, 50, device="cuda")
    for f in (lambda: pbd.pbd_op_evict(kv, 8 + big, g["lens"]), lambda: pbd.pbd_op_evict(kv, 8, g["lens"], n_recent=2 + big),
              lambda: pbd.pbd_op_evict(kv, 8, g["lens"], n_sink=2 - big), lambda: pbd.pbd_op_token_logprobs(x, k=2 + big),
              # more rows than 32 bits count, all of them the same one
              lambda: pbd.pbd_op_token_logprobs(x[:1, :1].expand(big + 3, 1))):
        with pytest.raises(pbd.PbdError) as e:
            f()
        assert e.value.status == 1
    torch.cuda.synchronize()
    assert torch.equal(g["weights"].cpu(), c["weights"]) and torch.equal(g["k"].cpu(), c["k"])
