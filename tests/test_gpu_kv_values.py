"""Values of V at the ends of their types' ranges."""
import pytest

import _kv_oracle as ref
from test_gpu_kv_ops import HALF, _check_attention, _handle, _to_gpu, env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n", [40, 20000])  # a cluster a row; the list of tiles
def test_infinite_values_stay_in_their_head_and_dimension(env, n, dtype):  # noqa: F811
    """An infinity among the attended values leaves no finite output where it is, and changes none elsewhere."""
    torch, pbd = env
    c = ref.make_cache(torch, [n], 2, 64, 16, getattr(torch, dtype), extra=0)
    q = torch.randn(1, 6, 64, generator=torch.Generator().manual_seed(1)).to(getattr(torch, dtype))
    want = ref.attention(torch, c, q)[0]
    p, o = int(c["table"][0, 1]), 5
    c["v"][p, 0, o, 33] = float("inf")
    c["v"][p, 1, o, 60] = -float("inf")
    g = _to_gpu(torch, c)
    out, lse = pbd.pbd_op_decode_attention(q.cuda(), _handle(pbd, g), want_lse=True)
    finite = out[0].isfinite().cpu()
    hit = torch.zeros(6, 64, dtype=torch.bool)
    hit[:3, 33] = hit[3:, 60] = True
    assert torch.equal(finite, ~hit)
    patched = torch.where(hit, want["out"].to(out.dtype), out[0].cpu())
    _check_attention(torch, want, patched, lse[0], n, HALF["bf16" if dtype == "bfloat16" else "fp16"])


@pytest.mark.parametrize("n", [40, 20000])
def test_values_up_to_the_documented_size(env, n):  # noqa: F811
    """bf16 values up to 2^123 / slots, fp16 up to the type's largest: products and sums stay in range."""
    torch, pbd = env
    for dtype, size in (("bfloat16", 2.0 ** 123 / n), ("float16", 65504.0)):
        dt = getattr(torch, dtype)
        c = ref.make_cache(torch, [n], 1, 128, 16, dt, extra=0, poison=False)
        c["k"].zero_()  # (equal weights: the largest sums)
        c["v"][:] = torch.where(c["v"] > 1, torch.tensor(size), torch.tensor(size) * 0.5).to(dt)
        q = torch.randn(1, 3, 128).to(dt)
        g = _to_gpu(torch, c)
        out, _ = pbd.pbd_op_decode_attention(q.cuda(), _handle(pbd, g))
        _check_attention(torch, ref.attention(torch, c, q)[0], out[0], None, n, HALF["bf16" if dtype == "bfloat16" else "fp16"])
