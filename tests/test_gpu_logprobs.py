"""Token log probabilities, entropy and top alternatives against the same in 64 bits."""
import math

import pytest

import _kv_oracle as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_12422_gb300 import pbd
    pbd.load()
    return torch, pbd


def _check(torch, pbd, x, tokens, k, T, view=None):
    """x on the CPU.  Errors: the sum of a row runs over at most V / 256 values a thread (in fp32, 2^-24 each) and some 16
    joins; a term's exponent t carries 2 roundings, so the term is off by |t| 2^-23 + 2^-22 of itself, which over the row is
    (entropy + 2) 2^-22 at most.  ln S is off by that, and by its own rounding; a log probability by two more."""
    got = pbd.pbd_op_token_logprobs(x.cuda() if view is None else view, tokens.cuda(), k=k, temperature=T)
    lp, ent, ids, top = ref.logprobs(torch, x, tokens, k, T)
    rel = (x.shape[1] / 256 + 32) * 2.0 ** -24 + (ent + 2) * 2.0 ** -22
    def near(a, b, tol):
        a = a.cpu().double()
        ok = (a == b) | ((a - b).abs() <= tol)
        assert ok.all(), (float(((a - b).abs() / tol)[~ok].max()), a[~ok][:4], b[~ok][:4])
    near(got.logprob, lp, rel + lp.abs().nan_to_num(posinf=0) * 2.0 ** -21)
    near(got.entropy, ent, rel * (1 + ent) * 2 + ent * 2.0 ** -21)
    if k:
        assert torch.equal(got.top_ids.cpu().long(), ids)
        near(got.top_logprobs, top, rel[:, None] + top.abs().nan_to_num(posinf=0) * 2.0 ** -21)
    else:
        assert got.top_ids is None and got.top_logprobs is None
    return got


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("M,V,k,T", [(1, 1, 1, 1.0), (1, 7, 7, 1.0), (3, 31, 5, 0.5), (2, 257, 32, 1.0), (5, 1000, 0, 1.0),
                                     (1, 32003, 20, 1.3), (17, 4096, 32, 1.0), (2, 50001, 1, 0.7), (700, 2049, 8, 1.0),
                                     (1, 151936, 20, 1.0), (620, 20001, 20, 1.0)])
def test_random_logits(env, M, V, k, T, dtype):
    torch, pbd = env
    g = torch.Generator().manual_seed(M + V)
    x = (torch.randn(M, V, generator=g) * 3).to(getattr(torch, dtype))
    _check(torch, pbd, x, torch.randint(0, V, (M,), generator=g, dtype=torch.int32), k, T)


ORDERS = {
    "rising": lambda t, V: t.arange(V) / 1000.0,          # every value is above all before it: the list overflows
    "falling": lambda t, V: -t.arange(V) / 1000.0,
    "equal": lambda t, V: t.zeros(V),                     # ties: the lowest ids
    "two values": lambda t, V: (t.arange(V) % 7 == 3).float(),
    "late": lambda t, V: (t.arange(V) >= V - 40).float() * 5 + t.arange(V) * 1e-6,
    "steps": lambda t, V: (t.arange(V) // 3000).float(),
    # every second run of 31 groups of 64 bytes above the rest, for both sizes of values
    "comb": lambda t, V: ((t.arange(V) // 16 % 64 < 31) * 9).float() + t.arange(V) % 1021 / 2048,
    "wide comb": lambda t, V: ((t.arange(V) // 32 % 64 < 31) * 9).float() + t.arange(V) % 1021 / 2048,
}


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("M", [1, 640])
@pytest.mark.parametrize("order", list(ORDERS))
def test_orders_and_ties(env, order, M, dtype):
    """Orders that defeat a threshold from the first tile, and equal values, in one slice a row and in several."""
    torch, pbd = env
    V = 150000 if "comb" in order else 40000
    M = min(M, 20) if "comb" in order else M
    x = ORDERS[order](torch, V).to(getattr(torch, dtype)).repeat(M, 1)
    _check(torch, pbd, x, torch.arange(M, dtype=torch.int32) * 31, 32, 1.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("columns", [1, 3, 40])
def test_largest_values_that_one_thread_reads(env, columns, dtype):
    """Runs of 32 values every 8192, a thread's part of all tiles, lie above the rest: more of them matter than a thread
    keeps."""
    torch, pbd = env
    V = 500000
    i = torch.arange(V)
    run = i // 32 % 256
    x = ((run % (256 // columns) == 5) & (run < 256 // columns * columns)).float() * 9 + i % 1021 / 2048
    x = torch.stack([x.roll(32 * j) for j in range(12)]).to(getattr(torch, dtype))
    _check(torch, pbd, x, torch.arange(12, dtype=torch.int32) * 31, 32, 1.0)
    _check(torch, pbd, x[:1], torch.zeros(1, dtype=torch.int32), 3, 1.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_masked_logits(env, dtype):
    """-inf and the type's lowest value as masks, in most places, all but one and everywhere; zeros of both signs tie."""
    torch, pbd = env
    dt = getattr(torch, dtype)
    V = 9000
    g = torch.Generator().manual_seed(1)
    x = torch.randn(8, V, generator=g).to(dt)
    x[0, 5:] = -math.inf
    x[1, :] = -math.inf
    x[2, :] = -math.inf
    x[2, 8999] = 3.0
    x[3, 100:] = torch.finfo(dt).min
    x[4, :] = torch.finfo(dt).min
    x[5, ::2], x[5, 1::2] = 0.0, -0.0
    x[6, :4500] = -math.inf
    x[7, 4:] = torch.finfo(dt).min
    got = _check(torch, pbd, x, torch.tensor([2, 2, 8999, 50, 7, 8, 0, -1], dtype=torch.int32), 10, 1.0)
    assert float(got.entropy[1]) == 0 and float(got.logprob[1]) == -math.inf and float(got.logprob[7]) == 0


def test_certain_tokens_keep_their_precision(env):
    """A token of probability almost 1: its log probability and the entropy are small numbers, right to their own size."""
    torch, pbd = env
    x = torch.zeros(3, 1000)
    x[:, 123] = torch.tensor([12.0, 14.0, 40.0])
    got = pbd.pbd_op_token_logprobs(x.cuda(), torch.full((3,), 123, dtype=torch.int32).cuda(), k=2)
    lp, ent, _, _ = ref.logprobs(torch, x, torch.full((3,), 123, dtype=torch.int32), 2, 1.0)
    # The sum is a little over 1 wherever the certain token's term is in it: its thread adds 15 others, then come 5 joins in
    # the warp and 8 of warps, and each of these 28 results is rounded by 2^-24 at most.  The logarithm of a number near 1
    # is off by as much (the terms' own errors are 2^-20 of a sum below 0.007).  The entropy adds an error of its own size.
    off = 28 * 2.0 ** -24
    assert (got.logprob.cpu().double() - lp).abs().max() < off
    assert ((got.entropy.cpu().double() - ent).abs() <= off + ent * 2.0 ** -18).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("M,V", [(1, 1000), (1, 151936), (3, 50000), (460, 20000)])
def test_almost_certain_tokens_to_their_own_size(env, M, V, dtype):
    """One value far above the rest, in any place, after smaller ones: what is left beside its 1 keeps its relative precision.
    The rest is a sum of V terms (V / 256 a thread and some 30 more, 2^-24 each), whose exponents of up to 20 carry two
    roundings (20 * 2^-23), exp2 2^-22; ln(1 + r) and the division two more."""
    torch, pbd = env
    g = torch.Generator().manual_seed(V)
    x = (torch.randn(M, V, generator=g) * 0.5).to(getattr(torch, dtype))
    at = torch.randint(0, V, (M,), generator=g)
    x[torch.arange(M), at] = 24.0
    x[:, V // 3] = torch.maximum(x[:, V // 3], torch.tensor(6.0, dtype=x.dtype))  # an earlier maximum
    got = pbd.pbd_op_token_logprobs(x.cuda(), at.int().cuda(), k=1)
    lp, ent, ids, _ = ref.logprobs(torch, x, at.int(), 1, 1.0)
    z = x.double() - 24.0
    z[torch.arange(M), at] = -math.inf
    rest = z.exp().sum(-1)  # 64 bits, the 1 left out
    rel = (V / 256 + 40) * 2.0 ** -24 + 24 * 2.0 ** -23 + 2.0 ** -21
    assert ((got.logprob.cpu().double() + torch.log1p(rest)).abs() <= torch.log1p(rest) * rel).all()
    want = torch.log1p(rest) + (torch.where(z == -math.inf, torch.zeros_like(z), -z) * z.exp()).sum(-1) / (1 + rest)
    assert ((got.entropy.cpu().double() - want).abs() <= want * 2 * rel).all()
    assert torch.equal(got.top_ids.cpu()[:, 0].long(), at)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("T", [1e-12, 1e-3, 1e4])
def test_extreme_temperatures(env, T, dtype):
    """Near 0 only the maxima count (ties share the probability), far above 1 all values alike; a maximum of 0 and a large one."""
    torch, pbd = env
    x = torch.randn(4, 3000, generator=torch.Generator().manual_seed(4)).to(getattr(torch, dtype))
    x[0] = -x[0].abs()
    x[0, 77], x[1, 5], x[1, 2999], x[2, 1500] = 0.0, 1000.0, 1000.0, -0.0
    got = pbd.pbd_op_token_logprobs(x.cuda(), torch.tensor([77, 2999, 8, 9], dtype=torch.int32).cuda(), k=3, temperature=T)
    # the temperature's inverse in 32 bits, as the kernel has it
    lp, ent, ids, top = ref.logprobs(torch, x, torch.tensor([77, 2999, 8, 9]), 3, 1.0 / float(torch.tensor(1.0) / torch.tensor(T)))
    assert torch.equal(got.top_ids.cpu().long(), ids)
    # (sums as elsewhere; an exponent of n carries n 2^-23, which counts where its term does, below 20 or so)
    for a, b in ((got.logprob, lp), (got.entropy, ent), (got.top_logprobs, top)):
        assert ((a.cpu().double() - b).abs() <= 2.0 ** -17 + b.abs() * 2.0 ** -20).all()


def test_nan_and_infinity(env):
    torch, pbd = env
    x = torch.randn(3, 3000)
    x[0, 77], x[1, 78] = math.nan, math.inf
    got = pbd.pbd_op_token_logprobs(x.cuda(), torch.tensor([1, 1, 1], dtype=torch.int32).cuda(), k=4)
    lp = got.logprob.cpu()
    assert lp[:2].isnan().all() and got.entropy.cpu()[:2].isnan().all() and got.top_logprobs.cpu()[:2].isnan().all()
    ids = got.top_ids.cpu()
    assert ((ids >= 0) & (ids < 3000)).all()
    want = ref.logprobs(torch, x[2:], torch.tensor([1]), 4, 1.0)
    assert abs(float(lp[2]) - float(want[0])) < 1e-5 and torch.equal(ids[2].long(), want[2][0])


def test_rows_apart_and_at_odd_addresses(env):
    """Rows of a wider buffer from an odd column on; what lies between the rows is NaN."""
    torch, pbd = env
    for dt in (torch.float32, torch.float16):
        buf = torch.full((20, 5003), math.nan, dtype=dt)
        for first, V in ((1, 5000), (3, 4999), (7, 13), (0, 5003)):
            x = torch.randn(20, V).to(dt)
            dev = buf.clone()
            dev[:, first:first + V] = x
            _check(torch, pbd, x, torch.randint(0, V, (20,), dtype=torch.int32), 9, 1.0, view=dev.cuda()[:, first:first + V])


def test_tokens_outside_the_vocabulary_are_reported(env):
    torch, pbd = env
    for M in (3, 700):
        x = torch.randn(M, 500).cuda()
        t = torch.zeros(M, dtype=torch.int32).cuda()
        t[1] = 500
        ws = pbd.op_workspace(pbd.token_logprobs_workspace_bytes(M, 500, 2))
        got = pbd.pbd_op_token_logprobs(x, t, k=2, workspace=ws, sync=False)
        assert got.logprob[1].isnan() and got.logprob[0].isfinite()
        with pytest.raises(pbd.PbdError) as e:
            pbd.pbd_op_status(ws)
        assert e.value.status == 6
        t[1] = -1
        pbd.pbd_op_token_logprobs(x, t, k=2, workspace=ws)


def test_logits_of_the_head_and_of_a_verify_block(env):
    """The read-out of one's own hidden states, and of an engine's verify block: the top id is the greedy one."""
    torch, pbd = env
    from paper_2607_12422_gb300 import synth
    g = torch.Generator().manual_seed(2)
    x, E = torch.randn(17, 256, generator=g).bfloat16(), (torch.randn(4096, 256, generator=g) * 0.05).bfloat16()
    ids, logits = pbd.pbd_op_lm_head_argmax(x.cuda(), E.cuda(), want_logits=True)
    got = _check(torch, pbd, logits.cpu(), ids.cpu(), 4, 1.0)
    assert torch.equal(got.top_ids[:, 0], ids) and torch.equal(got.top_logprobs[:, 0], got.logprob)
    S = synth.TINY
    eng = pbd.Engine(S, synth.gen_base_weights(S), synth.gen_adapter(S), block_D=4, max_batch=2, max_seq_len=96)
    eng.pbd_prefill(synth.gen_prompts(S, [40, 23]), max_new=16)
    eng.pbd_draft_block()
    v, lg = eng.pbd_verify_block(want_logits=True)
    rows = lg.view(-1, S.vocab)
    got = _check(torch, pbd, rows.cpu(), v.reshape(-1).cpu(), 3, 1.0, view=rows)
    assert torch.equal(got.top_ids[:, 0], v.reshape(-1))
    eng.close()


def test_refusals(env):
    torch, pbd = env
    x = torch.randn(4, 100).cuda()
    t = torch.zeros(4, dtype=torch.int32).cuda()
    for f in (lambda: pbd.pbd_op_token_logprobs(x.double()), lambda: pbd.pbd_op_token_logprobs(x.cpu()),
              lambda: pbd.pbd_op_token_logprobs(x[0]), lambda: pbd.pbd_op_token_logprobs(x.T),
              lambda: pbd.pbd_op_token_logprobs(x, t.long()), lambda: pbd.pbd_op_token_logprobs(x, t[:2]),
              lambda: pbd.pbd_op_token_logprobs(x, k=33), lambda: pbd.pbd_op_token_logprobs(x[:, :5], k=6),
              lambda: pbd.pbd_op_token_logprobs(x, k=-1), lambda: pbd.pbd_op_token_logprobs(x, temperature=0.0),
              lambda: pbd.pbd_op_token_logprobs(x, temperature=math.nan),
              lambda: pbd.pbd_op_token_logprobs(x, workspace=pbd.op_workspace(16)),
              lambda: pbd.pbd_op_token_logprobs(x[:0])):
        with pytest.raises(pbd.PbdError) as e:
            f()
        assert e.value.status in (1, 2)
