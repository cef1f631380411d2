"""Alternatives where the first bound of the selection lets through more groups than its list holds, so that the k-th one
is found bit by bit."""
import pytest

import numpy as np

from test_gpu_logprobs import _check, env  # noqa: F401

GROUP, THREADS, LIST = 32, 256, 512  # logprobs.cu: LP_GROUP, LP_THREADS, LP_LIST


def few_bins(V):
    """Of every run of 256 groups of 32 values, those of threads 0 to 111, which share 28 of the 64 bins, lie above the
    rest: for k = 32 the bound is one of the low groups'."""
    i = np.arange(V)
    return (i // GROUP % THREADS < 112) * 9.0 + i % 1021 / 2048


def groups_let_through(x, k, slices, vector):
    """For each slice of a row that begins on a 16-byte boundary, the groups that reach the k-th largest of the maxima of 64
    bins of four threads.  vector: values of 16 bytes."""
    V = len(x)
    per = -(-(-(-V // vector) + 1) // slices)        # vectors of a slice: (one more for rows that begin elsewhere)
    per = -(-per // THREADS) * THREADS * vector // GROUP  # groups
    top = np.pad(x, (0, -V % GROUP), constant_values=-np.inf).reshape(-1, GROUP).max(1)
    counts = []
    for at in range(0, len(top), per):
        m = top[at:at + per]
        rank = np.empty(len(m), int)
        rank[np.lexsort((np.arange(len(m)), -m))] = np.arange(len(m))
        lane, warp = np.arange(len(m)) % THREADS % 32, np.arange(len(m)) % THREADS // 32
        best = np.full(64, len(m))
        np.minimum.at(best, warp * 8 + lane % 4 + lane // 16 * 4, rank)
        counts.append(int((rank <= np.sort(best)[k - 1]).sum()))
    return counts


@pytest.mark.parametrize("V,slices", [(1_000_000, (1, 2, 4, 8, 10, 16)), (50_000, (1,))])
def test_the_pattern_overflows_the_list(V, slices):
    for vector, drop in ((4, 0), (8, 16), (8, 13)):  # fp32, bf16, fp16
        x = few_bins(V).astype(np.float32)
        if drop:  # (rounded to as many bits of the mantissa fewer)
            x = ((x.view(np.uint32) + (1 << drop - 1)) >> drop << drop).astype(np.uint32).view(np.float32)
        for s in slices:
            assert min(groups_let_through(x, 32, s, vector)) > LIST, (vector, s)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("M", [1, 5])
def test_few_bins_hold_the_largest_groups(env, M, dtype):  # noqa: F811
    """However many slices a row has."""
    torch, pbd = env
    x = torch.from_numpy(few_bins(1_000_000)).to(getattr(torch, dtype))
    x = torch.stack([x.roll(THREADS * GROUP * j) + j for j in range(M)]).contiguous()
    tokens = torch.arange(M, dtype=torch.int32) * 3001
    _check(torch, pbd, x, tokens, 32, 1.0)
    _check(torch, pbd, x, tokens, 29, 1.0)
    _check(torch, pbd, x, tokens, 5, 1.0)


@pytest.mark.gpu
def test_few_bins_in_rows_of_one_slice(env):  # noqa: F811
    """More rows than CTAs run at once: one slice each, and some CTAs take two rows."""
    torch, pbd = env
    x = torch.from_numpy(few_bins(50_000)).bfloat16()
    x = torch.stack([x.roll(THREADS * GROUP * (j % 7)) for j in range(470)])
    _check(torch, pbd, x, torch.arange(470, dtype=torch.int32) * 31, 32, 1.0)
