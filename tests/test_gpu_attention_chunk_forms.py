"""Attention of new tokens: the kernels' forms for every head size, for 256 rows a workgroup and for eight wavefronts of few rows."""
import math

import pytest
import torch

import paper_1910_00178_amd as ng
from attention_ref import check
from test_gpu_attention import F16, BF16, ctx, gen  # noqa: F401
from test_gpu_attention_chunk import make, run, wanted, weights

pytestmark = pytest.mark.gpu


def compare(ctx, seed, heads, new, starts, dtype, window=(0, 0), how="packed", shared=None):  # noqa: F811
    """shared: whether the call shares keys out, which its workspace tells."""
    if shared is not None:
        longest = max(a + b for a, b in zip(new, starts))
        assert (ng.ngemm_attention_chunk_workspace_bytes(len(new), *heads, sum(new), max(new), longest, *window) > 0) == shared
    cache, table, q = make(seed, heads, new, starts, dtype, page=64)
    scale = 1 / math.sqrt(heads[2])
    got = run(ctx, cache, table, q, new, starts, *window, scale, how=how)
    check(got, *wanted(cache, table, q, new, starts, *window, scale), dtype, weights=weights(heads, new, dtype))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("window", [(0, 0), (70, 5)], ids=["all", "window"])
@pytest.mark.parametrize("D", range(16, 257, 16))
def test_head_sizes(ctx, D, window, dtype):  # noqa: F811
    for new, starts in (([1, 2, 1], [0, 70, 900]), ([9, 12], [40, 700]), ([100, 3], [500, 17]), ([70], [10])):
        compare(ctx, D, (2, 1, D), new, starts, dtype, window)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("window", [(0, 0), (300, 70)], ids=["all", "window"])
@pytest.mark.parametrize("D", range(16, 193, 16))
def test_eight_wavefronts(ctx, D, window, dtype):  # noqa: F811
    """A tile's keys by the wavefronts of one workgroup: 35 sequences of 4 K/V heads, more tiles than wavefronts in some, fewer in others."""
    g = gen(D)
    starts = [int(n) for n in torch.randint(0, 1200, (35,), generator=g)]
    compare(ctx, D, (8, 4, D), [1 + b % 3 for b in range(35)], starts, dtype, window, shared=False)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("window", [(0, 0), (1100, 70)], ids=["all", "window"])
@pytest.mark.parametrize("how", ["packed", "odd"])
@pytest.mark.parametrize("D", [16, 48, 64, 80, 96, 112, 128])
def test_wide(ctx, D, how, window, dtype):  # noqa: F811
    """256 rows a workgroup, keys shared out: whole tiles, wavefronts without rows, sequences shorter than a tile beside them."""
    compare(ctx, D, (2, 1, D), [200, 140], [1500, 900], dtype, window, how, shared=True)
    compare(ctx, D + 1, (1, 1, D), [700, 1, 259], [900, 900, 0], dtype, window, how, shared=True)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("window", [(0, 0), (1100, 4)], ids=["all", "window"])
@pytest.mark.parametrize("D", [64, 80, 96, 128])
def test_wide_whole(ctx, D, window, dtype):  # noqa: F811
    """256 rows a workgroup, enough tiles for the device: each takes all of its keys."""
    compare(ctx, D, (32, 32, D), [300, 257, 256, 1, 311, 290, 299, 400], [1000, 0, 30, 1100, 1000, 200, 511, 800], dtype, window, shared=False)
